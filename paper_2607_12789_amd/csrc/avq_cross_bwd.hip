// Gradients of cross attention. With the weights P_ij = exp(S_ij - lse_i) again from
// the forward pass's lse:
//
//   delta_i = dY_i . Y_i = sum_j P_ij dP_ij,  dP_ij = dY_i . v_j
//   dS_ij = P_ij (dP_ij - delta_i)
//   dQ_i = scale sum_j dS_ij k_j,  dK_j = scale sum_i dS_ij q_i,  dV_j = sum_i P_ij dY_i
//
// where i runs over all queries of the source and all heads of the group. No sum is
// taken by atomics: one kernel owns rows and runs over the states (dQ), one owns
// states and runs over the rows (dK, dV), which computes P and dP twice: seven
// matrix products (bf16 eight, see below) instead of five, and the same result at every
// call.
//
// bf16: Y is rounded, and so delta_i is off, by the same amount for all j: an error
// that the sums over j do not average out. But sum_j dS_ij is 0, so its sum with that
// delta, rest_i, is what delta_i lacks: dK takes the mended delta, and dQ_i is corrected
// by -scale rest_i sum_j P_ij k_j, a fourth product of that kernel, whose operand is at
// hand. There rest_i is the sum of the dS as they are rounded for the product, whose
// errors then have no part along that sum either. dQ and dK against 64 bits, of their
// norms: 0.0032 to 0.0038 without, 0.0022 to 0.0025 with it, where rounding them alone
// leaves 0.0017; 4096 queries and states, 16/4 heads, d = 128, twice: 885 us without, 959
// with it (both kernels and the join, on one card; 995 to 1065 on others).
//
// Both as the forward kernel: 32 owned rows (or states) per wave, one per lane and
// its partner, the others in tiles of 32 through LDS, double buffered. What a tile
// gives is read row by row for P and dP, and transposed for the gradients.
#include "avq_launch.hpp"

#include <algorithm>

#include "avq_cross.hpp"

namespace avq {

namespace {

// Whole rows are stored at once (store_rows) where that leaves the kernels their
// registers: 4 sources of 4096 queries and 31 to 128 states, 12 heads, bf16, d = 64, 64.2
// us by store_row, 59.6 so; 4096 queries and states twice, d = 128, 1001 and 1065 (8 to 10
// registers spilled; as they are, dQ's kernel spills 3 with a mask, dK's and dV's 1 without
// one), 8 sources of 10 to 3000, fp32, d = 64, 709 and 765.
template <typename T, int D>
constexpr bool kWholeRows = Elem<T>::kBf16 && D == 64;

// ---- dQ: owns rows -------------------------------------------------------------------

template <typename T, int D, bool kMask>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(Elem<T>::kBf16 || D == 64 ? 2 : 1)))
void cross_dq_kernel(CrossArgs a) {
  constexpr int DT = D / 32, ESZ = sizeof(T), U = D * ESZ / 16, TILE = 32 * D * ESZ;
  constexpr bool kB = Elem<T>::kBf16;
  __shared__ __attribute__((aligned(16))) unsigned char k_even[TILE], k_odd[TILE];
  __shared__ __attribute__((aligned(16))) unsigned char v_even[TILE], v_odd[TILE];
  // bf16: dY waits in LDS, for the registers of two waves per SIMD at d = 128
  __shared__ RowFrag<T> s_dy[kCrossWaves][kB ? kRowSteps<T, D> : 1][kWave];
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int h = lane / 32, c = lane % 32;
  CrossTile t;
  if (!find_cross_tile<false>(a, lane, t)) return;
  const int n_tiles = (t.Lk + 31) / 32, hkv = t.hkv, split = t.split, splits = t.splits;
  const int t_begin = (int)((long long)n_tiles * split / splits);
  const int t_end = (int)((long long)n_tiles * (split + 1) / splits);

  const int rows = t.Lq * a.G, row0 = t.lt * kCrossTile + 32 * wave, row = row0 + c;
  const bool has_row = row < rows, wave_has = row0 < rows;
  const int at_row = min(row, rows - 1), qi = t.qa + at_row / a.G, hq = hkv * a.G + at_row % a.G;
  const size_t at = (size_t)qi * a.Hq + hq;

  const T* kbase = static_cast<const T*>(a.K) + (size_t)t.ka * a.k_stride + (size_t)hkv * D;
  const T* vbase = static_cast<const T*>(a.V) + (size_t)t.ka * a.v_stride + (size_t)hkv * D;
  auto kswz = [](int r) { return both_swizzle<U, kB>(r); };
  auto vswz = [](int r) { return key_swizzle<U>(r); };
  auto issue = [&](int i, uint32_t bits, unsigned char* k_to, unsigned char* v_to) {
    if (bits == 0) return;
    stage_states<T, D>(kbase + (size_t)i * 32 * a.k_stride, a.k_stride, bits, k_to, wave, lane,
                       kswz);
    stage_states<T, D>(vbase + (size_t)i * 32 * a.v_stride, a.v_stride, bits, v_to, wave, lane,
                       vswz);
  };
  Seen<kMask> seen;
  uint32_t bits = 0, next = 0;
  if (t_begin < t_end) {
    seen.request(a.mask, t.ka, t.Lk, 32 * t_begin, lane);
    next = seen.bits(t.Lk, 32 * t_begin);
    issue(t_begin, next, k_even, v_even);
    seen.request(a.mask, t.ka, t.Lk, 32 * (t_begin + 1), lane);
  }

  // the row's operands, delta and -lse log2(e) (a row that saw no state: weights 0)
  RowFrag<T> q[kRowSteps<T, D>], dy[kRowSteps<T, D>];
  load_row<T, D>(static_cast<const T*>(a.Q) + (size_t)qi * a.q_stride + (size_t)hq * D, h, q);
  load_row<T, D>(static_cast<const T*>(a.dY) + (size_t)qi * a.dy_stride + (size_t)hq * D, h, dy);
  float delta = 0.f;
  {
    RowFrag<T> y[kRowSteps<T, D>];
    load_row<T, D>(static_cast<const T*>(a.Y) + at * D, h, y);
#pragma unroll
    for (int k = 0; k < kRowSteps<T, D>; ++k) {
      if constexpr (kB) {
#pragma unroll
        for (int e = 0; e < 8; ++e) delta = fmaf((float)y[k][e], (float)dy[k][e], delta);
      } else {
        delta = fmaf(y[k], dy[k], delta);
      }
    }
    delta = add_xor<32>(delta);
  }
  if constexpr (kB) {
#pragma unroll
    for (int k = 0; k < kRowSteps<T, D>; ++k) s_dy[wave][k][lane] = dy[k];
  }
  const float lse = a.lse[at], off = lse == -INFINITY ? -INFINITY : -lse * kLog2e;

  // acc[0]: sum dS k; bf16 also acc[1]: sum P k, rest: sum dS, and rounded: of the dS
  // that the product takes
  constexpr int N = kB ? 2 : 1;
  f32x16 acc[N][DT];
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < DT; ++i) acc[n][i] = f32x16{};
  float rest = 0.f, rounded = 0.f;
  auto step = [&](int i, const unsigned char* kt, const unsigned char* vt, unsigned char* k_next,
                  unsigned char* v_next) {
    bits = next;
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();  // tile i has landed, tile i - 1 is read
    if (i + 1 < t_end) {
      next = seen.bits(t.Lk, 32 * (i + 1));
      issue(i + 1, next, k_next, v_next);
      seen.request(a.mask, t.ka, t.Lk, 32 * (i + 2), lane);
    }
    if (bits == 0 || !wave_has) return;
    f32x16 p = f32x16{}, g = f32x16{};
    row_product<T, D>(kt, lane, c, q, kswz, p);
    if constexpr (kB) {
      RowFrag<T> mine[kRowSteps<T, D>];
#pragma unroll
      for (int k = 0; k < kRowSteps<T, D>; ++k) mine[k] = s_dy[wave][k][lane];
      row_product<T, D>(vt, lane, c, mine, vswz, g);
    } else {
      row_product<T, D>(vt, lane, c, dy, vswz, g);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) p[r] = exp2_hw(fmaf(p[r], a.scale_log2, off));
    if (bits != ~0u) {
      const uint32_t mine = place(bits >> (4 * h));
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (!(mine & 1u << (8 * (r / 4) + r % 4))) p[r] = 0.f;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      g[r] = p[r] * (g[r] - delta);
      if constexpr (kB) rest += g[r];
    }
    if constexpr (kB) {
      const Weights<T> w[2] = {Weights<T>(g), Weights<T>(p)};
      rounded = w[0].sum(rounded);
      column_products<T, D, 2>(kt, lane, w, kswz, acc);
    } else {
      column_product<T, D>(kt, lane, g, kswz, acc[0]);
    }
  };
  for (int i = t_begin; i < t_end; i += 2) {
    step(i, k_even, v_even, k_odd, v_odd);
    if (i + 1 < t_end) step(i + 1, k_odd, v_odd, k_even, v_even);
  }
  if constexpr (kB) rest = add_xor<32>(rest), rounded = add_xor<32>(rounded);
  if (has_row && h == 0 && split == 0) a.delta[at] = splits > 1 ? delta : delta + rest;
  if (splits > 1) {
    if (!has_row) return;
    const size_t rows_all = (size_t)a.Tq * a.Hq, part = split * rows_all + at;
    store_row<float, D>(a.parts + part * D, h, 1.f, acc[0]);
    if constexpr (kB) {
      store_row<float, D>(a.parts + (a.splits * rows_all + part) * D, h, 1.f, acc[1]);
      if (h == 0) {
        a.parts[2 * a.splits * rows_all * D + part] = rest;
        a.parts[a.splits * rows_all * (2 * D + 1) + part] = rounded;
      }
    }
    return;
  }
  if constexpr (kB) {
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[0][i][r] -= rounded * acc[1][i][r];
  }
  if (kWholeRows<T, D> && rows - t.lt * kCrossTile > 32) {
    __syncthreads();  // the last tile is read
    if (!wave_has) return;
    const RowsOf row_of(a, t, row0);
    unsigned char* const area = wave == 0 ? k_even : wave == 1 ? k_odd : wave == 2 ? v_even : v_odd;
    store_rows<T, D, T>(area, lane, a.scale, acc[0], rows - row0,
                        [&](int r) { return static_cast<T*>(a.dQ) + row_of(a, t, r) * D; });
  } else if (has_row) {
    store_row<T, D>(static_cast<T*>(a.dQ) + at * D, h, a.scale, acc[0]);
  }
}

// ---- dK, dV: owns states ---------------------------------------------------------------

template <typename T, int D, bool kMask>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(Elem<T>::kBf16 || D == 64 ? 2 : 1)))
void cross_dkv_kernel(CrossArgs a) {
  constexpr int DT = D / 32, ESZ = sizeof(T), U = D * ESZ / 16, TILE = 32 * D * ESZ;
  constexpr int RPC = 64 / U, CPW = 32 / RPC / kCrossWaves;
  constexpr bool kB = Elem<T>::kBf16;
  // an array for each buffer, and the loop two steps at a time: the compiler then
  // knows that a step's reads do not touch what its copies write, and waits for none
  __shared__ __attribute__((aligned(16))) unsigned char q_even[TILE], q_odd[TILE];
  __shared__ __attribute__((aligned(16))) unsigned char y_even[TILE], y_odd[TILE];
  __shared__ __attribute__((aligned(16))) float s_row[2][2][32];  // -lse log2(e), delta
  __shared__ RowFrag<T> s_v[kCrossWaves][kB ? kRowSteps<T, D> : 1][kWave];
  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int h = lane / 32, c = lane % 32;
  CrossTile t;
  if (!find_cross_tile<true>(a, lane, t)) return;
  const int rows = t.Lq * a.G, n_tiles = (rows + 31) / 32;
  const int hkv = t.hkv, split = t.split, splits = t.splits;
  const int t_begin = (int)((long long)n_tiles * split / splits);
  const int t_end = (int)((long long)n_tiles * (split + 1) / splits);

  const int key0 = t.lt * kCrossTile + 32 * wave, key = key0 + c;
  const bool has_key = key < t.Lk, wave_has = key0 < t.Lk;
  const int at_key = t.ka + min(key, t.Lk - 1);
  const bool seen = has_key && (!kMask || a.mask[at_key] != 0);
  // a state that takes no part may hold anything: it is taken as 0
  RowFrag<T> k[kRowSteps<T, D>], v[kRowSteps<T, D>];
  load_row<T, D>(static_cast<const T*>(a.K) + (size_t)at_key * a.k_stride + (size_t)hkv * D, h, k);
  load_row<T, D>(static_cast<const T*>(a.V) + (size_t)at_key * a.v_stride + (size_t)hkv * D, h, v);
  if (kMask && !seen) {
#pragma unroll
    for (int i = 0; i < kRowSteps<T, D>; ++i) k[i] = RowFrag<T>{}, v[i] = RowFrag<T>{};
  }

  // bf16: the values wait in LDS, in registers they would leave room for one wave per
  // SIMD instead of two at
  // d = 128 (1319 to 1006 us for both kernels, 16 heads of 4096 rows and 4096 states)
  if constexpr (kB) {
#pragma unroll
    for (int i = 0; i < kRowSteps<T, D>; ++i) s_v[wave][i][lane] = v[i];
  }
  const T* qbase = static_cast<const T*>(a.Q) + (size_t)t.qa * a.q_stride + (size_t)hkv * a.G * D;
  const T* ybase = static_cast<const T*>(a.dY) + (size_t)t.qa * a.dy_stride + (size_t)hkv * a.G * D;
  auto swz = [](int r) { return both_swizzle<U, kB>(r); };
  float row_value = 0.f;  // threads 0..31: lse, 32..63: delta of a tile's rows
  auto issue = [&](int i, unsigned char* q_to, unsigned char* y_to) {
    // rows past the source's read its last one
    const int q0 = 32 * i / a.G, head0 = 32 * i % a.G, last = rows - 1 - 32 * i;
    const __amdgpu_buffer_rsrc_t rq = rsrc(qbase + (size_t)q0 * a.q_stride);
    const __amdgpu_buffer_rsrc_t ry = rsrc(ybase + (size_t)q0 * a.dy_stride);
#pragma unroll
    for (int n = 0; n < CPW; ++n) {
      const int j = wave * CPW + n, r = RPC * j + lane / U, x = head0 + min(r, last);
      const int dq = quotient(x, a.g_reciprocal), hd = x - dq * a.G;
      const uint32_t in = (uint32_t)(hd * D * ESZ) + 16u * ((lane % U) ^ swz(r));
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rq, (__attribute__((address_space(3))) void*)(q_to + 1024 * j), 16,
          (uint32_t)dq * (uint32_t)(a.q_stride * ESZ) + in, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          ry, (__attribute__((address_space(3))) void*)(y_to + 1024 * j), 16,
          (uint32_t)dq * (uint32_t)(a.dy_stride * ESZ) + in, 0, 0, 0);
    }
    if (tid < 64) {
      const int x = head0 + min(c, last), dq = quotient(x, a.g_reciprocal);
      const size_t at = (size_t)(t.qa + q0 + dq) * a.Hq + hkv * a.G + (x - dq * a.G);
      row_value = tid < 32 ? a.lse[at] : a.delta[at];
    }
  };

  f32x16 dk[DT], dv[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) dk[i] = f32x16{}, dv[i] = f32x16{};
  if (t_begin < t_end) issue(t_begin, q_even, y_even);
  auto step = [&](int i, int b, const unsigned char* qt, const unsigned char* yt,
                  unsigned char* q_next, unsigned char* y_next) {
    if (tid < 64) {
      // rows past the last one, and rows that saw no state: weights 0
      const bool none = 32 * i + c >= rows || row_value == -INFINITY;
      s_row[b][tid / 32][tid % 32] =
          tid >= 32 ? row_value : none ? -INFINITY : -row_value * kLog2e;
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();  // tile i has landed, tile i - 1 is read
    if (i + 1 < t_end) issue(i + 1, q_next, y_next);
    if (!wave_has) return;
    f32x16 p = f32x16{}, g = f32x16{};
    row_product<T, D>(qt, lane, c, k, swz, p);
    if constexpr (kB) {
      RowFrag<T> mine[kRowSteps<T, D>];
#pragma unroll
      for (int n = 0; n < kRowSteps<T, D>; ++n) mine[n] = s_v[wave][n][lane];
      row_product<T, D>(yt, lane, c, mine, swz, g);
    } else {
      row_product<T, D>(yt, lane, c, v, swz, g);
    }
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const f32x4 off = *reinterpret_cast<const f32x4*>(&s_row[b][0][2 * r + 4 * h]);
      const f32x4 delta = *reinterpret_cast<const f32x4*>(&s_row[b][1][2 * r + 4 * h]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float w = exp2_hw(fmaf(p[r + e], a.scale_log2, off[e]));
        if (kMask) w = seen ? w : 0.f;
        p[r + e] = w;
        g[r + e] = w * (g[r + e] - delta[e]);
      }
    }
    column_product<T, D>(yt, lane, p, swz, dv);
    column_product<T, D>(qt, lane, g, swz, dk);
  };
  for (int i = t_begin; i < t_end; i += 2) {
    step(i, 0, q_even, y_even, q_odd, y_odd);
    if (i + 1 < t_end) step(i + 1, 1, q_odd, y_odd, q_even, y_even);
  }
  if (kMask && !seen) {  // 0 also where a gradient is not finite
#pragma unroll
    for (int i = 0; i < DT; ++i) dk[i] = f32x16{}, dv[i] = f32x16{};
  }
  const size_t at0 = (size_t)(t.ka + key0) * a.Hkv + hkv, rows_all = (size_t)a.Tk * a.Hkv;
  float* const part = a.parts + (split * rows_all + at0) * D;
  if (kWholeRows<T, D> && t.Lk - t.lt * kCrossTile > 32) {
    __syncthreads();  // the last tile is read
    if (!wave_has) return;
    unsigned char* const area = wave == 0 ? q_even : wave == 1 ? q_odd : wave == 2 ? y_even : y_odd;
    const int n = t.Lk - key0;
    if (splits > 1) {
      auto row = [&](int r) { return part + (size_t)r * a.Hkv * D; };
      store_rows<T, D, float>(area, lane, 1.f, dk, n, row);
      store_rows<T, D, float>(area, lane, 1.f, dv, n,
                              [&](int r) { return row(r) + a.splits * rows_all * D; });
    } else {
      auto row = [&](void* out, int r) {
        return static_cast<T*>(out) + (at0 + (size_t)r * a.Hkv) * D;
      };
      store_rows<T, D, T>(area, lane, a.scale, dk, n, [&](int r) { return row(a.dK, r); });
      store_rows<T, D, T>(area, lane, 1.f, dv, n, [&](int r) { return row(a.dV, r); });
    }
    return;
  }
  if (!has_key) return;
  const size_t at = (size_t)at_key * a.Hkv + hkv;
  if (splits > 1) {
    store_row<float, D>(a.parts + (split * rows_all + at) * D, h, 1.f, dk);
    store_row<float, D>(a.parts + ((a.splits + split) * rows_all + at) * D, h, 1.f, dv);
    return;
  }
  store_row<T, D>(static_cast<T*>(a.dK) + at * D, h, a.scale, dk);
  store_row<T, D>(static_cast<T*>(a.dV) + at * D, h, 1.f, dv);
}

long long tiles_of(long long rows, int S) { return rows / kCrossTile + S; }

struct Plan {
  long long row_tiles, state_tiles;
  CrossSplit rows, states;
  size_t delta, parts;  // floats
};
template <typename T, int d>
Plan plan_of(int S, int Tq, int Tk, int Hq, int Hkv) {
  const long long rows = (long long)Tq * (Hq / Hkv);
  Plan p;
  p.row_tiles = tiles_of(rows, S), p.state_tiles = tiles_of(Tk, S);
  // as many workgroups as run at once: 2 per CU, of fp32 at d = 128 one (with 512 of
  // those 1024 rows and states of 8 heads take 190 instead of 175 us)
  constexpr int W = sizeof(T) == 4 && d == 128 ? 256 : 512;
  p.rows = cross_split(rows, Tk, S, Hkv, W, sizeof(T) == 4);
  p.states = cross_split(Tk, rows, S, Hkv, W, sizeof(T) == 4);
  p.delta = ((size_t)Tq * Hq + 3) / 4 * 4;
  // the two kernels' parts lie at the same place: dQ is joined before dK and dV start
  const size_t row = sizeof(T) == 4 ? d : 2 * d + 2;
  const size_t a = p.rows.splits > 1 ? (size_t)Tq * Hq * row * p.rows.splits : 0;
  const size_t b = p.states.splits > 1 ? 2 * (size_t)Tk * Hkv * d * p.states.splits : 0;
  p.parts = std::max(a, b);
  return p;
}

}  // namespace

template <typename T, int D>
size_t cross_attention_bwd_workspace(int S, int Tq, int Tk, int Hq, int Hkv) {
  const Plan p = plan_of<T, D>(S, Tq, Tk, Hq, Hkv);
  return (p.delta + p.parts + (p.parts > 0 ? 4 : 0)) * sizeof(float);  // and CrossArgs::steps
}

template <typename T, int D>
hipError_t launch_cross_attention_bwd(int S, int Tq, int Tk, int Hq, int Hkv, float scale,
                                      const void* Q, int64_t q_stride, const void* K,
                                      int64_t k_stride, const void* V, int64_t v_stride,
                                      const int32_t* cu_q, const int32_t* cu_k,
                                      const uint8_t* mask, const void* Y, const float* lse,
                                      const void* dY, int64_t dy_stride, void* dQ, void* dK,
                                      void* dV, void* workspace, hipStream_t stream) {
  const Plan p = plan_of<T, D>(S, Tq, Tk, Hq, Hkv);
  CrossArgs a{};
  a.Q = Q, a.K = K, a.V = V, a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride;
  a.cu_q = cu_q, a.cu_k = cu_k, a.mask = mask, a.Y = const_cast<void*>(Y);
  a.lse = const_cast<float*>(lse), a.dY = dY, a.dy_stride = dy_stride;
  a.dQ = dQ, a.dK = dK, a.dV = dV;
  a.S = S, a.Tq = Tq, a.Tk = Tk, a.Hq = Hq, a.Hkv = Hkv, a.G = Hq / Hkv;
  a.g_reciprocal = reciprocal_of(a.G);
  a.scale = scale, a.scale_log2 = scale * kLog2e;
  a.delta = static_cast<float*>(workspace), a.parts = a.delta + p.delta;
  a.steps = reinterpret_cast<int32_t*>(a.parts + p.parts);
  hipError_t e = hipSuccess;
  if (Tq > 0) {
    a.slots = cross_slots<T, D>(S, (long long)Tq * a.G, 512);
    a.tiles = (int)p.row_tiles, a.per = p.rows.per, a.splits = p.rows.splits;
    const dim3 grid((unsigned)(a.tiles * Hkv), (unsigned)a.splits);
    if (mask)
      hipLaunchKernelGGL((cross_dq_kernel<T, D, true>), grid, dim3(256), 0, stream, a);
    else
      hipLaunchKernelGGL((cross_dq_kernel<T, D, false>), grid, dim3(256), 0, stream, a);
    e = hipGetLastError();
    if (e == hipSuccess && a.splits > 1) e = launch_cross_join<T, D, kJoinQueries>(a, stream);
  }
  if (e != hipSuccess || Tk == 0) return e;
  a.slots = cross_slots<T, D>(S, Tk, 512);
  a.tiles = (int)p.state_tiles, a.per = p.states.per, a.splits = p.states.splits;
  const dim3 grid((unsigned)(a.tiles * Hkv), (unsigned)a.splits);
  if (mask)
    hipLaunchKernelGGL((cross_dkv_kernel<T, D, true>), grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((cross_dkv_kernel<T, D, false>), grid, dim3(256), 0, stream, a);
  e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  return launch_cross_join<T, D, kJoinStates>(a, stream);
}

#define AVQ_INSTANCE(T, D)                                                                        \
  template hipError_t launch_cross_attention_bwd<T, D>(                                           \
      int, int, int, int, int, float, const void*, int64_t, const void*, int64_t, const void*,    \
      int64_t, const int32_t*, const int32_t*, const uint8_t*, const void*, const float*,         \
      const void*, int64_t, void*, void*, void*, void*, hipStream_t);                             \
  template size_t cross_attention_bwd_workspace<T, D>(int, int, int, int, int);
AVQ_INSTANCE(bf16, 64)
AVQ_INSTANCE(bf16, 128)
AVQ_INSTANCE(float, 64)
AVQ_INSTANCE(float, 128)
#undef AVQ_INSTANCE

}  // namespace avq
