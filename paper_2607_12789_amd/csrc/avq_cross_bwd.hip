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
// matrix products instead of five, and the same result at every call.
//
// Both as the forward kernel: 32 owned rows (or states) per wave, one per lane and
// its partner, the others in tiles of 32 through LDS, double buffered. What a tile
// gives is read row by row for P and dP, and transposed for the gradients.
#include "avq_launch.hpp"

#include <algorithm>
#include <type_traits>

#include "avq_cross.hpp"

namespace avq {

namespace {

constexpr int kLeastTiles = 4;  // tiles of 32 that a workgroup takes, at least

// ---- dQ: owns rows -------------------------------------------------------------------

template <typename T, int D, bool kMask>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(Elem<T>::kBf16 || D == 64 ? 2 : 1)))
void cross_dq_kernel(CrossArgs a) {
  constexpr int DT = D / 32, ESZ = sizeof(T), U = D * ESZ / 16, TILE = 32 * D * ESZ;
  constexpr bool kB = Elem<T>::kBf16;
  __shared__ __attribute__((aligned(16))) unsigned char lds[4 * TILE];  // K0 K1 V0 V1
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int h = lane / 32, c = lane % 32;
  const int hkv = blockIdx.x % a.Hkv, tile = blockIdx.x / a.Hkv;
  CrossTile t;
  if (!find_cross_tile<false>(a, tile, lane, t)) return;
  const int n_tiles = (t.Lk + 31) / 32, splits = splits_of<kLeastTiles>(a, n_tiles);
  const int split = blockIdx.y;
  if (split >= splits) return;
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
  auto issue = [&](int i, uint32_t bits) {
    if (bits == 0) return;
    const int b = i & 1;
    stage_states<T, D>(kbase + (size_t)i * 32 * a.k_stride, a.k_stride, bits, lds + b * TILE, wave,
                       lane, kswz);
    stage_states<T, D>(vbase + (size_t)i * 32 * a.v_stride, a.v_stride, bits, lds + (2 + b) * TILE,
                       wave, lane, vswz);
  };
  Seen<kMask> seen;
  uint32_t bits = 0, next = 0;
  if (t_begin < t_end) {
    seen.request(a.mask, t.ka, t.Lk, 32 * t_begin, lane);
    next = seen.bits(t.Lk, 32 * t_begin);
    issue(t_begin, next);
    seen.request(a.mask, t.ka, t.Lk, 32 * (t_begin + 1), lane);
  }

  // the row's operands, delta and -lse log2(e) (a row that saw no state: weights 0)
  CrossFrag<T> q[kCrossSteps<T, D>], dy[kCrossSteps<T, D>];
  load_row<T, D>(static_cast<const T*>(a.Q) + (size_t)qi * a.q_stride + (size_t)hq * D, h, q);
  load_row<T, D>(static_cast<const T*>(a.dY) + (size_t)qi * a.dy_stride + (size_t)hq * D, h, dy);
  float delta = 0.f;
  {
    CrossFrag<T> y[kCrossSteps<T, D>];
    load_row<T, D>(static_cast<const T*>(a.Y) + at * D, h, y);
#pragma unroll
    for (int k = 0; k < kCrossSteps<T, D>; ++k) {
      if constexpr (kB) {
#pragma unroll
        for (int e = 0; e < 8; ++e) delta = fmaf((float)y[k][e], (float)dy[k][e], delta);
      } else {
        delta = fmaf(y[k], dy[k], delta);
      }
    }
    delta = add_xor<32>(delta);
  }
  const float lse = a.lse[at], off = lse == -INFINITY ? -INFINITY : -lse * kLog2e;
  if (has_row && h == 0 && split == 0) a.delta[at] = delta;

  f32x16 acc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) acc[i] = f32x16{};
  for (int i = t_begin; i < t_end; ++i) {
    const int b = i & 1;
    bits = next;
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();  // tile i has landed, tile i - 1 is read
    if (i + 1 < t_end) {
      next = seen.bits(t.Lk, 32 * (i + 1));
      issue(i + 1, next);
      seen.request(a.mask, t.ka, t.Lk, 32 * (i + 2), lane);
    }
    if (bits == 0 || !wave_has) continue;
    const unsigned char *kt = lds + b * TILE, *vt = lds + (2 + b) * TILE;
    f32x16 p = f32x16{}, g = f32x16{};
    row_product<T, D>(kt, lane, q, kswz, p);
    row_product<T, D>(vt, lane, dy, vswz, g);
#pragma unroll
    for (int r = 0; r < 16; ++r) p[r] = exp2_hw(fmaf(p[r], a.scale_log2, off)) * (g[r] - delta);
    if (bits != ~0u) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (!(bits >> (8 * (r / 4) + 4 * h + r % 4) & 1)) p[r] = 0.f;
    }
    column_product<T, D>(kt, lane, p, kswz, acc);
  }
  if (splits > 1) {
    if (has_row)
      store_lanes<D>(cross_part(a, tile, hkv, split, (size_t)kCrossTile * D), wave, lane, acc);
    return;
  }
  if (has_row) store_row<T, D>(static_cast<T*>(a.dQ) + at * D, h, a.scale, acc);
}

// ---- dK, dV: owns states ---------------------------------------------------------------

template <typename T, int D, bool kMask>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(Elem<T>::kBf16 && D == 64 ? 2 : 1)))
void cross_dkv_kernel(CrossArgs a) {
  constexpr int DT = D / 32, ESZ = sizeof(T), U = D * ESZ / 16, TILE = 32 * D * ESZ;
  constexpr int RPC = 64 / U, CPW = 32 / RPC / kCrossWaves;
  constexpr bool kB = Elem<T>::kBf16;
  __shared__ __attribute__((aligned(16))) unsigned char lds[4 * TILE];  // Q0 Q1 dY0 dY1
  __shared__ __attribute__((aligned(16))) float s_row[2][2][32];  // -lse log2(e), delta
  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int h = lane / 32, c = lane % 32;
  const int hkv = blockIdx.x % a.Hkv, tile = blockIdx.x / a.Hkv;
  CrossTile t;
  if (!find_cross_tile<true>(a, tile, lane, t)) return;
  const int rows = t.Lq * a.G;
  const int n_tiles = (rows + 31) / 32, splits = splits_of<kLeastTiles>(a, n_tiles);
  const int split = blockIdx.y;
  if (split >= splits) return;
  const int t_begin = (int)((long long)n_tiles * split / splits);
  const int t_end = (int)((long long)n_tiles * (split + 1) / splits);

  const int key0 = t.lt * kCrossTile + 32 * wave, key = key0 + c;
  const bool has_key = key < t.Lk, wave_has = key0 < t.Lk;
  const int at_key = t.ka + min(key, t.Lk - 1);
  const bool seen = has_key && (!kMask || a.mask[at_key] != 0);
  // a state that takes no part may hold anything: it is taken as 0
  CrossFrag<T> k[kCrossSteps<T, D>], v[kCrossSteps<T, D>];
  load_row<T, D>(static_cast<const T*>(a.K) + (size_t)at_key * a.k_stride + (size_t)hkv * D, h, k);
  load_row<T, D>(static_cast<const T*>(a.V) + (size_t)at_key * a.v_stride + (size_t)hkv * D, h, v);
  if (kMask && !seen) {
#pragma unroll
    for (int i = 0; i < kCrossSteps<T, D>; ++i) k[i] = CrossFrag<T>{}, v[i] = CrossFrag<T>{};
  }

  const T* qbase = static_cast<const T*>(a.Q) + (size_t)t.qa * a.q_stride + (size_t)hkv * a.G * D;
  const T* ybase = static_cast<const T*>(a.dY) + (size_t)t.qa * a.dy_stride + (size_t)hkv * a.G * D;
  auto swz = [](int r) { return both_swizzle<U, kB>(r); };
  float row_value = 0.f;  // threads 0..31: -lse log2(e), 32..63: delta of a tile's rows
  auto issue = [&](int i) {
    const int b = i & 1;
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
          rq, (__attribute__((address_space(3))) void*)(lds + b * TILE + 1024 * j), 16,
          (uint32_t)dq * (uint32_t)(a.q_stride * ESZ) + in, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          ry, (__attribute__((address_space(3))) void*)(lds + (2 + b) * TILE + 1024 * j), 16,
          (uint32_t)dq * (uint32_t)(a.dy_stride * ESZ) + in, 0, 0, 0);
    }
    if (tid < 64) {
      const int x = head0 + min(c, last), dq = quotient(x, a.g_reciprocal);
      const size_t at = (size_t)(t.qa + q0 + dq) * a.Hq + hkv * a.G + (x - dq * a.G);
      const float e = tid < 32 ? a.lse[at] : a.delta[at];
      // rows past the last one, and rows that saw no state: weights 0
      row_value = tid >= 32 ? e : c > last || e == -INFINITY ? -INFINITY : -e * kLog2e;
    }
  };

  f32x16 dk[DT], dv[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) dk[i] = f32x16{}, dv[i] = f32x16{};
  if (t_begin < t_end) issue(t_begin);
  for (int i = t_begin; i < t_end; ++i) {
    const int b = i & 1;
    if (tid < 64) s_row[b][tid / 32][tid % 32] = row_value;
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();  // tile i has landed, tile i - 1 is read
    if (i + 1 < t_end) issue(i + 1);
    if (!wave_has) continue;
    const unsigned char *qt = lds + b * TILE, *yt = lds + (2 + b) * TILE;
    f32x16 p = f32x16{}, g = f32x16{};
    row_product<T, D>(qt, lane, k, swz, p);
    row_product<T, D>(yt, lane, v, swz, g);
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
  }
  if (splits > 1) {
    float* part = cross_part(a, tile, hkv, split, 2 * (size_t)kCrossTile * D);
    if (has_key) {
      store_lanes<D>(part, wave, lane, dk);
      store_lanes<D>(part + kCrossTile * D, wave, lane, dv);
    }
    return;
  }
  if (!has_key) return;
  const size_t at = ((size_t)at_key * a.Hkv + hkv) * D;
  store_row<T, D>(static_cast<T*>(a.dK) + at, h, a.scale, dk);
  store_row<T, D>(static_cast<T*>(a.dV) + at, h, 1.f, dv);
}

// Joins the parts of a tile's rows (dQ) or states (dK, dV): one piece of 4 columns per
// thread, the parts in their order.
template <typename T, int D, bool kStates>
__global__ __launch_bounds__(256) void cross_sum_kernel(CrossArgs a) {
  const int hkv = blockIdx.x % a.Hkv, tile = blockIdx.x / a.Hkv;
  CrossTile t;
  if (!find_cross_tile<kStates>(a, tile, threadIdx.x % kWave, t)) return;
  const int rows = t.Lq * a.G;
  const int n = splits_of<kLeastTiles>(a, ((kStates ? rows : t.Lk) + 31) / 32);
  if (n == 1) return;
  const int piece = blockIdx.y * 256 + threadIdx.x, q = piece / kWave % (D / 8);
  const int r = 32 * (piece / kWave / (D / 8)) + piece % 32;
  const int d0 = 8 * q + 4 * (piece % kWave / 32);
  const int row = t.lt * kCrossTile + r;
  if (row >= (kStates ? t.Lk : rows)) return;
  constexpr size_t kOne = (size_t)kCrossTile * D, kAll = kStates ? 2 * kOne : kOne;
  const float* part = cross_part(a, tile, hkv, 0, kAll) + 4 * piece;
  f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f}, y = x;
#pragma unroll 8
  for (int i = 0; i < n; ++i) {
    x += *reinterpret_cast<const f32x4*>(part + i * kAll);
    if (kStates) y += *reinterpret_cast<const f32x4*>(part + i * kAll + kOne);
  }
  auto store = [&](void* out, size_t at, const f32x4& v) {
    T* o = static_cast<T*>(out) + at * D + d0;
    if constexpr (Elem<T>::kBf16)
      *reinterpret_cast<bf16x4*>(o) = bf16x4{(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
    else
      *reinterpret_cast<f32x4*>(o) = v;
  };
  if (kStates) {
    const size_t at = (size_t)(t.ka + row) * a.Hkv + hkv;
    store(a.dK, at, a.scale * x);
    store(a.dV, at, y);
  } else {
    store(a.dQ, (size_t)(t.qa + row / a.G) * a.Hq + hkv * a.G + row % a.G, a.scale * x);
  }
}

long long tiles_of(long long rows, int S) { return rows / kCrossTile + S; }

// Workgroups that share a tile's work: as many as fill the device, mean lengths
// standing for all. own: rows (or states) per source that a kernel owns, others:
// those it runs over.
int splits_for(long long own, long long others, int S, int Hkv) {
  const long long tiles = (std::max(1LL, own / S) + kCrossTile - 1) / kCrossTile * S * Hkv;
  const long long most = std::max(1LL, others / S / (32 * kLeastTiles));
  return (int)std::min({std::max(1LL, 512 / tiles), most, 64LL});
}

struct Plan {
  long long row_tiles, state_tiles;
  int row_splits, state_splits;
  size_t delta, parts;  // floats
};
Plan plan_of(int S, int Tq, int Tk, int Hq, int Hkv, int d) {
  const long long rows = (long long)Tq * (Hq / Hkv);
  Plan p;
  p.row_tiles = tiles_of(rows, S), p.state_tiles = tiles_of(Tk, S);
  p.row_splits = splits_for(rows, Tk, S, Hkv), p.state_splits = splits_for(Tk, rows, S, Hkv);
  p.delta = ((size_t)Tq * Hq + 3) / 4 * 4;
  // the two kernels' parts lie at the same place: dQ is joined before dK and dV start
  const size_t one = (size_t)kCrossTile * d * Hkv;
  const size_t a = p.row_splits > 1 ? p.row_tiles * p.row_splits * one : 0;
  const size_t b = p.state_splits > 1 ? p.state_tiles * p.state_splits * 2 * one : 0;
  p.parts = std::max(a, b);
  return p;
}

}  // namespace

size_t cross_attention_bwd_workspace(int S, int Tq, int Tk, int Hq, int Hkv, int d) {
  const Plan p = plan_of(S, Tq, Tk, Hq, Hkv, d);
  return (p.delta + p.parts) * sizeof(float);
}

template <typename T, int D>
hipError_t launch_cross_attention_bwd(int S, int Tq, int Tk, int Hq, int Hkv, float scale,
                                      const void* Q, int64_t q_stride, const void* K,
                                      int64_t k_stride, const void* V, int64_t v_stride,
                                      const int32_t* cu_q, const int32_t* cu_k,
                                      const uint8_t* mask, const void* Y, const float* lse,
                                      const void* dY, int64_t dy_stride, void* dQ, void* dK,
                                      void* dV, void* workspace, hipStream_t stream) {
  const Plan p = plan_of(S, Tq, Tk, Hq, Hkv, D);
  CrossArgs a{};
  a.Q = Q, a.K = K, a.V = V, a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride;
  a.cu_q = cu_q, a.cu_k = cu_k, a.mask = mask, a.Y = const_cast<void*>(Y);
  a.lse = const_cast<float*>(lse), a.dY = dY, a.dy_stride = dy_stride;
  a.dQ = dQ, a.dK = dK, a.dV = dV;
  a.S = S, a.Tq = Tq, a.Tk = Tk, a.Hq = Hq, a.Hkv = Hkv, a.G = Hq / Hkv;
  a.g_reciprocal = reciprocal_of(a.G);
  a.scale = scale, a.scale_log2 = scale * kLog2e;
  a.delta = static_cast<float*>(workspace), a.parts = a.delta + p.delta;
  hipError_t e = hipSuccess;
  if (Tq > 0) {
    a.tiles = (int)p.row_tiles, a.splits = p.row_splits;
    const dim3 grid((unsigned)(a.tiles * Hkv), (unsigned)a.splits);
    if (mask)
      hipLaunchKernelGGL((cross_dq_kernel<T, D, true>), grid, dim3(256), 0, stream, a);
    else
      hipLaunchKernelGGL((cross_dq_kernel<T, D, false>), grid, dim3(256), 0, stream, a);
    e = hipGetLastError();
    if (e == hipSuccess && a.splits > 1) {
      hipLaunchKernelGGL((cross_sum_kernel<T, D, false>),
                         dim3((unsigned)(a.tiles * Hkv), kCrossTile * D / 4 / 256), dim3(256), 0,
                         stream, a);
      e = hipGetLastError();
    }
  }
  if (e != hipSuccess || Tk == 0) return e;
  a.tiles = (int)p.state_tiles, a.splits = p.state_splits;
  const dim3 grid((unsigned)(a.tiles * Hkv), (unsigned)a.splits);
  if (mask)
    hipLaunchKernelGGL((cross_dkv_kernel<T, D, true>), grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((cross_dkv_kernel<T, D, false>), grid, dim3(256), 0, stream, a);
  e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  hipLaunchKernelGGL((cross_sum_kernel<T, D, true>),
                     dim3((unsigned)(a.tiles * Hkv), kCrossTile * D / 4 / 256), dim3(256), 0, stream,
                     a);
  return hipGetLastError();
}

#define AVQ_INSTANCE(T, D)                                                                        \
  template hipError_t launch_cross_attention_bwd<T, D>(                                           \
      int, int, int, int, int, float, const void*, int64_t, const void*, int64_t, const void*,    \
      int64_t, const int32_t*, const int32_t*, const uint8_t*, const void*, const float*,         \
      const void*, int64_t, void*, void*, void*, void*, hipStream_t);
AVQ_INSTANCE(bf16, 64)
AVQ_INSTANCE(bf16, 128)
AVQ_INSTANCE(float, 64)
AVQ_INSTANCE(float, 128)
#undef AVQ_INSTANCE

}  // namespace avq
