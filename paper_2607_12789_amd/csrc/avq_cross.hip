// Cross attention: packed queries over the packed states of their source (of
// another length), some of which a mask may hide.
//
//   S_ij = scale q_i . k_j,  Y_i = sum_j exp(S_ij - lse_i) v_j,
//   lse_i = ln sum_j exp(S_ij), over the states j of i's source that take part.
//
// One pass over the states with a running maximum and sum. A workgroup of four
// waves owns 128 rows of one key-value head, 32 per wave (avq_cross.hpp: a row is
// a query and a head of the group); the states stream through LDS in tiles of 32,
// double buffered, by direct global->LDS copies. Products are transposed, S^T = K
// Q^T with 32x32x16 bf16 (32x32x2 fp32) MFMA, so that a lane owns one row (with
// its partner lane l ^ 32) and 16 of 32 states, and the weights are the operand
// of Y^T = V^T P^T as they are; the values are read transposed from LDS.
//
// Single tokens: a tile has few rows, its states are shared out over several
// workgroups, and what bounds it is the states' bytes; a wave without rows only
// copies.
#include "avq_launch.hpp"

#include <algorithm>

#include "avq_cross.hpp"

namespace avq {

namespace {

template <typename T, int D>
constexpr int kPerCu = Elem<T>::kBf16 && D == 128 ? 3 : 2;  // waves per SIMD, at least

template <typename T, int D, bool kMask>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(kPerCu<T, D>)))
void cross_kernel(CrossArgs a) {
  constexpr int DT = D / 32, ESZ = sizeof(T), U = D * ESZ / 16, TILE = 32 * D * ESZ;
  constexpr bool kB = Elem<T>::kBf16;
  __shared__ __attribute__((aligned(16))) unsigned char lds[4 * TILE];  // K0 K1 V0 V1
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
  RowFrag<T> q[kRowSteps<T, D>];
  load_row<T, D>(static_cast<const T*>(a.Q) + (size_t)qi * a.q_stride + (size_t)hq * D, h, q);

  const T* kbase = static_cast<const T*>(a.K) + (size_t)t.ka * a.k_stride + (size_t)hkv * D;
  const T* vbase = static_cast<const T*>(a.V) + (size_t)t.ka * a.v_stride + (size_t)hkv * D;
  auto kswz = [](int r) { return key_swizzle<U>(r); };
  auto vswz = [](int r) { return value_swizzle<U, kB>(r); };
  auto issue = [&](int i, uint32_t bits) {
    if (bits == 0) return;
    const int b = i & 1;
    stage_states<T, D>(kbase + (size_t)i * 32 * a.k_stride, a.k_stride, bits, lds + b * TILE, wave,
                       lane, kswz);
    stage_states<T, D>(vbase + (size_t)i * 32 * a.v_stride, a.v_stride, bits, lds + (2 + b) * TILE,
                       wave, lane, vswz);
  };

  // m: the running max of s. The weights exp2((s - m) scale) are one fma with ms =
  // m scale and exp2; rows whose max is so large that the rounding of ms would
  // count subtract m first, and ms is 0.
  float m = kMaxFloor, ms = kMaxFloor, limit = kMaxFloor, l = 0.f;
  bool fused = true;
  f32x16 o[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) o[i] = f32x16{};

  // the bytes of the mask are asked for one tile ahead of the copies
  Seen<kMask> seen;
  uint32_t bits = 0, next = 0;
  if (t_begin < t_end) {
    seen.request(a.mask, t.ka, t.Lk, 32 * t_begin, lane);
    next = seen.bits(t.Lk, 32 * t_begin);
    issue(t_begin, next);
    seen.request(a.mask, t.ka, t.Lk, 32 * (t_begin + 1), lane);
  }
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
    f32x16 sc = f32x16{};
    row_product<T, D>(lds + b * TILE, lane, c, q, kswz, sc);
    if (bits != ~0u) {
      const uint32_t mine = place(bits >> (4 * h));
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (!(mine & 1u << (8 * (r / 4) + r % 4))) sc[r] = -INFINITY;
    }
    float mx = sc[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, sc[r]);
    if (__any(mx > limit)) {
      const float mn = fmaxf(m, max_xor<32>(mx)), mns = fmaxf(mn * a.scale_log2, kMaxFloor);
      const bool was = fused;
      fused = was && !__any(fabsf(mns) > kFused && mn > kMaxFloor);
      const float f = mn == kMaxFloor ? 1.f
                                      : exp2_hw(fused ? ms - mns
                                                : was ? fmaf(-mn, a.scale_log2, ms)
                                                      : (m - mn) * a.scale_log2);
      m = mn;
      ms = fused ? mns : 0.f;
      limit = fused ? mn + a.lazy : -INFINITY;
      if (!fused) {
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] -= m;
      }
      l *= f;
#pragma unroll
      for (int k = 0; k < DT; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[k][r] *= f;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      sc[r] = exp2_hw(fmaf(sc[r], a.scale_log2, -ms));
      l += sc[r];
    }
    // weights rounded to bf16 for the matrix product (by at most half a step, 2^-8),
    // their sum l of the unrounded ones
    column_product<T, D>(lds + (2 + b) * TILE, lane, sc, vswz, o);
  }

  l = add_xor<32>(l);
  if (!fused) ms = m * a.scale_log2;
  const size_t at = (size_t)qi * a.Hq + hq;
  const float inv = l > 0.f ? 1.f / l : 0.f;
  if (has_row && h == 0) {
    if (splits > 1) {
      const size_t rows_all = (size_t)a.Tq * a.Hq, part = split * rows_all + at;
      a.parts[a.splits * rows_all * D + part] = ms;
      a.parts[a.splits * rows_all * (D + 1) + part] = l;
    } else if (a.lse) {
      a.lse[at] = l > 0.f ? (ms + log2_hw(l)) * kLn2 : -INFINITY;
    }
  }
  if (splits > 1) {
    if (has_row)
      store_row<float, D>(a.parts + ((size_t)split * a.Tq * a.Hq + at) * D, h, 1.f, o);
  } else if (kB && rows - t.lt * kCrossTile > 32) {
    // whole rows: 4 sources of 4096 queries and 31 to 128 states, 12 heads, d = 64, 21.7
    // us by store_row, 18.6 so; of 1024 and 2048, 16 heads, d = 128, 113 and 109. For one
    // row the barrier is not worth it, nor in fp32 the registers.
    __syncthreads();  // the last tile is read
    if (!wave_has) return;
    const RowsOf row_of(a, t, row0);
    store_rows<T, D, T>(lds + wave * TILE, lane, inv, o, rows - row0,
                        [&](int r) { return static_cast<T*>(a.Y) + row_of(a, t, r) * D; });
  } else if (has_row) {
    store_row<T, D>(static_cast<T*>(a.Y) + at * D, h, inv, o);
  }
}

long long tiles_of(long long rows, int S) { return rows / kCrossTile + S; }

template <typename T>
CrossSplit split_for(int S, int Tq, int Tk, int Hq, int Hkv) {
  return cross_split((long long)Tq * (Hq / Hkv), Tk, S, Hkv, 768, sizeof(T) == 4);
}

}  // namespace

template <typename T, int D>
size_t cross_attention_workspace(int S, int Tq, int Tk, int Hq, int Hkv) {
  const int splits = split_for<T>(S, Tq, Tk, Hq, Hkv).splits;
  return splits == 1 ? 0 : ((size_t)Tq * Hq * splits * (D + 2) + 4) * sizeof(float);
}

template <typename T, int D>
hipError_t launch_cross_attention(int S, int Tq, int Tk, int Hq, int Hkv, float scale,
                                  const void* Q, int64_t q_stride, const void* K, int64_t k_stride,
                                  const void* V, int64_t v_stride, const int32_t* cu_q,
                                  const int32_t* cu_k, const uint8_t* mask, void* Y, float* lse,
                                  void* workspace, hipStream_t stream) {
  CrossArgs a{};
  a.Q = Q, a.K = K, a.V = V, a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride;
  a.cu_q = cu_q, a.cu_k = cu_k, a.mask = mask, a.Y = Y, a.lse = lse;
  a.S = S, a.Tq = Tq, a.Tk = Tk, a.Hq = Hq, a.Hkv = Hkv, a.G = Hq / Hkv;
  a.tiles = (int)tiles_of((long long)Tq * a.G, S);
  const CrossSplit split = split_for<T>(S, Tq, Tk, Hq, Hkv);
  a.per = split.per, a.splits = split.splits;
  a.g_reciprocal = reciprocal_of(a.G);
  a.scale = scale, a.scale_log2 = scale * kLog2e, a.lazy = kLazy / a.scale_log2;
  a.parts = static_cast<float*>(workspace);
  a.slots = cross_slots<T, D>(S, (long long)Tq * a.G, 768);
  a.steps = reinterpret_cast<int32_t*>(a.parts + (size_t)Tq * Hq * a.splits * (D + 2));
  const dim3 grid((unsigned)(a.tiles * Hkv), (unsigned)a.splits);
  if (mask)
    hipLaunchKernelGGL((cross_kernel<T, D, true>), grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((cross_kernel<T, D, false>), grid, dim3(256), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  return launch_cross_join<T, D, kJoinSoftmax>(a, stream);
}

#define AVQ_INSTANCE(T, D)                                                                        \
  template hipError_t launch_cross_attention<T, D>(                                               \
      int, int, int, int, int, float, const void*, int64_t, const void*, int64_t, const void*,    \
      int64_t, const int32_t*, const int32_t*, const uint8_t*, void*, float*, void*, hipStream_t);    \
  template size_t cross_attention_workspace<T, D>(int, int, int, int, int);
AVQ_INSTANCE(bf16, 64)
AVQ_INSTANCE(bf16, 128)
AVQ_INSTANCE(float, 64)
AVQ_INSTANCE(float, 128)
#undef AVQ_INSTANCE

}  // namespace avq
