// Cross attention, forward and backward: the rows of a source, its tiles, and
// the states a mask leaves.
//
// Nothing orders a source's queries, so the heads that share a key-value head are
// rows beside one another: row r of (source, key-value head) is query r / G, head
// r % G of its group, and 128 rows at a time read each state once. A tile is 128
// rows (or, for the states' gradients, 128 states) of one source; lengths are
// known on the device only, so the grid has rows / 128 + S tiles per key-value
// head, at least as many as the sources need, and workgroups that find none exit
// (many sources: tile first / 128 + s + i is the i-th of source s).
#pragma once

#include "avq_cache.hpp"
#include "avq_tiles.hpp"

#include <algorithm>

namespace avq {

struct CrossArgs {
  const void *Q, *K, *V;
  int64_t q_stride, k_stride, v_stride;  // elements between tokens
  const int32_t *cu_q, *cu_k;            // [S + 1]
  const uint8_t* mask;                   // [Tk], nullable
  void* Y;
  float* lse;      // nullable in the forward pass
  const void* dY;  // backward
  int64_t dy_stride;
  float* delta;    // [Tq][Hq]
  void *dQ, *dK, *dV;
  int S, Tq, Tk, Hq, Hkv, G;
  uint32_t g_reciprocal;
  int tiles;          // per key-value head, at most
  int per, splits;    // steps of 32 that a workgroup takes; workgroups of a tile, at most
  int slots;          // workgroups that run at once (0: steps are not chosen anew)
  int32_t* steps;     // steps that a workgroup takes, for the joining launch
  float scale, scale_log2;
  float lazy;  // kLazy / scale_log2
  float* parts;
};

constexpr int kCrossTile = 128;  // rows or states of a workgroup
constexpr int kCrossWaves = 4;

// Workgroups that share a tile's n steps, each about per of them. The same on the
// joining side.
__device__ __forceinline__ int splits_of(const CrossArgs& a, int per, int n) {
  return max(1, min(a.splits, (n + per - 1) / per));
}

// Time of `total` workgroups of `per` steps each, in steps: bf16, whose waves fill one
// another's latencies, in rounds of those that run at once; fp32, whose products add up,
// by the most on one CU, and one alone takes an eighth longer. Start and end of a workgroup
// cost about two steps.
__host__ __device__ inline float cross_cost(int slots, float total, float per) {
  return slots > 256 ? ceilf(total / slots) * (per + 2.f)
                     : per * fmaxf(1.12f, ceilf(total / 256.f)) + 2.f * ceilf(total / 256.f);
}

// Steps that a workgroup takes: the 64 lanes try a.per and the numbers behind it on the
// sources' lengths (lane s: workgroups of one part, steps). 2 to 16 sources: us, forward
// and backward, by the mean length and so: 5 of up to 517 queries and 1025 states, fp32, d =
// 64, 32.9 + 94.2 and 30.6 + 80.7; 8 of up to 1500 and 3000, 12 heads, d = 64, a quarter
// hidden, 92.1 + 187.7 and 81.2 + 193.9; 2 of 2048 and 1024, 16/4 heads, d = 64, 57.6 + 109.3
// and 44.3 + 110.2. fp32 at d = 128 lost by it (5 of up to 1500 and 3000, 6 heads, 82.7 +
// 563 and 90.1 + 583), as do few rows (8 of 5 and 784, 11.5 and 14.0).
// Backward in bf16, by the mean length and so: 3 sources of up to 1500 and 3000, 16/4 heads,
// d = 128, 251 and 212; 16 of up to 600 and 900, 8/2 heads, d = 128, 120 and 106; 4 of 4096
// and 31 to 128, 12 heads, d = 64, 59.6 and 58.2. Sources of one length are as they were or
// lose up to 2% (4 of 256 and 2048, 16/4 heads, d = 64, 86.0 and 87.4); most lost 8 of up to
// 1500 and 3000, 12 heads, d = 64, of other lengths than above: 155 and 170, all of it in dQ.
__device__ __forceinline__ int steps_of(const CrossArgs& a, int lane, int tiles, int n) {
  const int per = a.per + lane;
  const float inv = 1.f / per;
  float total = 0.f;
  for (int s = 0; s < a.S; ++s) {
    const float parts = floorf(((float)__builtin_amdgcn_readlane(n, s) + per - 0.5f) * inv);
    total += (float)__builtin_amdgcn_readlane(tiles, s) * fmaxf(1.f, fminf(parts, (float)a.splits));
  }
  const float cost = cross_cost(a.slots, total, per);
  float least = cost;
#pragma unroll
  for (int k = 1; k < kWave; k *= 2) least = fminf(least, __shfl_xor(least, k, kWave));
  return a.per + (int)__builtin_ctzll(__ballot(cost == least));
}

struct CrossTile {
  int s, lt, hkv;      // source, tile of its rows (or states), key-value head
  int qa, ka, Lq, Lk;  // its queries and states
  int split, splits;   // which of the workgroups that share its steps
};

// The tile of this workgroup's rows (kStates: states), false if it has none.
//
// Up to 64 sources, one per lane: tiles, heads and splits in one line, so that the
// workgroups without work come last. Among the others they leave some CUs with three
// workgroups and others with one (1024 queries and states of 8 heads, d = 64, fp32:
// forward 43.5 us so, 36.8 in one line, backward 110.7 and 99.2; 8 sources of 10 to 3000,
// fp32: 796 and 711; 4096 queries and states twice, bf16, loses 1%).
template <bool kStates>
__device__ __forceinline__ bool find_cross_tile(const CrossArgs& a, int lane, CrossTile& t) {
  if (a.S <= kWave) {
    int qa = 0, qb = 0, ka = 0, kb = 0;
    if (lane < a.S) {
      packed_range(a.cu_q, lane, a.Tq, qa, qb);
      packed_range(a.cu_k, lane, a.Tk, ka, kb);
    }
    const int rows = (qb - qa) * a.G, own = kStates ? kb - ka : rows, others = kStates ? rows : kb - ka;
    const int tiles = (own + kCrossTile - 1) / kCrossTile, steps = (others + 31) / 32;
    const int per = a.splits > 1 && a.slots > 0 ? steps_of(a, lane, tiles * a.Hkv, steps) : a.per;
    if (a.splits > 1 && blockIdx.x + blockIdx.y == 0 && threadIdx.x == 0) *a.steps = per;
    const int splits = splits_of(a, per, steps);
    // cu that decrease could ask for more than the grid has: no sum overflows
    const int n = min((long long)tiles * a.Hkv * splits, (long long)gridDim.x * gridDim.y);
    const int incl = wave_incl_scan(n), w = blockIdx.y * gridDim.x + blockIdx.x;
    if (w >= last_lane(incl)) return false;
    t.s = __popcll(__ballot(incl <= w));
    auto at = [&](int x) { return __builtin_amdgcn_readlane(x, t.s); };
    t.qa = at(qa), t.Lq = at(qb) - t.qa, t.ka = at(ka), t.Lk = at(kb) - t.ka, t.splits = at(splits);
    const int i = w - at(incl - n), j = i / a.Hkv;
    t.hkv = i - j * a.Hkv;
    t.split = j / at(tiles);
    t.lt = j - t.split * at(tiles);
    return true;
  }
  if (a.splits > 1 && blockIdx.x + blockIdx.y == 0 && threadIdx.x == 0) *a.steps = a.per;
  const int per = kStates ? 1 : a.G, T = kStates ? a.Tk : a.Tq;
  const int32_t* cu = kStates ? a.cu_k : a.cu_q;
  const int tile = blockIdx.x / a.Hkv;
  t.hkv = blockIdx.x - tile * a.Hkv;
  t.s = find_sequence(a.S, tile, lane, [&](int k) {
    return (long long)(min(max(cu[k], 0), T) * per / kCrossTile) + k;
  });
  int b;
  packed_range(a.cu_q, t.s, a.Tq, t.qa, b);
  t.Lq = b - t.qa;
  packed_range(a.cu_k, t.s, a.Tk, t.ka, b);
  t.Lk = b - t.ka;
  const int first = kStates ? t.ka : t.qa * a.G, n = kStates ? t.Lk : t.Lq * a.G;
  t.lt = tile - (first / kCrossTile + t.s);
  t.split = blockIdx.y;
  t.splits = splits_of(a, a.per, ((kStates ? t.Lq * a.G : t.Lk) + 31) / 32);
  return t.lt >= 0 && (long long)t.lt * kCrossTile < n && t.split < t.splits;
}

// How the work of a kernel's tiles is shared out. The host knows the sources' mean
// lengths only: with `own` rows (or states) and `others` it runs over per source, W
// workgroups take equal parts of the whole, but 2 to 8 steps at least. A source of
// four times the mean length is still divided like that, a longer one in as many
// parts. A tile has 64 parts at most, one for each lane of the joining wave: few tiles over
// very many states leave CUs without work (one query of 8 heads that share a key-value
// head, bf16, d = 128: 65536 states 30 us, 2^20 states 500, almost 5 times what their bytes
// take; of 16 heads, 4 key-value heads, 33 and 570).
struct CrossSplit {
  int per, splits;
};
inline CrossSplit cross_split(long long own, long long others, int S, int Hkv, int W, bool wide) {
  // parts of many rows cost as much as some more steps. Of few rows only one wave has
  // any, and a step of fp32 at d = 128 takes it 4 us (one query, 2000 states, 8 heads:
  // 24.1 us with 4 steps, 15.8 with 2; 4 queries of 8 sources of 1000, 2 key-value
  // heads, d = 64: 17.0 and 13.2), where one of bf16 is worth less than a part (8 sources
  // of 784, 12 heads, d = 64: 11.1 us with 4, 13.2 with 2).
  const int least = own / S > kCrossTile ? (wide ? 4 : 8) : wide && own / S <= 32 ? 2 : 4;
  const long long tiles = ((own + S - 1) / S + kCrossTile - 1) / kCrossTile * S * Hkv;
  // parts of few rows cost little: twice as many, shorter ones, which lengths of all
  // kinds leave less uneven
  if (own / S <= 32) W *= 2;
  if (tiles >= W || own == 0) return {least, 1};  // nothing to divide
  const long long mean = (others / S + 31) / 32, all = (others + 31) / 32;
  const long long per = std::max<long long>(least, (tiles * mean + W - 1) / W);
  const long long most = std::min((all + per - 1) / per, 4 * ((mean + per - 1) / per));
  return {(int)per, (int)std::max(1LL, std::min(most, 64LL))};
}

// CrossArgs::slots of a kernel that holds W workgroups at once (bf16). The steps of more
// than 16 sources are not chosen anew, which the forward call would pay for: us, forward and
// backward, so and chosen, of up to 500 and 1500, 4 heads, d = 64, bf16: 17 sources 27 + 74 and
// 29 + 68, 32 31 + 67 and 38 + 66, 64 51 + 99 and 71 + 100; fp32 of up to 400 and 900, 4/2
// heads: 17 47 + 145 and 47 + 129, 48 76 + 261 and 80 + 262. 8/2 heads, d = 128, bf16, would
// gain: 17 45 + 134 and 48 + 116, 32 79 + 203 and 72 + 189, 64 79 + 270 and 79 + 270.
template <typename T, int D>
int cross_slots(int S, long long own, int W) {
  if (S < 2 || S > 16 || own / S <= 32 || (!Elem<T>::kBf16 && D == 128)) return 0;
  return Elem<T>::kBf16 ? W : 256;
}

// Parts: rows [splits][rows][D], where row = query * Hq + head (states: state * Hkv +
// head); then, of the forward pass, maxima and sums [splits][rows] each; of dQ in bf16
// sum P k [splits][rows][D] and two sums of dS [splits][rows] each; of dK dV [splits][rows][D].
enum CrossJoin { kJoinSoftmax, kJoinQueries, kJoinStates };

// Joins the parts of one row, in their order: kWaves waves a row, whose lanes take 4
// columns of 256 / D parts each at a time.
template <typename T, int D, CrossJoin kWhat, int kWaves>
__global__ __launch_bounds__(256) void cross_join_kernel(CrossArgs a) {
  constexpr int TPP = D / 4, PG = kWaves * kWave / TPP, kRows = 4 / kWaves;
  constexpr bool kStates = kWhat == kJoinStates;
  constexpr bool kMend = kWhat == kJoinQueries && Elem<T>::kBf16;
  __shared__ __attribute__((aligned(16))) float s_acc[kWaves == 1 ? 1 : PG][D];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int heads = kStates ? a.Hkv : a.Hq, T_ = kStates ? a.Tk : a.Tq;
  const size_t rows = (size_t)T_ * heads;
  const size_t row = (size_t)blockIdx.x * kRows + (kWaves == 1 ? wave : 0);
  if (row >= rows) return;
  const int token = __builtin_amdgcn_readfirstlane((int)(row / heads));
  const int32_t* cu = kStates ? a.cu_k : a.cu_q;
  const int s = find_sequence(a.S, token, lane,
                              [&](int k) { return (long long)min(max(cu[k], 0), T_); });
  int qa, qb, ka, kb;
  packed_range(a.cu_q, s, a.Tq, qa, qb);
  packed_range(a.cu_k, s, a.Tk, ka, kb);
  if (token < (kStates ? ka : qa) || token >= (kStates ? kb : qb)) return;
  const int n = splits_of(a, *a.steps, (((kStates ? (qb - qa) * a.G : kb - ka)) + 31) / 32);
  if (n == 1) return;  // stored already
  const int pg = (wave % kWaves * kWave + lane) / TPP, d0 = lane % TPP * 4;
  const float* const ms = a.parts + (size_t)a.splits * rows * D;
  const float* const ls = ms + (size_t)a.splits * rows;
  float m = kMaxFloor, l = 0.f;
  if (kWhat == kJoinSoftmax) {
    // lane i: the parts i (at most 64), all waves the same
    const float mine = lane < n ? ms[lane * rows + row] : kMaxFloor;
    const float sum = lane < n ? ls[lane * rows + row] : 0.f;
    m = mine;
#pragma unroll
    for (int k = 1; k < kWave; k *= 2) m = fmaxf(m, __shfl_xor(m, k, kWave));
    l = exp2_hw(mine - m) * sum;
#pragma unroll
    for (int k = 1; k < kWave; k *= 2) l += __shfl_xor(l, k, kWave);
  }
  float rest = 0.f, rounded = 0.f;
  if (kMend) {
    const float* const rests = a.parts + 2 * (size_t)a.splits * rows * D;
    rest = lane < n ? rests[lane * rows + row] : 0.f;
    rounded = lane < n ? rests[(a.splits + lane) * rows + row] : 0.f;
#pragma unroll
    for (int k = 1; k < kWave; k *= 2) {
      rest += __shfl_xor(rest, k, kWave);
      rounded += __shfl_xor(rounded, k, kWave);
    }
  }
  f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f}, y = x;
#pragma unroll 4
  for (int i = pg; i < n; i += PG) {
    const float* part = a.parts + ((size_t)i * rows + row) * D + d0;
    const f32x4 v = *reinterpret_cast<const f32x4*>(part);
    if (kWhat == kJoinSoftmax)
      x += exp2_hw(ms[i * rows + row] - m) * v;
    else
      x += v;
    if (kStates || kMend) y += *reinterpret_cast<const f32x4*>(part + (size_t)a.splits * rows * D);
  }
  // the groups of lanes, then the waves
  auto gather = [&](f32x4& v) {
#pragma unroll
    for (int k = TPP; k < kWave; k *= 2)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += __shfl_xor(v[e], k, kWave);
    if constexpr (kWaves > 1) {
      if (lane < TPP) *reinterpret_cast<f32x4*>(&s_acc[wave][d0]) = v;
      __syncthreads();
      v = *reinterpret_cast<const f32x4*>(&s_acc[0][d0]);
#pragma unroll
      for (int w = 1; w < kWaves; ++w) v += *reinterpret_cast<const f32x4*>(&s_acc[w][d0]);
      __syncthreads();
    }
  };
  gather(x);
  if (kStates || kMend) gather(y);
  if (wave % kWaves != 0 || lane >= TPP) return;
  auto store = [&](void* out, const f32x4& v) {
    T* o = static_cast<T*>(out) + row * D + d0;
    if constexpr (Elem<T>::kBf16)
      *reinterpret_cast<bf16x4*>(o) = bf16x4{(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
    else
      *reinterpret_cast<f32x4*>(o) = v;
  };
  if (kWhat == kJoinSoftmax) {
    store(a.Y, (l > 0.f ? 1.f / l : 0.f) * x);
    if (a.lse && lane == 0) a.lse[row] = l > 0.f ? (m + log2_hw(l)) * kLn2 : -INFINITY;
  } else if (kWhat == kJoinQueries) {
    store(a.dQ, a.scale * (kMend ? x - rounded * y : x));
    if (kMend && lane == 0 && wave % kWaves == 0) a.delta[row] += rest;
  } else {
    store(a.dK, a.scale * x);
    store(a.dV, y);
  }
}

template <typename T, int D, CrossJoin kWhat>
hipError_t launch_cross_join(const CrossArgs& a, hipStream_t stream) {
  const size_t rows = kWhat == kJoinStates ? (size_t)a.Tk * a.Hkv : (size_t)a.Tq * a.Hq;
  // four waves a row where there are many parts and few rows: many rows wait less for
  // their loads with one (7056 rows of up to 9 parts, fp32: the forward call 44.6 us with
  // four, 38.4 with one)
  if (a.splits > 8 && rows <= 2048)
    hipLaunchKernelGGL((cross_join_kernel<T, D, kWhat, 4>), dim3((unsigned)rows), dim3(256), 0,
                       stream, a);
  else
    hipLaunchKernelGGL((cross_join_kernel<T, D, kWhat, 1>), dim3((unsigned)((rows + 3) / 4)),
                       dim3(256), 0, stream, a);
  return hipGetLastError();
}

// Which of 32 states, from k0 on, take part: those before Lk that the mask does
// not hide. request() asks for the lane's byte, bits() gathers them.
template <bool kMask>
struct Seen {
  int byte = 1;
  __device__ __forceinline__ void request(const uint8_t* mask, int ka, int Lk, int k0, int lane) {
    if constexpr (kMask) {
      const int k = k0 + lane % 32;
      byte = k < Lk ? mask[ka + k] : 0;
    }
  }
  __device__ __forceinline__ uint32_t bits(int Lk, int k0) const {
    if constexpr (kMask) return (uint32_t)__ballot(byte != 0);
    const int n = Lk - k0;
    return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
  }
};

// Copies 32 states to LDS, the places of their units permuted. A state that takes
// no part may hold anything, and 0 times an infinity is not 0: the copies read the
// tile's first one that does in its place.
template <typename T, int D, typename Swizzle>
__device__ __forceinline__ void stage_states(const T* base, int64_t stride, uint32_t bits,
                                             unsigned char* lds, int wave, int lane,
                                             Swizzle swizzle) {
  constexpr int ESZ = sizeof(T), U = D * ESZ / 16, RPC = 64 / U, CPW = 32 / RPC / kCrossWaves;
  const __amdgpu_buffer_rsrc_t from = rsrc(base);
  const int first = __builtin_ctz(bits);
#pragma unroll
  for (int i = 0; i < CPW; ++i) {
    const int j = wave * CPW + i;
    const int r = RPC * j + lane / U, rr = bits >> r & 1 ? r : first;
    const uint32_t o =
        (uint32_t)rr * (uint32_t)(stride * ESZ) + 16u * ((lane % U) ^ swizzle(r));
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        from, (__attribute__((address_space(3))) void*)(lds + 1024 * j), 16, o, 0, 0, 0);
  }
}

// Stores a wave's first n rows, times f (of the lane's row), to at(r): handed over in
// LDS (32 D sizeof(T) bytes of the wave's own), so that an instruction writes whole rows,
// or halves, instead of 16 bytes of each of 32.
template <typename T, int D, typename Out, typename At>
__device__ __forceinline__ void store_rows(unsigned char* lds, int lane, float f,
                                           const f32x16 (&o)[D / 32], int n, At at) {
  constexpr int P = sizeof(Out) / sizeof(T), C = D / P;  // passes, columns of each
  constexpr int U = C * (int)sizeof(Out) / 16, RPI = kWave / U;
  const int h = lane / 32, c = lane % 32;
#pragma unroll
  for (int p = 0; p < P; ++p) {
#pragma unroll
    for (int i = 0; i < C / 32; ++i)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const f32x16& x = o[p * (C / 32) + i];
        const int d0 = 32 * i + 2 * r;  // + 4 h
        if constexpr (sizeof(Out) == 2)
          *reinterpret_cast<bf16x4*>(lds + c * 16 * U + 16 * ((d0 / 8) ^ (c % U)) + 8 * h) =
              bf16x4{(bf16)(x[r] * f), (bf16)(x[r + 1] * f), (bf16)(x[r + 2] * f),
                     (bf16)(x[r + 3] * f)};
        else
          *reinterpret_cast<f32x4*>(lds + c * 16 * U + 16 * ((d0 / 4 + h) ^ (c % U))) =
              f32x4{x[r] * f, x[r + 1] * f, x[r + 2] * f, x[r + 3] * f};
      }
    __builtin_amdgcn_wave_barrier();  // only this wave reads them: its LDS accesses stay in order
#pragma unroll
    for (int k = 0; k < 32 / RPI; ++k) {
      const int r = RPI * k + lane / U, u = lane % U;
      if (r < n)
        *reinterpret_cast<f32x4*>(reinterpret_cast<unsigned char*>(at(r) + p * C) + 16 * u) =
            *reinterpret_cast<const f32x4*>(lds + r * 16 * U + 16 * (u ^ (r % U)));
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Query and head of row r of a wave's 32, whose first is row0 of its source and
// key-value head.
struct RowsOf {
  int q0, head0;  // of row0
  __device__ __forceinline__ RowsOf(const CrossArgs& a, const CrossTile& t, int row0)
      : q0(t.qa + row0 / a.G), head0(row0 % a.G) {}
  __device__ __forceinline__ size_t operator()(const CrossArgs& a, const CrossTile& t, int r) const {
    const int x = head0 + r, dq = quotient(x, a.g_reciprocal);
    return (size_t)(q0 + dq) * a.Hq + t.hkv * a.G + (x - dq * a.G);
  }
};

}  // namespace avq
