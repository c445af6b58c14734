// Cross attention, forward and backward: the rows of a source, its tiles, and
// the states a mask leaves.
//
// Nothing orders a source's queries, so the heads that share a key-value head are
// rows beside one another: row r of (source, key-value head) is query r / G, head
// r % G of its group, and 128 rows at a time read each state once. A tile is 128
// rows (or, for the states' gradients, 128 states) of one source; lengths are
// known on the device only, so the grid has rows / 128 + S tiles per key-value
// head, at least as many as the sources need: tile first / 128 + s + i is the
// i-th of source s, and those that belong to none exit.
#pragma once

#include "avq_cache.hpp"
#include "avq_tiles.hpp"

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
  int tiles, splits;  // per key-value head; workgroups that share a tile's work
  float scale, scale_log2;
  float lazy;  // kLazy / scale_log2
  float* parts;
};

constexpr int kCrossTile = 128;  // rows or states of a workgroup
constexpr int kCrossWaves = 4;

struct CrossTile {
  int s, lt;           // source, tile of its rows (or states)
  int qa, ka, Lq, Lk;  // its queries and states
};

// Tile of the source's rows (kStates: of its states), false if there is none.
template <bool kStates>
__device__ __forceinline__ bool find_cross_tile(const CrossArgs& a, int tile, int lane,
                                                CrossTile& t) {
  const int per = kStates ? 1 : a.G, T = kStates ? a.Tk : a.Tq;
  const int32_t* cu = kStates ? a.cu_k : a.cu_q;
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
  return t.lt >= 0 && (long long)t.lt * kCrossTile < n;
}

// Workgroups of a tile that have work: each as many of the n steps as the others,
// but kLeast at least. The same on the joining side.
template <int kLeast>
__device__ __forceinline__ int splits_of(const CrossArgs& a, int n) {
  return max(1, min(a.splits, n / kLeast));
}

// A part of rows: numerators [128][D], then maxima and sums [128]. The numerators
// lie as the lanes hold them, so that every store and load of a wave covers 1 KB:
// piece q = 4 i + j of wave w, [w][q][64 lanes][4], are the columns
// 32 i + 8 j + 4 (lane / 32) + 0 .. 3 of row 32 w + lane % 32.
__host__ __device__ constexpr size_t cross_part_floats(int D) {
  return (size_t)kCrossTile * (D + 2);
}
// Place of (tile, head)'s first part.
__device__ __forceinline__ float* cross_part(const CrossArgs& a, int tile, int head, int split,
                                             size_t floats) {
  return a.parts + (((size_t)tile * a.Hkv + head) * a.splits + split) * floats;
}

template <int D>
__device__ __forceinline__ void store_lanes(float* part, int wave, int lane,
                                            const f32x16 (&o)[D / 32]) {
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      *reinterpret_cast<f32x4*>(part + ((wave * (D / 8) + 4 * i + r / 4) * kWave + lane) * 4) =
          f32x4{o[i][r], o[i][r + 1], o[i][r + 2], o[i][r + 3]};
}

// The lane's columns of one row, times f: 32 i + 2 r + 4 h + 0 .. 3.
template <typename T, int D>
__device__ __forceinline__ void store_row(T* y, int h, float f, const f32x16 (&o)[D / 32]) {
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const int d0 = 32 * i + 2 * r + 4 * h;
      if constexpr (Elem<T>::kBf16)
        *reinterpret_cast<bf16x4*>(y + d0) = bf16x4{(bf16)(o[i][r] * f), (bf16)(o[i][r + 1] * f),
                                                    (bf16)(o[i][r + 2] * f),
                                                    (bf16)(o[i][r + 3] * f)};
      else
        *reinterpret_cast<f32x4*>(y + d0) =
            f32x4{o[i][r] * f, o[i][r + 1] * f, o[i][r + 2] * f, o[i][r + 3] * f};
    }
}

// One row as the operand of a 32x32 product whose contraction runs over d: bf16
// step k columns 16 k + 8 h + 0 .. 7; fp32 step 4 i + e column 8 i + 4 h + e.
template <typename T>
using CrossFrag = typename std::conditional<Elem<T>::kBf16, bf16x8, float>::type;
template <typename T, int D>
constexpr int kCrossSteps = Elem<T>::kBf16 ? D / 16 : D / 2;

template <typename T, int D>
__device__ __forceinline__ void load_row(const T* p, int h,
                                         CrossFrag<T> (&x)[kCrossSteps<T, D>]) {
#pragma unroll
  for (int k = 0; k < kCrossSteps<T, D>; ++k) {
    if constexpr (Elem<T>::kBf16) {
      x[k] = *reinterpret_cast<const bf16x8*>(p + 16 * k + 8 * h);
    } else if (k % 4 == 0) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(p + 2 * k + 4 * h);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[k + e] = v[e];
    }
  }
}

// acc[row][lane's column] += sum_d tile[row][d] x[d]: 32 staged rows, read row by
// row (lane c the row c), against the lanes' own ones.
template <typename T, int D, typename Swizzle>
__device__ __forceinline__ void row_product(const unsigned char* tile, int lane,
                                            const CrossFrag<T> (&x)[kCrossSteps<T, D>],
                                            Swizzle swizzle, f32x16& acc) {
  const int h = lane / 32, r = lane % 32;
  const unsigned char* rowp = tile + r * (D * (int)sizeof(T));
#pragma unroll
  for (int k = 0; k < D * (int)sizeof(T) / 32; ++k) {
    const unsigned char* p = rowp + 16 * ((2 * k + h) ^ swizzle(r));
    if constexpr (Elem<T>::kBf16) {
      acc = mfma32(*reinterpret_cast<const bf16x8*>(p), x[k], acc);
    } else {
      const f32x4 v = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc = mfma32(v[e], x[4 * k + e], acc);
    }
  }
}

// acc[i][column of 32 i ..][lane's column] += sum_row tile[row][column] w[row]: 32
// staged rows read transposed, the weights as the row product left them (row
// 8 (r / 4) + 4 h + r % 4 in register r). bf16: the matrix product takes them
// rounded to bf16.
template <typename T, int D, typename Swizzle>
__device__ __forceinline__ void column_product(const unsigned char* tile, int lane, const f32x16& w,
                                               Swizzle swizzle, f32x16 (&acc)[D / 32]) {
  const int h = lane / 32, c = lane % 32;
  constexpr int kRow = D * (int)sizeof(T);
  if constexpr (Elem<T>::kBf16) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {  // 16 rows: 4 h + 0..3 and 8 + 4 h + 0..3 per lane
      bf16x8 p;
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = (bf16)w[8 * k + e];
      const int row = 16 * k + 4 * h + lane % 16 / 4;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        const int unit = 4 * i + lane / 16 % 2 * 2 + lane % 4 / 2;
        bf16x8 v;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int r = row + 8 * e;
          const bf16x4 part = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
              (__attribute__((address_space(3))) bf16x4*)(tile + r * kRow +
                                                          16 * (unit ^ swizzle(r)) + 8 * (lane % 2)));
#pragma unroll
          for (int j = 0; j < 4; ++j) v[4 * e + j] = part[j];
        }
        acc[i] = mfma32(v, p, acc[i]);
      }
    }
  } else {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = 8 * (r / 4) + 4 * h + r % 4;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        const float v = *reinterpret_cast<const float*>(
            tile + row * kRow + 16 * ((8 * i + c / 4) ^ swizzle(row)) + 4 * (c % 4));
        acc[i] = mfma32(v, w[r], acc[i]);
      }
    }
  }
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

}  // namespace avq
