// Tiles of 32 rows and 32 keys shared by the exact attentions: MFMA wrappers
// with their lane layouts, places of a staged row's units in LDS, constants of
// the running softmax.
#pragma once

#include "avq_common.hpp"

#include <type_traits>

namespace avq {

constexpr float kLazy = 8.f;         // log2 units the running max may lag behind
constexpr float kMaxFloor = -3e38f;  // finite start of the running max
constexpr float kFused = 0x1p24f;    // largest |max scale| at which s scale - max scale is one fma
constexpr float kLn2 = 0.6931471805599453f;

typedef float f32x16 __attribute__((ext_vector_type(16)));

// v_mfma_f32_32x32x16_bf16: lane l, h = l / 32, c = l % 32; A[c][8h .. 8h+7],
// B[8h .. 8h+7][c], D[8 (r/4) + 4 h + r % 4][c], r = 0..15.
// v_mfma_f32_32x32x2_f32: A[c][h], B[h][c], D as above.
__device__ __forceinline__ f32x16 mfma32(const bf16x8& a, const bf16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma32(float a, float b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}

// Positions of the 16-byte units of a staged row. Keys: 32 rows read one unit
// each, so consecutive rows permute their units. Values: 32 lanes of the
// transpose read take 64 bytes (four units) of 4 consecutive keys, 256 bytes
// and one pass over the 64 banks if these lie in different quarters: of 256
// bytes, one row at d = 128 (permuting pairs of units instead leaves two keys
// in one quarter: a third of the LDS cycles were conflicts) and two at d = 64.
template <int U>
__device__ __forceinline__ int key_swizzle(int r) {
  return U >= 16 ? r & 15 : (r >> 1) & 7;
}
template <int U, bool kB>
__device__ __forceinline__ int value_swizzle(int r) {
  if constexpr (!kB) return (r >> 2 & 1) << 3;
  return U >= 16 ? (r & 3) << 2 : (r & 3) << 1;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const void* p) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, 0x7fffffff, 0x00020000);
}

// Rows that are read both ways: one unit of 32 rows (16 consecutive rows take 16
// places), and transposed (bf16: 4 consecutive rows in different quarters of 256
// bytes; fp32: rows r and r + 4 in different halves).
template <int U, bool kB>
__device__ __forceinline__ int both_swizzle(int r) {
  if constexpr (!kB) return (r & 3) | (r >> 2 & 1) << 3 | (r >> 3 & 1) << 2;
  return U >= 16 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3);
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
using RowFrag = typename std::conditional<Elem<T>::kBf16, bf16x8, float>::type;
template <typename T, int D>
constexpr int kRowSteps = Elem<T>::kBf16 ? D / 16 : D / 2;

template <typename T, int D>
__device__ __forceinline__ void load_row(const T* p, int h,
                                         RowFrag<T> (&x)[kRowSteps<T, D>]) {
#pragma unroll
  for (int k = 0; k < kRowSteps<T, D>; ++k) {
    if constexpr (Elem<T>::kBf16) {
      x[k] = *reinterpret_cast<const bf16x8*>(p + 16 * k + 8 * h);
    } else if (k % 4 == 0) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(p + 2 * k + 4 * h);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[k + e] = v[e];
    }
  }
}

// A lane's place in a staged tile, computed where it is used: held over the loop, the
// places of all reads (8 to 32 of them) would take the registers of the products.
// Others follow from it by exchanging bits, as the swizzles are linear over them:
// swizzle(r ^ x) = swizzle(r) ^ swizzle(x).
__device__ __forceinline__ uint32_t place(uint32_t at) {
  asm volatile("" : "+v"(at));
  return at;
}

// acc[row][lane's column] += sum_d tile[row][d] x[d]: 32 staged rows, of which the
// lane reads row r, against the lanes' own ones.
template <typename T, int D, typename Swizzle>
__device__ __forceinline__ void row_product(const unsigned char* tile, int lane, uint32_t r,
                                            const RowFrag<T> (&x)[kRowSteps<T, D>],
                                            Swizzle swizzle, f32x16& acc) {
  constexpr uint32_t kRow = D * sizeof(T);
  const uint32_t h = lane / 32, at = place(r * kRow + 16 * (h ^ swizzle(r)));
#pragma unroll
  for (int k = 0; k < (int)kRow / 32; ++k) {
    const unsigned char* p = tile + (at ^ (32u * k));
    if constexpr (Elem<T>::kBf16) {
      acc = mfma32(*reinterpret_cast<const bf16x8*>(p), x[k], acc);
    } else {
      const f32x4 v = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc = mfma32(v[e], x[4 * k + e], acc);
    }
  }
}

// The weights of 32 rows as the row product left them (row 8 (r / 4) + 4 h + r % 4 in
// register r), as the operand of a product over the rows: bf16 rounded, 16 rows each.
template <typename T>
struct Weights {
  f32x16 w;
  __device__ __forceinline__ explicit Weights(const f32x16& x) : w(x) {}
};
template <>
struct Weights<bf16> {
  bf16x8 w[2];
  __device__ __forceinline__ explicit Weights(const f32x16& x) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) w[k][e] = (bf16)x[8 * k + e];
  }
  // x plus the sum of the rounded weights: two of them a step
  __device__ __forceinline__ float sum(float x) const {
    const bf16x2 one{(bf16)1.f, (bf16)1.f};
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int e = 0; e < 8; e += 2)
        x = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{w[k][e], w[k][e + 1]}, one, x, false);
    return x;
  }
};

// acc[n][i][column of 32 i ..][lane's column] += sum_row tile[row][column] w[n][row]:
// 32 staged rows read transposed, once for N sets of weights.
template <typename T, int D, int N, typename Swizzle>
__device__ __forceinline__ void column_products(const unsigned char* tile, int lane,
                                                const Weights<T> (&w)[N], Swizzle swizzle,
                                                f32x16 (&acc)[N][D / 32]) {
  constexpr uint32_t kRow = D * sizeof(T);
  const uint32_t h = lane / 32, c = lane % 32;
  if constexpr (Elem<T>::kBf16) {
    // 16 rows a step, 4 h + 0..3 and 8 + 4 h + 0..3 per lane; 32 bytes of 32 columns
    const uint32_t row = 4 * h + c % 16 / 4;
    const uint32_t at =
        place(row * kRow + 16 * ((c / 16 * 2 + c % 4 / 2) ^ swizzle(row)) + 8 * (c % 2));
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        bf16x8 v;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const bf16x4 part = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
              (__attribute__((address_space(3))) bf16x4*)(
                  tile + (at ^ (64u * i) ^ (16u * swizzle(8 * e))) + (16 * k + 8 * e) * kRow));
#pragma unroll
          for (int j = 0; j < 4; ++j) v[4 * e + j] = part[j];
        }
#pragma unroll
        for (int n = 0; n < N; ++n) acc[n][i] = mfma32(v, w[n].w[k], acc[n][i]);
      }
  } else {
    const uint32_t at = place(4 * h * kRow + 16 * (c / 4 ^ swizzle(4 * h)) + 4 * (c % 4));
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const uint32_t row = 8 * (r / 4) + r % 4;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        const float v = *reinterpret_cast<const float*>(
            tile + (at ^ (128u * i) ^ (16u * swizzle(row))) + row * kRow);
#pragma unroll
        for (int n = 0; n < N; ++n) acc[n][i] = mfma32(v, w[n].w[r], acc[n][i]);
      }
    }
  }
}
template <typename T, int D, typename Swizzle>
__device__ __forceinline__ void column_product(const unsigned char* tile, int lane, const f32x16& w,
                                               Swizzle swizzle, f32x16 (&acc)[D / 32]) {
  const Weights<T> one[1] = {Weights<T>(w)};
  column_products<T, D, 1>(tile, lane, one, swizzle,
                           reinterpret_cast<f32x16(&)[1][D / 32]>(acc));
}

// Index of row r of a tile of rows that are numbered row = query * G + head:
// the division of small numbers by G as one product (exact for x < 2^32 / G).
__host__ __device__ inline uint32_t reciprocal_of(int G) {
  return G == 1 ? 0u : (uint32_t)(0x100000000ull / (unsigned)G + 1);
}
__device__ __forceinline__ int quotient(int x, uint32_t reciprocal) {
  return reciprocal == 0u ? x : (int)__umulhi((unsigned)x, reciprocal);
}

}  // namespace avq
