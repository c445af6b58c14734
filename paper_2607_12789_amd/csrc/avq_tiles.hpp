// Tiles of 32 rows and 32 keys shared by the exact attentions: MFMA wrappers
// with their lane layouts, places of a staged row's units in LDS, constants of
// the running softmax.
#pragma once

#include "avq_common.hpp"

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

// Index of row r of a tile of rows that are numbered row = query * G + head:
// the division of small numbers by G as one product (exact for x < 2^32 / G).
__host__ __device__ inline uint32_t reciprocal_of(int G) {
  return G == 1 ? 0u : (uint32_t)(0x100000000ull / (unsigned)G + 1);
}
__device__ __forceinline__ int quotient(int x, uint32_t reciprocal) {
  return reciprocal == 0u ? x : (int)__umulhi((unsigned)x, reciprocal);
}

}  // namespace avq
