// The paged key-value cache: page layout, place of a position, and the 4-bit
// format (shared by the append, gather and attention kernels).
//
// A page holds page_size consecutive positions of one sequence for every
// key-value head; (page, head) is one block of E bytes of the pool
// [n_pages][Hkv][E]. Keys lie row by row, values in octets of 8 positions
// ([d][8], as in the packed aggregates): 8 positions of one column are then
// one lane's operand of the value product.
//   native  K [ps][d], V [ps/8][d][8] in the element type
//   fp4     K codes [ps][d/2], V codes [ps/8][d/2][8], K scales [ps][d/32],
//           V scales [ps/8][d/32][8] (bytes)
// 4-bit values are e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) times
// a power of two shared by 32 consecutive dimensions of one position, stored
// as its biased exponent; a code byte holds dimensions 2i (low four bits) and
// 2i + 1. A value byte is therefore one position's: with its own scale it is
// decoded by one conversion, and a single position is appended without
// touching a neighbour's bits.
#pragma once

#include "avq_common.hpp"

namespace avq {

struct PageLayout {
  uint32_t v, ks, vs;  // byte offsets of V, of the K scales and of the V scales
  uint32_t bytes;      // E
};

__host__ __device__ inline PageLayout page_layout(bool fp4, int esz, int ps, int d) {
  PageLayout L;
  const uint32_t body = fp4 ? (uint32_t)ps * d / 2 : (uint32_t)ps * d * esz;
  const uint32_t scales = fp4 ? (uint32_t)ps * d / 32 : 0u;
  L.v = body;
  L.ks = 2 * body;
  L.vs = 2 * body + scales;
  L.bytes = 2 * body + 2 * scales;
  return L;
}

// Where the cached positions lie. ps_log2: log2 of the page size.
struct CacheArgs {
  unsigned char* pool;
  const int32_t* table;  // [S][max_pages]
  int n_pages, max_pages, ps_log2, Hkv;
};

// The block of (page, head) that holds position pos of sequence s, or null:
// past the table's end, or an entry outside [0, n_pages).
__device__ __forceinline__ unsigned char* page_of(const CacheArgs& a, uint32_t page_bytes, int s,
                                                  int pos, int head) {
  const int i = pos >> a.ps_log2;
  if (pos < 0 || i >= a.max_pages) return nullptr;
  const int page = a.table[(size_t)s * a.max_pages + i];
  if ((unsigned)page >= (unsigned)a.n_pages) return nullptr;
  return a.pool + ((size_t)page * a.Hkv + head) * page_bytes;
}

// Biased exponent of a block's scale: the smallest 2^e with amax <= 6 2^e, so
// that no value saturates (with the exponent of amax alone, values in
// (6, 8) 2^e would lose up to a quarter). amax = m 2^x, 1 <= m < 2, needs
// e = x - 2, or x - 1 if m > 1.5. Kept in [1, 254]: normal powers of two.
__device__ __forceinline__ uint32_t fp4_scale(float amax) {
  const uint32_t b = __float_as_uint(amax);
  const int x = (int)(b >> 23) - 2 + ((b & 0x7fffffu) > 0x400000u ? 1 : 0);
  return (uint32_t)min(max(x, 1), 254);
}

// Number of octet slots for T packed tokens of S sequences: the new tokens of
// sequence s touch at most len / 8 + 2 octets of its positions, and slots
// cu[s] / 8 + 2 s .. are at least as many. No length is known on the host.
__host__ __device__ inline long long octet_slots(long long T, long long S) { return T / 8 + 2 * S; }

// The sequence that item i belongs to, where first(s) does not decrease:
// the largest s in [0, S) with first(s) <= i. All 64 lanes look at once, so
// one round of loads narrows the range 64 times.
template <typename F>
__device__ __forceinline__ int find_sequence(int S, long long i, int lane, F first) {
  int lo = 0, n = S;
  while (n > 1) {
    const int step = (n + kWave - 1) / kWave;
    const int at = lane * step;
    const bool in = at < n && (lane == 0 || first(lo + at) <= i);
    // the lanes that hold form a prefix (lane 0 always)
    const int cnt = __popcll(__ballot(in));
    lo += (cnt - 1) * step;
    n = min(step, n - (cnt - 1) * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Row range [a, b) of sequence s among T packed rows, kept inside [0, T)
// whatever cu holds.
__device__ __forceinline__ void packed_range(const int32_t* cu, int s, int T, int& a, int& b) {
  a = min(max(cu[s], 0), T);
  b = min(max(cu[s + 1], a), T);
}

}  // namespace avq
