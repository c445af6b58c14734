// Exact attention of the newest tokens over the paged cache for groups of sequences
// that share their first positions: these are read once for the whole group.
//
// Positions below P_g (avq_cache_attention.hpp: shared_length) are taken through the
// pages of the group's first sequence, for the rows of all its sequences together:
// row r of (group, key-value head) is sequence r / (n_q G), token r / G % n_q, head
// r % G of the heads that share the key-value head. 128 rows at a time, 32 per wave,
// see each key once: keys and values go through LDS in tiles of 32 positions, double
// buffered (native: direct global->LDS copies, 4 bits: decoded once on the way), and
// products are transposed, S^T = K Q^T and Y^T = V^T P^T with 32x32x16 bf16 (32x32x2
// fp32) MFMA. The key rows are taken with bits 2 and 3 of their number exchanged: a
// lane then has the weights of whole octets, and its operand of the value product is
// an octet of one column, which lies together in the page.
//
// Behind P_g every sequence is attended to as in avq_cache_attention.hip. Both are
// one launch: its first workgroups take the shared positions, those of each tile of
// rows in as many runs of equal length as give every workgroup its share of the
// whole; the others take the sequences' own positions. All leave running maxima, sums
// and numerators, and a second launch joins them, row by row.
#include "avq_cache_attention.hpp"
#include "avq_launch.hpp"

#include <algorithm>

namespace avq {

namespace {

constexpr int kTile = 128;       // rows of a workgroup
constexpr int kLeastTiles = 4;   // tiles of 32 positions that a workgroup takes, at least
constexpr int kMaxSplits = 64;

struct PrefixArgs {
  CacheAttnArgs c;
  int shared_blocks;    // workgroups for the shared positions
  int splits;           // runs of one tile of rows, at most
  float lazy;           // kLazy / scale_log2
  float* shared_parts;  // numerators [splits][S n_q Hq][D], then maxima and sums
                        // [splits][S n_q Hq] each
  int32_t* per;         // tiles of 32 positions of a run, for the joining launch
};

struct Group {
  int first, rows, P;  // first sequence, rows per key-value head, shared positions
  __device__ __forceinline__ int row_tiles() const { return P > 0 ? (rows + kTile - 1) / kTile : 0; }
  __device__ __forceinline__ int tiles() const { return (P + 31) / 32; }
};
__device__ __forceinline__ Group group_of(const CacheAttnArgs& a, int g) {
  Group x;
  x.first = group_first(a, g);
  const int end = max(group_first(a, g + 1), x.first);
  x.rows = (end - x.first) * a.n_q * a.G;
  x.P = shared_length(a, g, x.first, end);
  return x;
}
// Runs of n tiles, the same on the joining side.
__device__ __forceinline__ int runs_of(int n, int per, int splits) {
  return max(1, min(splits, (n + per - 1) / per));
}
__device__ __forceinline__ float wave_sum(float x) {  // the same bits in every lane
#pragma unroll
  for (int k = 1; k < kWave; k *= 2) x += __shfl_xor(x, k, kWave);
  return x;
}

// Four values of a byte's word: the positions' bytes with their scales.
template <typename T>
__device__ __forceinline__ void decode4(uint32_t w, const float* f, T (*e)[2]) {
  if constexpr (Elem<T>::kBf16) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f[0], 0);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f[1], 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f[2], 2);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f[3], 3);
#pragma unroll
    for (int i = 0; i < 2; ++i) e[0][i] = a[i], e[1][i] = b[i], e[2][i] = c[i], e[3][i] = d[i];
  } else {
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, f[0], 0);
    const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, f[1], 1);
    const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, f[2], 2);
    const auto d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, f[3], 3);
#pragma unroll
    for (int i = 0; i < 2; ++i) e[0][i] = a[i], e[1][i] = b[i], e[2][i] = c[i], e[3][i] = d[i];
  }
}

// The operands of a tile's two products, as read from LDS: keys row by row (lane c the
// row r), values in octets, [octet][column][8]. bf16 reads all of them before the first
// product: one by one, each product would wait for its own read, and a workgroup of
// these is alone with its latencies (1 to 2 waves per SIMD).
template <typename T, int D>
struct Operands {
  static constexpr bool kB = Elem<T>::kBf16;
  bf16x8 k[kB ? D / 16 : 1], v[kB ? D / 16 : 1];

  __device__ __forceinline__ void read(const unsigned char* kt, const unsigned char* vt, int lane,
                                       uint32_t r) {
    if constexpr (kB) {
      const uint32_t h = lane / 32, c = lane % 32;
      const uint32_t at_k = place(r * (2 * D) + 16 * (h ^ key_swizzle<D / 8>(r)));
      const uint32_t at_v = place((h * D + c) * 16);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) k[i] = *reinterpret_cast<const bf16x8*>(kt + (at_k ^ (32u * i)));
#pragma unroll
      for (int i = 0; i < D / 16; ++i)  // octets h and 2 + h, D / 32 columns each
        v[i] = *reinterpret_cast<const bf16x8*>(vt + at_v +
                                                (2 * (i / (D / 32)) * D + 32 * (i % (D / 32))) * 16);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  __device__ __forceinline__ void logits(const unsigned char* kt, int lane, uint32_t r,
                                         const RowFrag<T> (&q)[kRowSteps<T, D>], f32x16& s) const {
    if constexpr (kB) {
#pragma unroll
      for (int i = 0; i < D / 16; ++i) s = mfma32(k[i], q[i], s);
    } else {
      row_product<T, D>(kt, lane, r, q, [](int x) { return key_swizzle<D * sizeof(T) / 16>(x); }, s);
    }
  }
  // o += V^T P^T: register 8 j + e of the weights is position e of octet 2 j + h. bf16:
  // the matrix product takes the weights rounded to bf16 (by at most half a step, 2^-8;
  // their sum is of the unrounded ones).
  __device__ __forceinline__ void values(const unsigned char* vt, int lane, const f32x16& w,
                                         f32x16 (&o)[D / 32]) const {
    const uint32_t h = lane / 32, c = lane % 32, at = place((h * D + c) * 8 * sizeof(T));
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if constexpr (kB) {
        bf16x8 p;
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = (bf16)w[8 * j + e];
#pragma unroll
        for (int i = 0; i < D / 32; ++i) o[i] = mfma32(v[j * (D / 32) + i], p, o[i]);
      } else {
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
          for (int e = 0; e < 8; e += 4) {
            const f32x4 x =
                *reinterpret_cast<const f32x4*>(vt + at + (2 * j * D + 32 * i) * 32 + 4 * e);
#pragma unroll
            for (int n = 0; n < 4; ++n) o[i] = mfma32(x[n], w[8 * j + e + n], o[i]);
          }
      }
    }
  }
};

// Buffers of staged tiles, as far ahead as the copies are issued: a tile of a workgroup
// alone on its CU takes less time than a copy needs to land. Three native buffers, two
// tiles ahead; two where a third would take the LDS of a second workgroup (fp32, d =
// 128). 4 bits wait in registers, two tiles ahead, and are decoded to two buffers.
// Each is an array of its own, and the loop unrolled over them: the compiler then
// knows that a step's reads do not touch what its copies write, and waits for none.
template <typename T, int D, bool FP4>
constexpr int kBuffers = !FP4 && 32 * D * sizeof(T) <= 8192 ? 3 : 2;
template <typename T, int D, bool FP4>
constexpr int kTilesAhead = FP4 || kBuffers<T, D, FP4> == 3 ? 2 : 1;
struct Buffers {
  unsigned char *k[3], *v[3];
};
// The same arrays as the exchange area of the other workgroups (one for each wave),
// the units of consecutive rows permuted.
template <int D>
struct SharedExchange {
  unsigned char* o[kWaves];
  __device__ __forceinline__ f32x4& unit(int wave, int row, int u) {
    unsigned char* p = wave == 0 ? o[0] : wave == 1 ? o[1] : wave == 2 ? o[2] : o[3];
    return reinterpret_cast<f32x4*>(p)[row * (D / 4) + (u ^ row % 16)];
  }
};

// Run `split` of `runs` of the shared positions of rows r0 .. r0 + 127 of a group
// and one key-value head.
template <typename T, int D, bool FP4>
__device__ __forceinline__ void shared_run(const PrefixArgs& p, const Group& t, int r0, int hkv,
                                           int split, int runs, const Buffers& lds) {
  constexpr bool kB = Elem<T>::kBf16;
  constexpr int ESZ = sizeof(T), U = D * ESZ / 16;
  constexpr int RPC = 64 / U, CPW = 8 / RPC, DT = D / 32;
  const CacheAttnArgs& a = p.c;
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int h = lane / 32, c = lane % 32;
  const int n_tiles = t.tiles();
  const int t_begin = (int)((long long)n_tiles * split / runs);
  const int t_end = (int)((long long)n_tiles * (split + 1) / runs);

  // ---- the lane's row -------------------------------------------------------------
  const int per = a.n_q * a.G;
  const int row0 = r0 + 32 * wave, row = row0 + c;
  const int at_row = min(row, t.rows - 1), s = t.first + at_row / per, len = length_of(a, s);
  const bool has_row = row < t.rows && len >= t.P, wave_has = row0 < t.rows;
  const int qi = at_row % per / a.G, hq = hkv * a.G + at_row % a.G;
  const int see = min(t.P, len - a.n_q + qi + 1);  // positions it sees
  RowFrag<T> q[kRowSteps<T, D>];
  load_row<T, D>(static_cast<const T*>(a.Q) + ((size_t)s * a.n_q + qi) * a.q_stride +
                     (size_t)hq * D,
                 h, q);

  // ---- pages, and tiles to LDS -------------------------------------------------------
  // A tile lies in one page, or (16 positions a page) in two; wave w copies its
  // positions 8 w .. 8 w + 7. Without a page the first one is read, which exists, and
  // the positions take no part.
  const PageLayout L = page_layout(FP4, ESZ, 1 << a.cache.ps_log2, D);
  const int ps_mask = (1 << a.cache.ps_log2) - 1;
  // read as constants (no kernel writes the table): scalar loads, which do not stand
  // behind the copies
  const auto pages = (const __attribute__((address_space(4))) int32_t*)(
      uintptr_t)(a.cache.table + (size_t)t.first * a.cache.max_pages);
  struct Pages {
    int id[2];
  };
  // asked for a tile before they are used, so nothing is decided on them here;
  // positions past the last one ask for its page
  auto lookup = [&](int i) {
    Pages r;
#pragma unroll
    for (int k = 0; k < 2; ++k) r.id[k] = pages[min(32 * i + 16 * k, t.P - 1) >> a.cache.ps_log2];
    return r;
  };
  auto exists = [&](int id) { return (unsigned)id < (unsigned)a.cache.n_pages; };
  auto bits_of = [&](int i, const Pages& g) {  // positions that can be read
    const int n = t.P - 32 * i;
    const uint32_t in = n >= 32 ? ~0u : (1u << n) - 1u;
    return in & ((exists(g.id[0]) ? 0xffffu : 0u) | (exists(g.id[1]) ? 0xffff0000u : 0u));
  };
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  struct Raw {  // 4 bits: a thread's share of a tile (d = 64: the first words)
    u32x2 k, v, vs;
    uint32_t ks;
  };
  auto block_of = [&](const Pages& g) {
    const int id = wave < 2 ? g.id[0] : g.id[1];
    return a.cache.pool + ((size_t)(exists(id) ? id : 0) * a.cache.Hkv + hkv) * L.bytes;
  };
  auto issue = [&](int i, const Pages& g, Raw& raw, unsigned char* k_to, unsigned char* v_to) {
    const unsigned char* block = block_of(g);
    const int slot0 = (32 * i + 8 * wave) & ps_mask;
    if constexpr (FP4) {
      // a wave's share of codes, and of scales, lies together
      const __amdgpu_buffer_rsrc_t from = rsrc(block);
      const int codes = slot0 * (D / 2), scales = slot0 * (D / 32), pair = D == 128 ? lane : lane / 2;
      const int at = lane * (D / 16);
      // K scales: of the lane's D / 8 dimensions; V scales: of its positions
      const int at_ks = lane / 8 * (D / 32) + lane % 8 * (D / 8) / 32;
      const int at_vs = pair / 16 * 8 + (D == 128 ? 0 : lane % 2 * 4);
      raw.ks = __builtin_amdgcn_raw_buffer_load_b8(from, at_ks, L.ks + scales, 0);
      if constexpr (D == 128) {
        raw.k = __builtin_amdgcn_raw_buffer_load_b64(from, at, codes, 0);
        raw.v = __builtin_amdgcn_raw_buffer_load_b64(from, at, L.v + codes, 0);
        raw.vs = __builtin_amdgcn_raw_buffer_load_b64(from, at_vs, L.vs + scales, 0);
      } else {
        raw.k[0] = __builtin_amdgcn_raw_buffer_load_b32(from, at, codes, 0);
        raw.v[0] = __builtin_amdgcn_raw_buffer_load_b32(from, at, L.v + codes, 0);
        raw.vs[0] = __builtin_amdgcn_raw_buffer_load_b32(from, at_vs, L.vs + scales, 0);
      }
    } else {
      const __amdgpu_buffer_rsrc_t rk = rsrc(block + (size_t)slot0 * D * ESZ);
      const __amdgpu_buffer_rsrc_t rv = rsrc(block + L.v + (size_t)slot0 * D * ESZ);
#pragma unroll
      for (int n = 0; n < CPW; ++n) {
        const int r = RPC * n + lane / U;  // of the wave's 8 positions
        const uint32_t ko = r * D * ESZ + 16u * ((lane % U) ^ key_swizzle<U>(8 * wave + r));
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            rk, (__attribute__((address_space(3))) void*)(k_to + 1024 * (wave * CPW + n)), 16, ko, 0,
            0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            rv, (__attribute__((address_space(3))) void*)(v_to + 1024 * (wave * CPW + n)), 16,
            1024 * n + 16 * lane, 0, 0, 0);
      }
    }
  };
  auto unpack = [&](const Raw& raw, unsigned char* kt, unsigned char* vt) {  // 4 bits to LDS
    if constexpr (FP4) {
      const int r = 8 * wave + lane / 8;
      const float f = __uint_as_float(raw.ks << 23);
      const float fs[4] = {f, f, f, f};
#pragma unroll
      for (int n = 0; n < D / 64; ++n) {
        T e[4][2];
        decode4<T>(raw.k[n], fs, e);
        const int dim = lane % 8 * (D / 8) + 8 * n;  // 8 of them
        if constexpr (kB) {
          *reinterpret_cast<bf16x8*>(kt + r * D * ESZ + 16 * (dim / 8 ^ key_swizzle<U>(r))) =
              bf16x8{e[0][0], e[0][1], e[1][0], e[1][1], e[2][0], e[2][1], e[3][0], e[3][1]};
        } else {
#pragma unroll
          for (int k = 0; k < 2; ++k)
            *reinterpret_cast<f32x4*>(kt + r * D * ESZ +
                                      16 * ((dim / 4 + k) ^ key_swizzle<U>(r))) =
                f32x4{e[2 * k][0], e[2 * k][1], e[2 * k + 1][0], e[2 * k + 1][1]};
        }
      }
      // values: columns 2 pair, 2 pair + 1 of 8 positions (or 4 of them at d = 64)
      const int pair = D == 128 ? lane : lane / 2;
      unsigned char* vp = vt + (wave * D + 2 * pair) * 8 * ESZ + (D == 128 ? 0 : lane % 2 * 4 * ESZ);
      constexpr int N = D / 16;  // positions
      T e[N][2];
#pragma unroll
      for (int n = 0; n < D / 64; ++n) {
        float g[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) g[k] = __uint_as_float((raw.vs[n] >> (8 * k) & 0xffu) << 23);
        decode4<T>(raw.v[n], g, e + 4 * n);
      }
      typedef T Column __attribute__((ext_vector_type(N)));
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        Column x;
#pragma unroll
        for (int n = 0; n < N; ++n) x[n] = e[n][k];
        *reinterpret_cast<Column*>(vp + k * 8 * ESZ) = x;
      }
    }
  };

  // ---- the running softmax, as in the attention of whole prompts -----------------------
  float m = kMaxFloor, ms = kMaxFloor, limit = kMaxFloor, l = 0.f;
  bool fused = true;
  f32x16 o[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) o[i] = f32x16{};
  const int key_row = (c & 0x13) | (c & 4) << 1 | (c & 8) >> 1;  // bits 2 and 3 exchanged

  constexpr int NB = kBuffers<T, D, FP4>, AHEAD = kTilesAhead<T, D, FP4>;
  Raw raw[2];
  uint32_t bits_in[NB];
  Pages first[AHEAD];
#pragma unroll
  for (int x = 0; x < AHEAD; ++x) first[x] = lookup(t_begin + x);
  Pages ahead = lookup(t_begin + AHEAD);
#pragma unroll
  for (int x = 0; x < AHEAD; ++x)
    if (t_begin + x < t_end) {
      bits_in[x] = bits_of(t_begin + x, first[x]);
      issue(t_begin + x, first[x], raw[x % 2], lds.k[x], lds.v[x]);
    }
  // the queries arrive here, before the loop: a wait for them inside it would be one
  // for the copies too
#pragma unroll
  for (int k = 0; k < kRowSteps<T, D>; ++k) asm volatile("" : "+v"(q[k]));
  unpack(raw[0], lds.k[0], lds.v[0]);
  auto step = [&](int i, auto slot) {
    constexpr int S = decltype(slot)::value, N = (S + AHEAD) % NB;
    unsigned char *kt = lds.k[S], *vt = lds.v[S];
    const uint32_t bits = bits_in[S];
    // this wave's copies of tile i have landed (those of tile i + 1 may be on their
    // way), and what it has decoded is written; then everyone's, and tile i - 1 is read
    constexpr int kNoVm = 0xc00f, kNoExp = 0x70;
    if (FP4)
      __builtin_amdgcn_s_waitcnt(kNoVm | kNoExp);
    else if (AHEAD == 2 && i + 1 < t_end)
      __builtin_amdgcn_s_waitcnt(2 * CPW | kNoExp);
    else
      __builtin_amdgcn_s_waitcnt(kNoExp);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (i + AHEAD < t_end) {
      bits_in[N] = bits_of(i + AHEAD, ahead);
      issue(i + AHEAD, ahead, raw[N % 2], lds.k[N], lds.v[N]);
      ahead = lookup(i + AHEAD + 1);
    }
    // Positions that cannot be read (behind the last shared one, or without a page)
    // have weight 0, and what lies there may be anything, also infinities and NaN:
    // their values are cleared, by each wave in its octet.
    if (bits != ~0u && bits != 0) {
      T* oct = reinterpret_cast<T*>(vt) + wave * D * 8;
      for (int x = lane; x < D * 8; x += kWave)
        if (!(bits >> (8 * wave + x % 8) & 1)) oct[x] = (T)0.f;
      __syncthreads();
    }
    if (wave_has && bits != 0) {
      Operands<T, D> in;
      in.read(kt, vt, lane, key_row);
      f32x16 sc = f32x16{};
      in.logits(kt, lane, key_row, q, sc);
      // register 8 j + e: position e of octet 2 j + h
      const bool masked = bits != ~0u || __any(32 * i + 32 > see);
      if (masked) {
        const int n = see - 32 * i;  // of the lane's row
        const uint32_t sees = n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
        const uint32_t mine = place((bits & sees) >> (8 * h));
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (!(mine & 1u << (16 * (r / 8) + r % 8))) sc[r] = -INFINITY;
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
        limit = fused ? mn + p.lazy : -INFINITY;
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
      in.values(vt, lane, sc, o);
    }
    if (FP4 && i + 1 < t_end) unpack(raw[(S + 1) % 2], lds.k[(S + 1) % NB], lds.v[(S + 1) % NB]);
  };
  for (int i = t_begin; i < t_end; i += NB) {
    step(i, std::integral_constant<int, 0>());
    if (i + 1 < t_end) step(i + 1, std::integral_constant<int, 1>());
    if constexpr (NB == 3)
      if (i + 2 < t_end) step(i + 2, std::integral_constant<int, 2>());
  }

  // ---- the rows' states, row by row --------------------------------------------------
  l = add_xor<32>(l);
  if (!fused) ms = m * a.scale_log2;
  if (!has_row) return;
  const size_t rows_all = (size_t)a.S * a.n_q * a.Hq;
  const size_t part = split * rows_all + ((size_t)s * a.n_q + qi) * a.Hq + hq;
  if (h == 0) {
    p.shared_parts[p.splits * rows_all * D + part] = ms;
    p.shared_parts[p.splits * rows_all * (D + 1) + part] = l;
  }
  store_row<float, D>(p.shared_parts + part * D, h, 1.f, o);
}

// Tiles of 32 positions of a run: the fewest that leave no workgroup a second run, if
// there are that many workgroups. Runs are whole tiles, so with t tiles of rows and
// heads, n positions' tiles in all and W workgroups that is between n / W and
// n / (W - t); for up to 16 groups the lanes try 64 lengths between (80 sequences of 5
// groups in 4 bits 58 to 44 us). For more, every workgroup would go through all groups
// first. us, by the longest and so, groups of 2 to 6, d = 128, bf16 and 4 bits: 32 that share
// up to 6000, one key-value head, 27 / 29 and 31 / 32; 48 of up to 8000 38 / 39 and 42 / 44; 64
// of up to 6000 41 / 43 and 44 / 46. With 4 key-value heads it would gain: 17 of up to 12000
// 64 / 70 and 58 / 62, 32 of up to 6000 71 / 78 and 58 / 62.
__device__ __forceinline__ int run_tiles(const PrefixArgs& p, int lane, const Group& mine) {
  const CacheAttnArgs& a = p.c;
  const float W = p.shared_blocks, heads = a.cache.Hkv;
  float n = 0.f, t = 0.f;
  for (int g = lane; g < a.n_groups; g += kWave) {
    const Group x = g < kWave ? mine : group_of(a, g);
    n += (float)x.row_tiles() * (float)x.tiles() * heads;
    t += (float)x.row_tiles() * heads;
  }
  n = wave_sum(n), t = wave_sum(t);
  const int lo = max(kLeastTiles, (int)fminf(ceilf(n / W), 1e9f));
  if (t >= W) return __builtin_amdgcn_readfirstlane(lo);
  const int hi = max(lo, (int)fminf(ceilf(n / (W - t)), 1e9f));
  if (a.n_groups > 16) return __builtin_amdgcn_readfirstlane(hi);
  const int per = lo + (int)((long long)(hi - lo) * lane / (kWave - 1));
  float runs = 0.f;
  for (int g = 0; g < a.n_groups; ++g) {
    const Group x{0, __builtin_amdgcn_readlane(mine.rows, g), __builtin_amdgcn_readlane(mine.P, g)};
    runs += (float)x.row_tiles() * (float)runs_of(x.tiles(), per, p.splits) * heads;
  }
  const unsigned long long fits = __ballot(runs <= W);
  return __builtin_amdgcn_readlane(per, fits ? (int)__builtin_ctzll(fits) : kWave - 1);
}

// Workgroup w of those that take shared positions: the runs of all groups, row tiles
// and key-value heads in one line, of which it takes every p.shared_blocks-th. Groups
// are looked at 64 at a time, one per lane.
template <typename T, int D, bool FP4>
__device__ __forceinline__ void shared_runs(const PrefixArgs& p, int w, const Buffers& lds) {
  const CacheAttnArgs& a = p.c;
  const int lane = threadIdx.x % kWave;
  Group mine{0, 0, 0};  // the lane's group of those looked at
  if (lane < a.n_groups) mine = group_of(a, lane);
  const int per = run_tiles(p, lane, mine);
  if (w == 0 && threadIdx.x == 0) *p.per = per;
  long long before = 0;  // runs of the groups before g0
  long long next = w;
  for (int g0 = 0; g0 < a.n_groups; g0 += kWave) {
    if (g0 > 0) mine = g0 + lane < a.n_groups ? group_of(a, g0 + lane) : Group{0, 0, 0};
    const int runs = runs_of(mine.tiles(), per, p.splits);
    const int n = mine.row_tiles() * runs * a.cache.Hkv;  // at most 2^24 tiles of 64 runs
    const int incl = wave_incl_scan(n), all = last_lane(incl);
    while (next < before + all) {
      const int x = (int)(next - before);
      const int at = __popcll(__ballot(incl <= x));
      const Group t{__builtin_amdgcn_readlane(mine.first, at),
                    __builtin_amdgcn_readlane(mine.rows, at),
                    __builtin_amdgcn_readlane(mine.P, at)};
      const int i = x - __builtin_amdgcn_readlane(incl - n, at);
      const int r = __builtin_amdgcn_readlane(runs, at);
      // runs of one row tile and head, then heads, then row tiles: those that read the
      // same positions lie a multiple of the runs apart
      shared_run<T, D, FP4>(p, t, i / (r * a.cache.Hkv) * kTile, i / r % a.cache.Hkv, i % r, r, lds);
      __syncthreads();  // the tiles in LDS are read
      next += p.shared_blocks;
    }
    before += all;
  }
}

template <typename T, int D, bool FP4, int NT>
constexpr int kPrefixPerCu = D == 128 ? 2 : kPerCu<T, D, FP4, NT>;

template <typename T, int D, bool FP4, int NT>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(kPrefixPerCu<T, D, FP4, NT>)))
void prefix_kernel(PrefixArgs a) {
  constexpr int TILE = 32 * D * sizeof(T), kThird = kBuffers<T, D, FP4> == 3 ? TILE : 16;
  __shared__ __attribute__((aligned(16))) unsigned char k0[TILE], k1[TILE], k2[kThird];
  __shared__ __attribute__((aligned(16))) unsigned char v0[TILE], v1[TILE], v2[kThird];
  const int n = a.shared_blocks;
  // (assigned: LDS addresses in an initializer do not compile without optimisation)
  if ((int)blockIdx.x < n) {
    Buffers lds;
    lds.k[0] = k0, lds.k[1] = k1, lds.k[2] = k2;
    lds.v[0] = v0, lds.v[1] = v1, lds.v[2] = v2;
    shared_runs<T, D, FP4>(a, blockIdx.x, lds);
  } else {
    SharedExchange<D> area;
    area.o[0] = k0, area.o[1] = k1, area.o[2] = v0, area.o[3] = v1;
    cache_attention_run<T, D, FP4, NT, true>(a.c, blockIdx.x - n, gridDim.x - n, area);
  }
}

// Joins one row's states, a wave a row: those of its own positions (parts of its
// segment, or the one that a whole segment left) and those of the shared ones. The
// lanes take 4 columns of 256 / D states each at a time.
template <typename T, int D, int NT>
__global__ __launch_bounds__(kThreads) void prefix_join_kernel(PrefixArgs p) {
  constexpr int R = NT * kRows, TPP = D / 4, PG = kWave / TPP;
  const CacheAttnArgs& a = p.c;
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int seg = blockIdx.x, heads = a.cache.Hkv * a.row_tiles;
  const int rr = blockIdx.y * kWaves + wave;
  const int s = seg / heads, hr = seg % heads;
  const int kvh = hr / a.row_tiles, row = hr % a.row_tiles * R + rr;
  if (rr >= R || row >= a.n_q * a.G) return;
  const int4 join = *reinterpret_cast<const int4*>(a.joins + 4 * (size_t)seg);
  const int first_own = join.x, n_own = join.y, P = join.z;
  if (n_own == 1 && P == 0) return;  // stored already
  const int n_shared = P > 0 ? runs_of((P + 31) / 32, *p.per, p.splits) : 0, n = n_own + n_shared;
  const size_t at = ((size_t)s * a.n_q + row / a.G) * a.Hq + kvh * a.G + row % a.G;
  const size_t rows_all = (size_t)a.S * a.n_q * a.Hq;
  struct State {
    const float *o, *m, *l;
  };
  auto state = [&](int i) {
    if (i >= n_own) {
      const size_t part = (i - n_own) * rows_all + at;
      return State{p.shared_parts + part * D, p.shared_parts + p.splits * rows_all * D + part,
                   p.shared_parts + p.splits * rows_all * (D + 1) + part};
    }
    if (n_own == 1)
      return State{a.states + at * D, a.states + rows_all * D + at,
                   a.states + rows_all * (D + 1) + at};
    const float* x =
        a.parts + (size_t)(i == 0 ? first_own : 2 * (first_own / 2 + i)) * part_floats(R, D);
    return State{x + rr * D, x + R * D + rr, x + R * (D + 1) + rr};
  };
  float m = kMaxFloor, l = 0.f;
  for (int i = lane; i < n; i += kWave) {  // a running sum per lane, then over the lanes
    const State x = state(i);
    const float mi = *x.m, mn = fmaxf(m, mi);
    l = l * exp2_hw(m - mn) + *x.l * exp2_hw(mi - mn);
    m = mn;
  }
  const float mine = m;
#pragma unroll
  for (int k = 1; k < kWave; k *= 2) m = fmaxf(m, __shfl_xor(m, k, kWave));
  l *= exp2_hw(mine - m);
#pragma unroll
  for (int k = 1; k < kWave; k *= 2) l += __shfl_xor(l, k, kWave);
  const int d0 = lane % TPP * 4;
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int i = lane / TPP; i < n; i += PG) {
    const State x = state(i);
    acc += exp2_hw(*x.m - m) * *reinterpret_cast<const f32x4*>(x.o + d0);
  }
#pragma unroll
  for (int k = TPP; k < kWave; k *= 2)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], k, kWave);
  if (lane >= TPP) return;
  const float inv = l > 0.f ? 1.f / l : 0.f;
  T* y = static_cast<T*>(a.Y) + at * D + d0;
  if constexpr (Elem<T>::kBf16)
    *reinterpret_cast<bf16x4*>(y) = bf16x4{(bf16)(acc[0] * inv), (bf16)(acc[1] * inv),
                                           (bf16)(acc[2] * inv), (bf16)(acc[3] * inv)};
  else
    *reinterpret_cast<f32x4*>(y) = acc * inv;
  if (a.lse && lane == 0) a.lse[at] = l > 0.f ? (m + log2_hw(l)) * kLn2 : -INFINITY;
}

int row_tiles_of(int n_q, int G, int NT) { return (n_q * G + NT * kRows - 1) / (NT * kRows); }

// Parts of the workspace, in floats (joins and per: as many 4-byte integers).
struct Plan {
  int splits;
  size_t parts, states, shared, joins;
};
Plan plan_of(int S, int n_groups, int n_q, int Hq, int Hkv, int D) {
  const long long rows = (long long)S * n_q * (Hq / Hkv);
  Plan p;
  // four times the runs of a tile that fill the device if all groups were alike: the
  // longest shared positions are divided finer; none where the tiles alone fill it
  const long long own = std::max((rows + kTile - 1) / kTile, (long long)n_groups) * Hkv;
  constexpr int kBlocks = 256;
  p.splits = own >= kBlocks ? 1
                            : (int)std::min<long long>(4 * ((kBlocks + own - 1) / own), kMaxSplits);
  p.parts = kMaxWorkgroups * 2 * part_floats(kRows, D);
  p.states = ((size_t)S * n_q * Hq * (D + 2) + 3) / 4 * 4;
  p.shared = ((size_t)S * n_q * Hq * p.splits * (D + 2) + 3) / 4 * 4;
  p.joins = (size_t)S * Hkv * row_tiles_of(n_q, Hq / Hkv, 1) * 4;
  return p;
}

template <typename T, int D, bool FP4, int NT>
hipError_t launch_tiles(PrefixArgs& a, hipStream_t stream) {
  a.c.row_tiles = row_tiles_of(a.c.n_q, a.c.G, NT);
  const long long segs = (long long)a.c.S * a.c.cache.Hkv * a.c.row_tiles;
  a.c.unit = kUnit;
  DeviceInfo dev;
  hipError_t e = device_info(&dev);
  if (e != hipSuccess) return e;
  // As many workgroups as run at once, one per CU of them (the first) for the shared
  // positions: two of these on a CU take nearly twice as long. us (d = 128, bf16) with
  // 256 of 512 workgroups and with as many as the work's proportion asks for, up to 448:
  // 256 sequences that share 32000 positions 139 / 163, 64 that share 16000 41 / 42. Those
  // that find nothing shared exit, and the sequences' own positions have the others alone:
  // with nothing to share this takes longer than the attention without groups (64 groups of
  // one sequence of 4000, 16/4 heads: bf16 100 and 100, 4 bits 49 and 32; 16 of these: 32
  // and 27, 22 and 16).
  const int W = std::min(kMaxWorkgroups / NT, dev.cus * kPrefixPerCu<T, D, FP4, NT>);
  a.shared_blocks = std::min(dev.cus, W / 2);
  hipLaunchKernelGGL((prefix_kernel<T, D, FP4, NT>), dim3((unsigned)W), dim3(kThreads), 0, stream, a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((prefix_join_kernel<T, D, NT>),
                     dim3((unsigned)segs, (unsigned)(std::min(NT * kRows, a.c.n_q * a.c.G) + kWaves - 1) /
                                              kWaves),
                     dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

size_t prefix_attention_workspace(int S, int n_groups, int n_q, int Hq, int Hkv, int d) {
  const Plan p = plan_of(S, n_groups, n_q, Hq, Hkv, d);
  return (p.parts + p.states + p.shared + p.joins + 4) * sizeof(float);
}

template <typename T, int D>
hipError_t launch_prefix_attention(const CacheShape& c, int S, int n_groups, int n_q, int Hq,
                                   float scale, const void* Q, int64_t q_stride, const void* cache,
                                   const int32_t* lens, const int32_t* table,
                                   const int32_t* cu_groups, const int32_t* shared, void* Y,
                                   float* lse, void* workspace, hipStream_t stream) {
  // Caches with room for few positions are attended to without sharing, by one launch:
  // 4 sequences that share 300 positions 7.6 us instead of 11.7, 64 that share 400 of
  // 512 11.7 instead of 17.4.
  if ((long long)c.max_pages * c.page_size <= AVQ_CACHE_UNDIVIDED)
    return launch_cache_attention<T, D>(c, S, n_q, Hq, scale, Q, q_stride, cache, lens, table, Y,
                                        lse, nullptr, stream);
  const Plan plan = plan_of(S, n_groups, n_q, Hq, c.Hkv, D);
  PrefixArgs p{};
  CacheAttnArgs& a = p.c;
  a.cache = {static_cast<unsigned char*>(const_cast<void*>(cache)), table, c.n_pages, c.max_pages,
             31 - __builtin_clz((unsigned)c.page_size), c.Hkv};
  a.Q = Q, a.q_stride = q_stride, a.lens = lens, a.Y = Y, a.lse = lse;
  a.S = S, a.n_q = n_q, a.Hq = Hq, a.G = Hq / c.Hkv;
  a.scale_log2 = scale * kLog2e;
  a.cu_groups = cu_groups, a.shared = shared, a.n_groups = n_groups;
  a.parts = static_cast<float*>(workspace);
  a.states = a.parts + plan.parts;
  p.shared_parts = a.states + plan.states;
  a.joins = reinterpret_cast<int32_t*>(p.shared_parts + plan.shared);
  p.per = a.joins + plan.joins;
  p.splits = plan.splits;
  p.lazy = kLazy / a.scale_log2;
  if constexpr (Elem<T>::kBf16) {
    if (n_q * a.G > kRows)
      return c.fp4 ? launch_tiles<T, D, true, 2>(p, stream) : launch_tiles<T, D, false, 2>(p, stream);
  }
  return c.fp4 ? launch_tiles<T, D, true, 1>(p, stream) : launch_tiles<T, D, false, 1>(p, stream);
}

#define AVQ_INSTANCE(T, D)                                                                         \
  template hipError_t launch_prefix_attention<T, D>(                                               \
      const CacheShape&, int, int, int, int, float, const void*, int64_t, const void*,             \
      const int32_t*, const int32_t*, const int32_t*, const int32_t*, void*, float*, void*,        \
      hipStream_t);
AVQ_INSTANCE(bf16, 64)
AVQ_INSTANCE(bf16, 128)
AVQ_INSTANCE(float, 64)
AVQ_INSTANCE(float, 128)
#undef AVQ_INSTANCE

}  // namespace avq
