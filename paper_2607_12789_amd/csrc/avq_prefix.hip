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
// one launch: its first workgroups take the shared positions of a tile of rows, in
// a.splits equal runs, the others the sequences' own ones. All leave running maxima,
// sums and numerators, and a second launch joins them, row by row.
#include "avq_cache_attention.hpp"
#include "avq_launch.hpp"

#include <algorithm>

namespace avq {

namespace {

constexpr int kTile = 128;       // rows of a workgroup
constexpr int kLeastTiles = 4;   // tiles of 32 positions that a workgroup takes, at least
constexpr int kMaxSplits = 64;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct PrefixArgs {
  CacheAttnArgs c;
  int tiles, splits;   // tiles of rows, at most; workgroups that share one's positions
  int shared_blocks;   // workgroups for the shared positions
  float lazy;          // kLazy / scale_log2
  float* shared_parts; // [tiles][Hkv][splits] of part_floats(kTile, D)
};

struct RowTile {
  int first, rows, r0;  // the group's first sequence, its rows, the tile's first one
  int P;                // shared positions
};

__device__ __forceinline__ long long tile_of(int first, int g, int per) {
  return (long long)first * per / kTile + g;
}
// Runs of P positions, the same on the joining side.
__device__ __forceinline__ int runs_of(int P, int splits) {
  return max(1, min(splits, (P + 31) / 32 / kLeastTiles));
}
__device__ __forceinline__ bool find_rows(const CacheAttnArgs& a, int tile, int lane, RowTile& t) {
  const int per = a.n_q * a.G;
  const int g = find_sequence(a.n_groups, tile, lane,
                              [&](int k) { return tile_of(group_first(a, k), k, per); });
  t.first = group_first(a, g);
  const int end = group_first(a, g + 1);
  t.rows = (end - t.first) * per;
  t.r0 = (int)(tile - tile_of(t.first, g, per)) * kTile;
  if (t.r0 < 0 || t.r0 >= t.rows) return false;
  t.P = shared_length(a, g, t.first, end);
  return t.P > 0;
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

// Run `split` of the shared positions of one tile of rows and one key-value head.
template <typename T, int D, bool FP4>
__device__ __forceinline__ void shared_run(const PrefixArgs& p, int tile, int hkv, int split,
                                           unsigned char* lds) {
  constexpr bool kB = Elem<T>::kBf16;
  constexpr int ESZ = sizeof(T), U = D * ESZ / 16, TILE = 32 * D * ESZ;
  constexpr int RPC = 64 / U, CPW = 8 / RPC, DT = D / 32;
  constexpr int KQ = kB ? D / 16 : D / 2;
  using Frag = typename std::conditional<kB, bf16x8, float>::type;
  const CacheAttnArgs& a = p.c;
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int h = lane / 32, c = lane % 32;
  RowTile t;
  if (!find_rows(a, tile, lane, t)) return;
  const int n_tiles = (t.P + 31) / 32, runs = runs_of(t.P, p.splits);
  if (split >= runs) return;
  const int t_begin = (int)((long long)n_tiles * split / runs);
  const int t_end = (int)((long long)n_tiles * (split + 1) / runs);

  // ---- the lane's row -------------------------------------------------------------
  const int per = a.n_q * a.G;
  const int row0 = t.r0 + 32 * wave, row = row0 + c;
  const bool has_row = row < t.rows, wave_has = row0 < t.rows;
  const int at_row = min(row, t.rows - 1), s = t.first + at_row / per;
  const int qi = at_row % per / a.G, hq = hkv * a.G + at_row % a.G;
  const int see = min(t.P, length_of(a, s) - a.n_q + qi + 1);  // positions it sees
  Frag q[KQ];
  {
    const T* qp = static_cast<const T*>(a.Q) + ((size_t)s * a.n_q + qi) * a.q_stride +
                  (size_t)hq * D;
#pragma unroll
    for (int k = 0; k < KQ; ++k) {
      if constexpr (kB) {
        q[k] = *reinterpret_cast<const bf16x8*>(qp + 16 * k + 8 * h);
      } else if (k % 4 == 0) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(qp + 2 * k + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) q[k + e] = v[e];
      }
    }
  }

  // ---- pages, and tiles to LDS -------------------------------------------------------
  // A tile lies in one page, or (16 positions a page) in two; wave w copies its
  // positions 8 w .. 8 w + 7. Without a page the first one is read, which exists, and
  // the positions take no part.
  const PageLayout L = page_layout(FP4, ESZ, 1 << a.cache.ps_log2, D);
  const int ps_mask = (1 << a.cache.ps_log2) - 1;
  const int32_t* pages = a.cache.table + (size_t)t.first * a.cache.max_pages;
  struct Pages {
    int id[2];  // -1: none
  };
  auto lookup = [&](int i) {
    Pages r{{-1, -1}};
    if (i >= t_end) return r;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int pos = 32 * i + 16 * k;
      if (pos >= t.P) continue;
      const int id = pages[pos >> a.cache.ps_log2];
      r.id[k] = (unsigned)id < (unsigned)a.cache.n_pages ? id : -1;
    }
    return r;
  };
  auto bits_of = [&](int i, const Pages& g) {  // positions that can be read
    const int n = t.P - 32 * i;
    const uint32_t in = n >= 32 ? ~0u : (1u << n) - 1u;
    return in & ((g.id[0] < 0 ? 0u : 0xffffu) | (g.id[1] < 0 ? 0u : 0xffff0000u));
  };
  struct Raw {  // 4 bits: a thread's share of a tile
    uint32_t k[D / 64], v[D / 64], vs[D / 64], ks;
  };
  auto block_of = [&](const Pages& g) {
    const int id = max(wave < 2 ? g.id[0] : g.id[1], 0);
    return a.cache.pool + ((size_t)id * a.cache.Hkv + hkv) * L.bytes;
  };
  auto issue = [&](int i, const Pages& g, Raw& raw) {
    const unsigned char* block = block_of(g);
    const int slot0 = (32 * i + 8 * wave) & ps_mask, b = i & 1;
    if constexpr (FP4) {
      const unsigned char* kp = block + (slot0 + lane / 8) * (D / 2) + lane % 8 * (D / 16);
      const unsigned char* vp = block + L.v + slot0 / 8 * (D * 4) + lane * (D / 16);
      // K scales: of the lane's D / 8 dimensions; V scales: of its positions
      raw.ks = block[L.ks + (slot0 + lane / 8) * (D / 32) + lane % 8 * (D / 8) / 32];
      const int pair = D == 128 ? lane : lane / 2;
      const unsigned char* sp = block + L.vs + (slot0 / 8 * (D / 32) + pair / 16) * 8 +
                                (D == 128 ? 0 : lane % 2 * 4);
#pragma unroll
      for (int n = 0; n < D / 64; ++n) {
        raw.k[n] = reinterpret_cast<const uint32_t*>(kp)[n];
        raw.v[n] = reinterpret_cast<const uint32_t*>(vp)[n];
        raw.vs[n] = reinterpret_cast<const uint32_t*>(sp)[n];
      }
    } else {
      const __amdgpu_buffer_rsrc_t rk = rsrc(block + (size_t)slot0 * D * ESZ);
      const __amdgpu_buffer_rsrc_t rv = rsrc(block + L.v + (size_t)slot0 * D * ESZ);
#pragma unroll
      for (int n = 0; n < CPW; ++n) {
        const int r = RPC * n + lane / U;  // of the wave's 8 positions
        const uint32_t ko = r * D * ESZ + 16u * ((lane % U) ^ key_swizzle<U>(8 * wave + r));
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            rk, (__attribute__((address_space(3))) void*)(lds + b * TILE + 1024 * (wave * CPW + n)),
            16, ko, 0, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            rv,
            (__attribute__((address_space(3))) void*)(lds + (2 + b) * TILE + 1024 * (wave * CPW + n)),
            16, 1024 * n + 16 * lane, 0, 0, 0);
      }
    }
  };
  auto unpack = [&](int i, const Raw& raw) {  // 4 bits to the tile's buffer
    if constexpr (FP4) {
      unsigned char *kt = lds + (i & 1) * TILE, *vt = lds + (2 + (i & 1)) * TILE;
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
#pragma unroll
      for (int n = 0; n < D / 64; ++n) {
        float g[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) g[k] = __uint_as_float((raw.vs[n] >> (8 * k) & 0xffu) << 23);
        T e[4][2];
        decode4<T>(raw.v[n], g, e);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          unsigned char* to = vp + k * 8 * ESZ + n * 4 * ESZ;
          if constexpr (kB)
            *reinterpret_cast<bf16x4*>(to) = bf16x4{e[0][k], e[1][k], e[2][k], e[3][k]};
          else
            *reinterpret_cast<f32x4*>(to) = f32x4{e[0][k], e[1][k], e[2][k], e[3][k]};
        }
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

  Raw raw;
  Pages now = lookup(t_begin), ahead = lookup(t_begin + 1);
  issue(t_begin, now, raw);
  unpack(t_begin, raw);
  for (int i = t_begin; i < t_end; ++i) {
    const int b = i & 1;
    const uint32_t bits = bits_of(i, now);
    now = ahead;
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();  // tile i has landed, tile i - 1 is read
    const bool more = i + 1 < t_end;
    if (more) {
      issue(i + 1, now, raw);
      ahead = lookup(i + 2);
    }
    if (wave_has && bits != 0) {
      const unsigned char *kt = lds + b * TILE, *vt = lds + (2 + b) * TILE;
      f32x16 sc = f32x16{};
      const unsigned char* rowp = kt + key_row * (D * ESZ);
#pragma unroll
      for (int k = 0; k < U / 2; ++k) {
        const unsigned char* x = rowp + 16 * ((2 * k + h) ^ key_swizzle<U>(key_row));
        if constexpr (kB) {
          sc = mfma32(*reinterpret_cast<const bf16x8*>(x), q[k], sc);
        } else {
          const f32x4 v = *reinterpret_cast<const f32x4*>(x);
#pragma unroll
          for (int e = 0; e < 4; ++e) sc = mfma32(v[e], q[4 * k + e], sc);
        }
      }
      // register 8 j + e: position e of octet 2 j + h
      const bool masked = bits != ~0u || __any(32 * i + 32 > see);
      if (masked) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int k = 16 * (r / 8) + 8 * h + r % 8;
          if (!(bits >> k & 1) || 32 * i + k >= see) sc[r] = -INFINITY;
        }
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
      // Positions that cannot be read have weight 0, and what lies there may be
      // anything, also infinities and NaN: their values are cleared. bf16: the matrix
      // product takes the weights rounded to bf16 (by at most half a step, 2^-8),
      // their sum l is of the unrounded ones.
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t ok = bits >> (16 * j + 8 * h) & 0xffu;
        const unsigned char* oct = vt + (2 * j + h) * D * 8 * ESZ;
        if constexpr (kB) {
          bf16x8 w;
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] = (bf16)sc[8 * j + e];
#pragma unroll
          for (int k = 0; k < DT; ++k) {
            u32x4 x = *reinterpret_cast<const u32x4*>(oct + (32 * k + c) * 16);
            if (bits != ~0u) {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                x[e] &= (ok >> (2 * e) & 1 ? 0xffffu : 0u) |
                        (ok >> (2 * e + 1) & 1 ? 0xffff0000u : 0u);
            }
            o[k] = mfma32(__builtin_bit_cast(bf16x8, x), w, o[k]);
          }
        } else {
#pragma unroll
          for (int k = 0; k < DT; ++k)
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
              f32x4 x = *reinterpret_cast<const f32x4*>(oct + ((32 * k + c) * 8 + e) * 4);
#pragma unroll
              for (int n = 0; n < 4; ++n) {
                if (bits != ~0u && !(ok >> (e + n) & 1)) x[n] = 0.f;
                o[k] = mfma32(x[n], sc[8 * j + e + n], o[k]);
              }
            }
        }
      }
    }
    if (more) unpack(i + 1, raw);
  }

  // ---- the rows' states, row by row --------------------------------------------------
  l = add_xor<32>(l);
  if (!fused) ms = m * a.scale_log2;
  float* part = p.shared_parts +
                (((size_t)tile * a.cache.Hkv + hkv) * p.splits + split) * part_floats(kTile, D);
  const int r0 = 32 * wave + c;
  if (!has_row) return;
  if (h == 0) {
    part[kTile * D + r0] = ms;
    part[kTile * (D + 1) + r0] = l;
  }
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      *reinterpret_cast<f32x4*>(part + r0 * D + 32 * i + 2 * r + 4 * h) =
          f32x4{o[i][r], o[i][r + 1], o[i][r + 2], o[i][r + 3]};
}

template <typename T, int D, bool FP4, int NT>
constexpr int kPrefixPerCu = sizeof(T) == 4 && D == 128 ? 2 : kPerCu<T, D, FP4, NT>;

template <typename T, int D, bool FP4, int NT>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(kPrefixPerCu<T, D, FP4, NT>)))
void prefix_kernel(PrefixArgs a) {
  constexpr int kTiles = 4 * 32 * D * sizeof(T);
  __shared__ __attribute__((aligned(16))) unsigned char lds[std::max<int>(kTiles, sizeof(Exchange<D>))];
  if ((int)blockIdx.x < a.shared_blocks) {
    const int i = blockIdx.x / a.splits;
    shared_run<T, D, FP4>(a, i / a.c.cache.Hkv, i % a.c.cache.Hkv, blockIdx.x % a.splits, lds);
  } else {
    cache_attention_run<T, D, FP4, NT, true>(a.c, blockIdx.x - a.shared_blocks,
                                             gridDim.x - a.shared_blocks,
                                             *reinterpret_cast<Exchange<D>*>(lds));
  }
}

// Joins one row's states: those of its own positions (parts of its segment, or the one
// that a whole segment left) and those of the shared ones.
template <typename T, int D, int NT>
__global__ __launch_bounds__(kThreads) void prefix_join_kernel(PrefixArgs p) {
  constexpr int R = NT * kRows;
  constexpr int TPP = D / 4;          // threads per state
  constexpr int PG = kThreads / TPP;  // states in flight
  __shared__ float s_f[kMaxWorkgroups + kMaxSplits];  // weight of each state
  __shared__ float s_red[2 * kWaves];
  __shared__ __attribute__((aligned(16))) float s_acc[PG][D];
  const CacheAttnArgs& a = p.c;
  const int tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave;
  const int seg = blockIdx.x, rr = blockIdx.y, heads = a.cache.Hkv * a.row_tiles;
  const int s = seg / heads, hr = seg % heads;
  const int kvh = hr / a.row_tiles, row = hr % a.row_tiles * R + rr, per = a.n_q * a.G;
  if (row >= per) return;
  // the group's shared positions, and its tile that holds the row
  const int g = find_sequence(a.n_groups, s, lane,
                              [&](int k) { return (long long)group_first(a, k); });
  const int first = group_first(a, g), end = group_first(a, g + 1);
  const int P = s >= first && s < end ? shared_length(a, g, first, end) : 0;
  const int n_own = a.joins[2 * (size_t)seg + 1], first_own = a.joins[2 * (size_t)seg];
  if (n_own == 1 && P == 0) return;  // stored already
  const int n_shared = P > 0 ? runs_of(P, p.splits) : 0, n = n_own + n_shared;
  const size_t at = ((size_t)s * a.n_q + row / a.G) * a.Hq + kvh * a.G + row % a.G;
  const size_t rows_all = (size_t)a.S * a.n_q * a.Hq;
  const int r = (s - first) * per + row, rt = r % kTile;
  const float* shared_parts =
      p.shared_parts +
      ((size_t)(tile_of(first, g, per) + r / kTile) * a.cache.Hkv + kvh) * p.splits *
          part_floats(kTile, D);
  struct State {
    const float *o, *m, *l;
  };
  auto state = [&](int i) {
    if (i >= n_own) {
      const float* x = shared_parts + (size_t)(i - n_own) * part_floats(kTile, D);
      return State{x + rt * D, x + kTile * D + rt, x + kTile * (D + 1) + rt};
    }
    if (n_own == 1)
      return State{a.states + at * D, a.states + rows_all * D + at,
                   a.states + rows_all * (D + 1) + at};
    const float* x =
        a.parts + (size_t)(i == 0 ? first_own : 2 * (first_own / 2 + i)) * part_floats(R, D);
    return State{x + rr * D, x + R * D + rr, x + R * (D + 1) + rr};
  };
  float m = kMaxFloor;
  for (int i = tid; i < n; i += kThreads) {
    s_f[i] = *state(i).m;
    m = fmaxf(m, s_f[i]);
  }
#pragma unroll
  for (int k = 1; k < kWave; k *= 2) m = fmaxf(m, __shfl_xor(m, k, kWave));
  if (lane == 0) s_red[wave] = m;
  __syncthreads();
  for (int i = 0; i < kWaves; ++i) m = fmaxf(m, s_red[i]);
  float l = 0.f;
  for (int i = tid; i < n; i += kThreads) {
    const float f = exp2_hw(s_f[i] - m);
    s_f[i] = f;
    l = fmaf(f, *state(i).l, l);
  }
#pragma unroll
  for (int k = 1; k < kWave; k *= 2) l += __shfl_xor(l, k, kWave);
  if (lane == 0) s_red[kWaves + wave] = l;
  __syncthreads();
  l = 0.f;
  for (int i = 0; i < kWaves; ++i) l += s_red[kWaves + i];
  const int pg = tid / TPP, d0 = tid % TPP * 4;
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = pg; i < n; i += PG) acc += s_f[i] * *reinterpret_cast<const f32x4*>(state(i).o + d0);
  *reinterpret_cast<f32x4*>(&s_acc[pg][d0]) = acc;
  __syncthreads();
  const float inv = l > 0.f ? 1.f / l : 0.f;
  if (tid < D) {
    float y = 0.f;
#pragma unroll
    for (int i = 0; i < PG; ++i) y += s_acc[i][tid];
    static_cast<T*>(a.Y)[at * D + tid] = (T)(y * inv);
  }
  if (a.lse && tid == 0) a.lse[at] = l > 0.f ? (m + log2_hw(l)) * kLn2 : -INFINITY;
}

int row_tiles_of(int n_q, int G, int NT) { return (n_q * G + NT * kRows - 1) / (NT * kRows); }

// Parts of the workspace, in floats (joins: as many 4-byte integers).
struct Plan {
  long long tiles;
  int splits;
  size_t parts, states, shared, joins;
};
Plan plan_of(int S, int n_groups, int n_q, int Hq, int Hkv, int D) {
  const long long rows = (long long)S * n_q * (Hq / Hkv);
  Plan p;
  p.tiles = rows / kTile + n_groups;
  // as if all groups had as many sequences; about a workgroup per CU
  const long long own = std::max((rows + kTile - 1) / kTile, (long long)n_groups) * Hkv;
  p.splits = (int)std::min<long long>(std::max(1LL, 256 / own), kMaxSplits);
  p.parts = kMaxWorkgroups * 2 * part_floats(kRows, D);
  p.states = ((size_t)S * n_q * Hq * (D + 2) + 3) / 4 * 4;
  p.shared = (size_t)p.tiles * Hkv * p.splits * part_floats(kTile, D);
  p.joins = (size_t)S * Hkv * row_tiles_of(n_q, Hq / Hkv, 1) * 2;
  return p;
}

template <typename T, int D, bool FP4, int NT>
hipError_t launch_tiles(PrefixArgs& a, hipStream_t stream) {
  a.c.row_tiles = row_tiles_of(a.c.n_q, a.c.G, NT);
  const long long segs = (long long)a.c.S * a.c.cache.Hkv * a.c.row_tiles;
  // short sequences are not divided, as without groups
  const long long room =
      (((long long)a.c.cache.max_pages << a.c.cache.ps_log2) + kUnit - 1) / kUnit;
  a.c.unit = kUnit * (room <= kWholeSteps ? (int)room : 1);
  const long long cap = room <= kWholeSteps ? 1 : room;  // units of a segment, at most
  DeviceInfo dev;
  hipError_t e = device_info(&dev);
  if (e != hipSuccess) return e;
  const long long slots = std::min(kMaxWorkgroups / NT, dev.cus * kPrefixPerCu<T, D, FP4, NT>);
  const unsigned W = (unsigned)std::min(segs * cap, slots);
  hipLaunchKernelGGL((prefix_kernel<T, D, FP4, NT>), dim3((unsigned)a.shared_blocks + W),
                     dim3(kThreads), 0, stream, a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((prefix_join_kernel<T, D, NT>),
                     dim3((unsigned)segs, (unsigned)std::min(NT * kRows, a.c.n_q * a.c.G)),
                     dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

size_t prefix_attention_workspace(int S, int n_groups, int n_q, int Hq, int Hkv, int d) {
  const Plan p = plan_of(S, n_groups, n_q, Hq, Hkv, d);
  return (p.parts + p.states + p.shared + p.joins) * sizeof(float);
}

template <typename T, int D>
hipError_t launch_prefix_attention(const CacheShape& c, int S, int n_groups, int n_q, int Hq,
                                   float scale, const void* Q, int64_t q_stride, const void* cache,
                                   const int32_t* lens, const int32_t* table,
                                   const int32_t* cu_groups, const int32_t* shared, void* Y,
                                   float* lse, void* workspace, hipStream_t stream) {
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
  p.tiles = (int)plan.tiles, p.splits = plan.splits;
  p.shared_blocks = (int)(plan.tiles * c.Hkv * plan.splits);
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
