// Exact attention of the newest tokens over the paged cache (single tokens, or
// a few drafted ones): softmax(scale Q K^T) V per sequence, grouped heads.
//
// Bound by the cache: every byte of it is read once and each key takes 4 d
// flop per query row, so the rows of one key-value head (n_q tokens x Hq/Hkv
// heads) are processed together, 16 or 32 at once. Everything is computed
// transposed, keys x queries, with 16x16x32 bf16 (16x16x4 fp32) MFMA, from
// registers: nothing is staged in LDS. A wave takes 32 keys per step. Row 4 g
// + r of logit tile t is key 8 g + 4 t + r, so lane (g, c) ends up with the
// logits of query c and the 8 keys of octet g: after exp2 they are the B
// operand of the value product, whose A operand, the same octet at one
// column, lies together in the page ([d][8]). The contraction over d may run
// in any order: with a 4-bit cache lane g takes the contiguous quarter g of
// a key's row (one 16-byte load at d = 128, and one scale), decoded by one
// conversion per pair; a value byte (two columns of one key) is decoded with
// its key's scale and the pairs are separated by byte permutes.
//
// Division of the work: lengths are known on the device only. A unit is 128
// keys (one step of the workgroup's four waves) of one (row tile, head,
// sequence), or all of its keys where the cache has room for 512 at most;
// the units lie in one line, (row tile, head) slowest, then the
// sequences, and each workgroup takes an equal run of it, whatever the
// lengths. A run covers parts of one or more segments (a segment is all of
// one (row tile, head, sequence)): a whole segment is normalised and stored,
// a part leaves its running max, sum and numerator in the workspace, and a
// second launch joins the parts. At most a run's first and last segment are
// parts, so two slots per workgroup hold them.
#include "../../include/avq.h"
#include "avq_cache.hpp"
#include "avq_launch.hpp"

#include <algorithm>
#include <type_traits>

namespace avq {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kRows = 16;                  // query rows per MFMA tile
constexpr int kStep = 32;                  // keys per wave and step
constexpr int kUnit = kStep * kWaves;      // keys per step of a workgroup
// steps of sequences that are not divided
constexpr int kWholeSteps = AVQ_CACHE_UNDIVIDED / kUnit;
constexpr int kMaxWorkgroups = 1024;       // slots in the workspace
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLazy = 8.f;         // log2 units the running max may lag behind
constexpr float kMaxFloor = -3e38f;  // finite start of the running max

struct CacheAttnArgs {
  CacheArgs cache;
  const void* Q;
  int64_t q_stride;     // elements between tokens
  const int32_t* lens;  // [S]
  void* Y;
  float* lse;           // nullable
  float* parts;         // [workgroups][2] of part_floats(D): see there
  int32_t* joins;       // [segments][2]: first workgroup and its slot, parts;
                        // null where no segment is divided
  int S, n_q, Hq, G, row_tiles;
  int unit;  // keys per unit, a multiple of kUnit
  float scale_log2;
};

// cached positions of sequence s that can be read
__device__ __forceinline__ int length_of(const CacheAttnArgs& a, int s) {
  const long long cap = (long long)a.cache.max_pages << a.cache.ps_log2;
  const int n = max(a.lens[s], 0);
  return (long long)n < cap ? n : (int)cap;
}
// every segment has a unit, so that empty ones are stored too
__device__ __forceinline__ int units_of(int len, int unit) {
  return max(1, (len + unit - 1) / unit);
}

// x y, rounded before anything is subtracted from it: fused with the running
// max it would leave the max's own rounding error in the exponent, which for
// logits beyond 2^31 no weight can hold.
__device__ __forceinline__ float product_of(float x, float y) {
#pragma clang fp contract(off)
  return x * y;
}

// A part: numerators [rows][D], then maxima [rows] and sums [rows].
__host__ __device__ constexpr size_t part_floats(int rows, int D) { return (size_t)rows * (D + 2); }

template <typename T, int D, bool FP4>
struct Keys {
  static constexpr bool kB = Elem<T>::kBf16;
  static constexpr int H2 = D / 64;  // halves of 64 columns
  // raw registers of one step: keys (two tiles), values, scales
  static constexpr int KW = FP4 ? D / 32 : D * (int)sizeof(T) / 16;       // words per key tile
  static constexpr int VW = FP4 ? 4 : 4 * 8 * (int)sizeof(T) / 4;         // words per 64 columns
  uint32_t k[2][KW];
  uint32_t v[H2][VW];
  uint32_t ks[2];
  uint32_t vs[H2][2];
};

template <int N>
__device__ __forceinline__ void load_words(const unsigned char* p, uint32_t* w) {
  if constexpr (N == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    w[0] = v.x, w[1] = v.y;
  } else {
    static_assert(N % 4 == 0, "16-byte loads");
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const uint4 v = *reinterpret_cast<const uint4*>(p + 4 * i);
      w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
    }
  }
}

// Workgroups per CU: three (168 registers a lane), whose loads are in flight
// while others compute; two where a step's rows fill the registers (fp32, d =
// 128, native). Four, where they fit (4 bits), are a little slower: 64
// sequences of up to 16000 positions 136.8 us with three, 140.8 with four;
// the bf16 native cache at d = 128 spills with four (20.2 and 36.1 us for 16
// sequences of 4 tokens).
// NT: MFMA tiles of query rows that share a step's keys. Two where there are
// more than 16 rows: the cache is then read, and 4 bits decoded, half as often
// (fp32's products bound it either way: always one).
template <typename T, int D, bool FP4, int NT>
constexpr int kPerCu = NT == 2 || (!Elem<T>::kBf16 && D == 128 && !FP4) ? 2 : 3;

template <typename T, int D, bool FP4, int NT>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(kPerCu<T, D, FP4, NT>)))
void cache_attention_kernel(CacheAttnArgs a) {
  constexpr bool kB = Elem<T>::kBf16;
  using Raw = Keys<T, D, FP4>;
  constexpr int H2 = D / 64, R = NT * kRows;
  constexpr int KQ = kB ? D / 32 : D / 4;  // k-steps of the logit product
  using QFrag = typename std::conditional<kB, bf16x8, float>::type;

  __shared__ int s_wave[kWaves];
  __shared__ int s_first[3];             // where the run starts
  __shared__ float s_m[kWaves][kRows], s_l[kWaves][kRows];
  __shared__ __attribute__((aligned(16))) float s_o[kWaves][kRows][D + 4];

  const int tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave;
  const int g = lane / 16, c = lane % 16;
  const int w = blockIdx.x;

  // ---- units of each thread's sequences, and before them -------------------
  const int per = (a.S + kThreads - 1) / kThreads;
  int mine = 0, mine_len = 0;  // mine_len: length of the first
  for (int i = 0; i < per; ++i) {
    const int s = tid * per + i;
    if (s >= a.S) break;
    const int n = length_of(a, s);
    if (i == 0) mine_len = n;
    mine += units_of(n, a.unit);
  }
  const int incl = wave_incl_scan(mine);
  if (lane == kWave - 1) s_wave[wave] = incl;
  __syncthreads();
  int before = 0, total = 0;
  for (int i = 0; i < kWaves; ++i) {
    if (i < wave) before += s_wave[i];
    total += s_wave[i];
  }

  const int heads = a.cache.Hkv * a.row_tiles;
  const long long U = (long long)total * heads;
  const int W = (int)min((long long)gridDim.x, U);  // each takes a unit at least
  if (w >= W) return;
  long long u = U * w / W;
  const long long u_end = U * (w + 1) / W;
  const long long u_first = u;

  // head and sequence of the run's first unit, from the thread whose sequences
  // hold it (every sequence has a unit)
  int hr = (int)(u / total);
  int x = (int)(u % total) - (before + incl - mine);
  if (x >= 0 && x < mine) s_first[0] = tid * per, s_first[1] = x, s_first[2] = mine_len;
  __syncthreads();
  int s = s_first[0], len = s_first[2], n_units = units_of(len, a.unit);
  x = s_first[1];
  while (x >= n_units && s + 1 < a.S) {
    x -= n_units;
    ++s;
    len = length_of(a, s);
    n_units = units_of(len, a.unit);
  }

  const PageLayout L = page_layout(FP4, sizeof(T), 1 << a.cache.ps_log2, D);
  const int ps_mask = (1 << a.cache.ps_log2) - 1;
  const int rows_all = a.n_q * a.G;

  while (true) {
    // ---- one segment: units [x, x_end) of sequence s, head hr ---------------
    const int x_end = (int)min((long long)n_units, x + (u_end - u));
    const int steps = a.unit / kUnit, y_end = x_end * steps;  // steps of kUnit keys
    const int kvh = hr / a.row_tiles, row0 = hr % a.row_tiles * R;
    const int all_see = len - a.n_q + 1;  // keys every row sees
    int last[NT];                         // keys the lane's rows see
    QFrag q[NT][KQ];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int row = row0 + kRows * n + c;
      const bool has_row = row < rows_all;
      const int qi = has_row ? row / a.G : 0;
      const int hq = kvh * a.G + (has_row ? row % a.G : 0);
      last[n] = has_row ? len - a.n_q + qi + 1 : 0;
      const T* qp = static_cast<const T*>(a.Q) + ((size_t)s * a.n_q + qi) * a.q_stride +
                    (size_t)hq * D;
#pragma unroll
      for (int k = 0; k < KQ; ++k) {
        if constexpr (kB) {
          const int d0 = FP4 ? D / 4 * g + 8 * k : 32 * k + 8 * g;
          q[n][k] = *reinterpret_cast<const bf16x8*>(qp + d0);
        } else {
          q[n][k] = qp[FP4 ? D / 4 * g + k : 16 * (k / 4) + 4 * g + k % 4];
        }
      }
    }

    float m[NT], l[NT];
    f32x4 o[NT][H2][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      m[n] = kMaxFloor, l[n] = 0.f;
#pragma unroll
      for (int h = 0; h < H2; ++h)
#pragma unroll
        for (int k = 0; k < 4; ++k) o[n][h][k] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // ---- loads: the octet's page for values, the key rows' for keys ---------
    // Pages are looked up one step ahead; rows are not requested ahead (a
    // second set of registers costs a workgroup per CU: 141 against 137 us for
    // 64 sequences in 4 bits). Without a page (past the end, or a bad entry) a
    // lane reads page 0, which exists, and its keys take no part.
    struct Place {
      int vpage, kpage;  // -1: none
    };
    auto lookup = [&](int y) {
      Place p{-1, -1};
      const int key0 = y * kUnit + wave * kStep;
      if (y >= y_end || key0 >= len) return p;  // wave-uniform
      const int32_t* row = a.cache.table + (size_t)s * a.cache.max_pages;
      const int vpos = key0 + 8 * g, kpos = key0 + 8 * (c / 4);
      if (vpos < len) p.vpage = row[vpos >> a.cache.ps_log2];
      if (kpos < len) p.kpage = row[kpos >> a.cache.ps_log2];
      if ((unsigned)p.vpage >= (unsigned)a.cache.n_pages) p.vpage = -1;
      if ((unsigned)p.kpage >= (unsigned)a.cache.n_pages) p.kpage = -1;
      return p;
    };
    auto request = [&](int y, const Place& pl, Raw& raw) {
      const int key0 = y * kUnit + wave * kStep;
      const int vpos = key0 + 8 * g, kpos = key0 + 8 * (c / 4);
      const unsigned char* vp =
          a.cache.pool + ((size_t)max(pl.vpage, 0) * a.cache.Hkv + kvh) * L.bytes;
      const unsigned char* kp =
          a.cache.pool + ((size_t)max(pl.kpage, 0) * a.cache.Hkv + kvh) * L.bytes;
      const int oct = (vpos & ps_mask) / 8, slot0 = (kpos & ps_mask) + c % 4;
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const int slot = slot0 + 4 * tt;
        if constexpr (FP4) {
          load_words<Raw::KW>(kp + slot * (D / 2) + D / 8 * g, raw.k[tt]);
          raw.ks[tt] = kp[L.ks + slot * (D / 32) + (D / 4 * g) / 32];
        } else {
          const unsigned char* rowp = kp + (size_t)slot * D * sizeof(T);
#pragma unroll
          for (int k = 0; k < Raw::KW / 4; ++k)  // 16-byte pieces g, g + 4, ...
            load_words<4>(rowp + 64 * k + 16 * g, &raw.k[tt][4 * k]);
        }
      }
#pragma unroll
      for (int h = 0; h < H2; ++h) {
        if constexpr (FP4) {
          load_words<4>(vp + L.v + (oct * (D / 2) + 32 * h + 2 * c) * 8, raw.v[h]);
          load_words<2>(vp + L.vs + (oct * (D / 32) + 2 * h + c / 8) * 8, raw.vs[h]);
        } else {
          load_words<Raw::VW>(vp + L.v + (size_t)(oct * D + 64 * h + 4 * c) * 8 * sizeof(T),
                              raw.v[h]);
        }
      }
    };

    Place ahead = lookup(x * steps);
    for (int y = x * steps; y < y_end; ++y) {
      const int key0 = y * kUnit + wave * kStep;
      if (key0 >= len) break;
      Raw raw;
      request(y, ahead, raw);
      const bool vok = ahead.vpage >= 0;
      const int vpos = key0 + 8 * g;
      ahead = lookup(y + 1);

      // ---- logits: tile tt, keys 8 g + 4 tt + r ------------------------------
      f32x4 sc[NT][2];
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
#pragma unroll
        for (int n = 0; n < NT; ++n) sc[n][tt] = f32x4{0.f, 0.f, 0.f, 0.f};
        auto product = [&](int k, auto key) {  // step k of the contraction
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            if constexpr (kB)
              sc[n][tt] = mfma_bf16(key, q[n][k], sc[n][tt]);
            else
              sc[n][tt] = mfma_f32(key, q[n][k], sc[n][tt]);
          }
        };
        if constexpr (FP4) {
          const float scale = __uint_as_float(raw.ks[tt] << 23);
#pragma unroll
          for (int k = 0; k < D / 32; ++k) {  // a word holds 8 dimensions
            const uint32_t wd = raw.k[tt][k];
            if constexpr (kB) {
              const bf16x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(wd, scale, 0);
              const bf16x2 p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(wd, scale, 1);
              const bf16x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(wd, scale, 2);
              const bf16x2 p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(wd, scale, 3);
              product(k, bf16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]});
            } else {
              const auto p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(wd, scale, 0);
              const auto p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(wd, scale, 1);
              const auto p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(wd, scale, 2);
              const auto p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(wd, scale, 3);
              const float e[8] = {p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
#pragma unroll
              for (int i = 0; i < 8; ++i) product(8 * k + i, e[i]);
            }
          }
        } else {
#pragma unroll
          for (int k = 0; k < Raw::KW / 4; ++k) {
            if constexpr (kB) {
              product(k, __builtin_bit_cast(bf16x8, *reinterpret_cast<uint4*>(&raw.k[tt][4 * k])));
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i) product(4 * k + i, __uint_as_float(raw.k[tt][4 * k + i]));
            }
          }
        }
      }

      // ---- masks (only where a key of the step is not seen by every row), running
      // max, weights
      const bool masked = key0 + kStep > all_see || __any(!vok);
      float p[NT][8];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          p[n][i] = product_of(sc[n][i / 4][i % 4], a.scale_log2);
        if (masked) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (!vok || vpos + i >= last[n]) p[n][i] = -INFINITY;
        }
        float mx = fmaxf(fmaxf(fmaxf(p[n][0], p[n][1]), fmaxf(p[n][2], p[n][3])),
                         fmaxf(fmaxf(p[n][4], p[n][5]), fmaxf(p[n][6], p[n][7])));
        if (__any(mx > m[n] + kLazy)) {
          mx = max_xor<32>(max_xor<16>(mx));
          const float mn = fmaxf(m[n], mx);
          const float f = exp2_hw(m[n] - mn);
          m[n] = mn;
          l[n] *= f;
#pragma unroll
          for (int h = 0; h < H2; ++h)
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
              for (int r = 0; r < 4; ++r) o[n][h][k][r] *= f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          p[n][i] = exp2_hw(p[n][i] - m[n]);
          l[n] += p[n][i];
        }
      }

      // ---- values ------------------------------------------------------------
      // Masked keys have weight 0; what lies in their slots may be anything
      // (never written, or not a page of this sequence), also infinities and
      // NaN, and 0 times those is not 0: their values are cleared.
      if (masked) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const bool ok = vok && vpos + i < len;
          if constexpr (FP4) {
            if (!ok)
#pragma unroll
              for (int h = 0; h < H2; ++h) raw.vs[h][i / 4] &= ~(0xffu << (8 * (i % 4)));
          } else if constexpr (kB) {
            if (!ok)
#pragma unroll
              for (int h = 0; h < H2; ++h)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                  raw.v[h][4 * k + i / 2] &= i % 2 ? 0x0000ffffu : 0xffff0000u;
          } else {
            if (!ok)
#pragma unroll
              for (int h = 0; h < H2; ++h)
#pragma unroll
                for (int k = 0; k < 4; ++k) raw.v[h][8 * k + i] = 0u;
          }
        }
      }
      // bf16: the matrix product takes the weights rounded to bf16 (by at most
      // half a step, 2^-8; their sum l is of the unrounded ones)
      if constexpr (kB) {
        bf16x8 pb[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 8; ++i) pb[n][i] = (bf16)p[n][i];
        auto product = [&](int h, int k, const bf16x8& v) {  // columns 64 h + 4 c + k
#pragma unroll
          for (int n = 0; n < NT; ++n) o[n][h][k] = mfma_bf16(v, pb[n], o[n][h][k]);
        };
#pragma unroll
        for (int h = 0; h < H2; ++h) {
          if constexpr (FP4) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
              f[i] = __uint_as_float((raw.vs[h][i / 4] >> (8 * (i % 4)) & 0xffu) << 23);
#pragma unroll
            for (int pr = 0; pr < 2; ++pr) {  // pairs 2c, 2c + 1: columns 4c + 2 pr ..
              bf16x2 e[8];
#pragma unroll
              for (int i = 0; i < 8; i += 4) {
                const uint32_t wd = raw.v[h][2 * pr + i / 4];
                e[i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(wd, f[i], 0);
                e[i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(wd, f[i + 1], 1);
                e[i + 2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(wd, f[i + 2], 2);
                e[i + 3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(wd, f[i + 3], 3);
              }
#pragma unroll
              for (int b = 0; b < 2; ++b)
                product(h, 2 * pr + b,
                        bf16x8{e[0][b], e[1][b], e[2][b], e[3][b], e[4][b], e[5][b], e[6][b], e[7][b]});
            }
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              product(h, k, __builtin_bit_cast(bf16x8, *reinterpret_cast<uint4*>(&raw.v[h][4 * k])));
          }
        }
      } else {
        auto product = [&](int h, int k, int i, float v) {  // key i of the octet
#pragma unroll
          for (int n = 0; n < NT; ++n) o[n][h][k] = mfma_f32(v, p[n][i], o[n][h][k]);
        };
#pragma unroll
        for (int h = 0; h < H2; ++h) {
          if constexpr (FP4) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
              f[i] = __uint_as_float((raw.vs[h][i / 4] >> (8 * (i % 4)) & 0xffu) << 23);
#pragma unroll
            for (int pr = 0; pr < 2; ++pr)
#pragma unroll
              for (int i = 0; i < 8; i += 4) {
                const uint32_t wd = raw.v[h][2 * pr + i / 4];
                const auto e0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(wd, f[i], 0);
                const auto e1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(wd, f[i + 1], 1);
                const auto e2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(wd, f[i + 2], 2);
                const auto e3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(wd, f[i + 3], 3);
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                  product(h, 2 * pr + b, i, e0[b]);
                  product(h, 2 * pr + b, i + 1, e1[b]);
                  product(h, 2 * pr + b, i + 2, e2[b]);
                  product(h, 2 * pr + b, i + 3, e3[b]);
                }
              }
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
              for (int i = 0; i < 8; ++i) product(h, k, i, __uint_as_float(raw.v[h][8 * k + i]));
          }
        }
      }
    }

    // ---- the four waves joined, 16 rows at a time -------------------------------
    const long long seg = (long long)s * heads + hr;
    const int slot = u == u_first ? 0 : 1;
    const bool whole = x == 0 && x_end == n_units;
    if (tid == 0 && x == 0 && a.joins) {
      // the workgroup that holds unit v is ((v + 1) W - 1) / U
      const long long w_last = ((u + n_units) * W - 1) / U;
      a.joins[2 * seg] = 2 * w + slot;
      a.joins[2 * seg + 1] = whole ? 1 : (int)(w_last - w) + 1;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (n > 0) __syncthreads();  // the exchange area is used again
      const float ln = add_xor<32>(add_xor<16>(l[n]));
      if (g == 0) {
        s_m[wave][c] = m[n];
        s_l[wave][c] = ln;
      }
      // row 4 g + r of value tile k of half h is column 64 h + 4 (4 g + r) + k
#pragma unroll
      for (int h = 0; h < H2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *reinterpret_cast<f32x4*>(&s_o[wave][c][64 * h + 16 * g + 4 * r]) =
              f32x4{o[n][h][0][r], o[n][h][1][r], o[n][h][2][r], o[n][h][3][r]};
      __syncthreads();
      constexpr int C = D / 16;  // columns per thread
      const int rr = tid / 16, d0 = tid % 16 * C;
      float mm = s_m[0][rr];
      for (int i = 1; i < kWaves; ++i) mm = fmaxf(mm, s_m[i][rr]);
      float ll = 0.f, acc[C] = {};
      for (int i = 0; i < kWaves; ++i) {
        const float f = exp2_hw(s_m[i][rr] - mm);
        ll = fmaf(f, s_l[i][rr], ll);
#pragma unroll
        for (int k = 0; k < C; ++k) acc[k] = fmaf(f, s_o[i][rr][d0 + k], acc[k]);
      }
      const int row = kRows * n + rr, out_row = row0 + row;
      if (out_row < rows_all) {
        if (whole) {
          const int oi = out_row / a.G, oh = kvh * a.G + out_row % a.G;
          const size_t at = ((size_t)s * a.n_q + oi) * a.Hq + oh;
          const float inv = ll > 0.f ? 1.f / ll : 0.f;
          T* y = static_cast<T*>(a.Y) + at * D + d0;
#pragma unroll
          for (int k = 0; k < C; ++k) y[k] = (T)(acc[k] * inv);
          if (a.lse && d0 == 0) a.lse[at] = ll > 0.f ? (mm + log2_hw(ll)) * kLn2 : -INFINITY;
        } else {
          float* part = a.parts + (size_t)(2 * w + slot) * part_floats(R, D);
#pragma unroll
          for (int k = 0; k < C; ++k) part[row * D + d0 + k] = acc[k];
          if (d0 == 0) {
            part[R * D + row] = mm;
            part[R * D + R + row] = ll;
          }
        }
      }
    }
    u += x_end - x;
    if (u >= u_end) break;
    __syncthreads();  // the exchange area is used again
    x = 0;
    if (++s == a.S) {
      s = 0;
      ++hr;
    }
    len = length_of(a, s);
    n_units = units_of(len, a.unit);
  }
}

// Joins the parts of one row of one segment: the first part is in the slot
// that joins names, the others in slot 0 of the workgroups that follow. All
// maxima are read first, so that the numerators are plain weighted sums, read
// by all threads (4 columns each) without waiting for one another.
template <typename T, int D, int NT>
__global__ __launch_bounds__(kThreads) void cache_join_kernel(CacheAttnArgs a) {
  constexpr int R = NT * kRows;
  constexpr int TPP = D / 4;              // threads per part
  constexpr int PG = kThreads / TPP;      // parts in flight
  __shared__ float s_f[kMaxWorkgroups];   // weight of each part
  __shared__ float s_red[2 * kWaves];
  __shared__ __attribute__((aligned(16))) float s_acc[PG][D];
  const int seg = blockIdx.x, rr = blockIdx.y;
  const int n = a.joins[2 * (size_t)seg + 1];
  if (n == 1) return;
  const int first = a.joins[2 * (size_t)seg];
  const int heads = a.cache.Hkv * a.row_tiles;
  const int s = seg / heads, hr = seg % heads;
  const int kvh = hr / a.row_tiles, row = hr % a.row_tiles * R + rr;
  if (row >= a.n_q * a.G) return;
  const int tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave;
  auto part = [&](int i) {
    return a.parts + (size_t)(i == 0 ? first : 2 * (first / 2 + i)) * part_floats(R, D);
  };
  float m = kMaxFloor;
  for (int i = tid; i < n; i += kThreads) {
    s_f[i] = part(i)[R * D + rr];
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
    l = fmaf(f, part(i)[R * D + R + rr], l);
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
  for (int i = pg; i < n; i += PG)
    acc += s_f[i] * *reinterpret_cast<const f32x4*>(part(i) + rr * D + d0);
  *reinterpret_cast<f32x4*>(&s_acc[pg][d0]) = acc;
  __syncthreads();
  const size_t at = ((size_t)s * a.n_q + row / a.G) * a.Hq + kvh * a.G + row % a.G;
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
// Two tiles run on half as many workgroups.
size_t parts_bytes(int D) { return kMaxWorkgroups * 2 * part_floats(kRows, D) * sizeof(float); }

template <typename T, int D, bool FP4, int NT>
hipError_t launch_tiles(CacheAttnArgs& a, hipStream_t stream) {
  a.row_tiles = row_tiles_of(a.n_q, a.G, NT);
  const long long segs = (long long)a.S * a.cache.Hkv * a.row_tiles;
  // Short sequences are not divided: four steps take less than the joining
  // launch that dividing them needs.
  const long long room =
      (((long long)a.cache.max_pages << a.cache.ps_log2) + kUnit - 1) / kUnit;
  a.unit = kUnit * (room <= kWholeSteps ? (int)room : 1);
  const long long cap = room <= kWholeSteps ? 1 : room;  // units of a segment, at most
  if (cap == 1) a.joins = nullptr;
  // as many workgroups as run at once: one more would start when the first
  // ends, after as long again
  DeviceInfo dev;
  hipError_t e = device_info(&dev);
  if (e != hipSuccess) return e;
  const long long slots = std::min(kMaxWorkgroups / NT, dev.cus * kPerCu<T, D, FP4, NT>);
  const unsigned W = (unsigned)std::min(segs * cap, slots);
  hipLaunchKernelGGL((cache_attention_kernel<T, D, FP4, NT>), dim3(W), dim3(kThreads), 0, stream, a);
  e = hipGetLastError();
  if (e != hipSuccess || cap == 1) return e;  // segments of one unit are never in parts
  hipLaunchKernelGGL((cache_join_kernel<T, D, NT>),
                     dim3((unsigned)segs, (unsigned)std::min(NT * kRows, a.n_q * a.G)),
                     dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

size_t cache_attention_workspace(int S, int n_q, int Hq, int Hkv, int d) {
  const size_t segs = (size_t)S * Hkv * row_tiles_of(n_q, Hq / Hkv, 1);
  return parts_bytes(d) + segs * 2 * sizeof(int32_t);
}

template <typename T, int D>
hipError_t launch_cache_attention(const CacheShape& c, int S, int n_q, int Hq, float scale,
                                  const void* Q, int64_t q_stride, const void* cache,
                                  const int32_t* lens, const int32_t* table, void* Y, float* lse,
                                  void* workspace, hipStream_t stream) {
  CacheAttnArgs a;
  a.cache = {static_cast<unsigned char*>(const_cast<void*>(cache)), table, c.n_pages, c.max_pages,
             31 - __builtin_clz((unsigned)c.page_size), c.Hkv};
  a.Q = Q, a.q_stride = q_stride, a.lens = lens, a.Y = Y, a.lse = lse;
  a.parts = static_cast<float*>(workspace);
  a.joins = reinterpret_cast<int32_t*>(static_cast<unsigned char*>(workspace) + parts_bytes(D));
  a.S = S, a.n_q = n_q, a.Hq = Hq, a.G = Hq / c.Hkv;
  a.scale_log2 = scale * kLog2e;
  if constexpr (Elem<T>::kBf16) {
    if (n_q * a.G > kRows)
      return c.fp4 ? launch_tiles<T, D, true, 2>(a, stream) : launch_tiles<T, D, false, 2>(a, stream);
  }
  return c.fp4 ? launch_tiles<T, D, true, 1>(a, stream) : launch_tiles<T, D, false, 1>(a, stream);
}

#define AVQ_INSTANCE(T, D)                                                                         \
  template hipError_t launch_cache_attention<T, D>(                                                \
      const CacheShape&, int, int, int, float, const void*, int64_t, const void*, const int32_t*,  \
      const int32_t*, void*, float*, void*, hipStream_t);
AVQ_INSTANCE(bf16, 64)
AVQ_INSTANCE(bf16, 128)
AVQ_INSTANCE(float, 64)
AVQ_INSTANCE(float, 128)
#undef AVQ_INSTANCE

}  // namespace avq
