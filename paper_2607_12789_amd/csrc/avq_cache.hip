// The paged cache: appending rotated keys, values (and rotating the queries)
// and reading cached positions back.
//
// Rotation: for pairs (a, b) of dimensions, a' = a cos - b sin, b' = b cos + a
// sin in fp32 from a table of the caller's (position x pair), each product
// rounded by itself; rotated queries and keys are rounded once to the element
// type, the 4-bit codes are taken from the fp32 values.
//
// Both kernels only move bytes, so every load and store of dense rows covers 1
// KB of one token: 8 elements (a chunk) per lane, 512 / d heads per wave
// (reading 256 bytes of each of four tokens instead costs a fifth more time).
// Queries and keys go token by token: a wave takes a token's place and angles
// once for up to kRowSteps such pieces, whose loads are in flight together; a
// rotation whose pairs are rot/2 apart loads the partner's chunk too, from the
// cache line its own row brings in. Values go by octets of positions: a lane
// holds 8 positions of its 8 columns, which are pieces of the page's [d][8]
// layout (4 bits: the conversion puts each position's code into its byte of
// the piece); only octets that the call covers in part are written position by
// position.
#include "avq_cache.hpp"
#include "avq_launch.hpp"

#include <algorithm>
#include <type_traits>

namespace avq {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kRowSteps = 4;  // pieces of a token that a wave takes

// Workgroups lie in rows of kGridRow: a launch has fewer than 2^32 threads along x.
constexpr long long kGridRow = 1 << 22;
__device__ __forceinline__ int block_of() {
  return (int)(blockIdx.y * (unsigned)kGridRow + blockIdx.x);
}

struct TokenArgs {
  const int32_t* cu;     // [S + 1], null: one token per sequence
  const int32_t* start;  // [S]
  int S, T;
};

struct AppendArgs {
  CacheArgs cache;
  TokenArgs tok;
  const void *Q, *K, *V;
  int64_t q_stride, k_stride, v_stride;  // elements between tokens
  void *Q_out, *K_out;                   // nullable
  const float *cos, *sin;                // [n_pos][rot / 2], null without rotation
  int n_pos, rot, interleaved, Hq;
  int q_steps, k_steps;  // pieces of a token's queries (0 without them) and keys
  int groups, steps;     // waves per token, pieces per wave
  int row_blocks;        // workgroups for queries and keys; the others take values
};

// A position that no table reaches and no angles cover (both hold fewer than
// 2^31): it stands for all beyond it.
constexpr int kNoPlace = 0x7fffffff;

// Tokens that the cache holds before the call's (start[s]). A negative number:
// -1, the sequence takes no part, or with kAll its positions have no page.
template <bool kAll>
__device__ __forceinline__ int start_of(const TokenArgs& a, int s) {
  const int p = a.start[s];
  return p >= 0 ? p : kAll ? kNoPlace : -1;
}

// Sequence and position of packed token t, the same for the whole wave (-1: of
// no sequence).
template <bool kAll>
__device__ __forceinline__ int place(const TokenArgs& a, int t, int lane, int& pos) {
  int s = t, i = 0;
  if (a.cu) {
    s = find_sequence(a.S, t, lane, [&](int k) { return (long long)a.cu[k]; });
    int b, e;
    packed_range(a.cu, s, a.T, b, e);
    if (t < b || t >= e) return -1;
    i = t - b;
  }
  const int p0 = start_of<kAll>(a, s);
  if (p0 < 0) return -1;
  pos = p0 + min(i, kNoPlace - p0);
  return s;
}

// A chunk as it lies in memory
template <typename T>
struct Chunk {
  uint4 w[8 * sizeof(T) / 16];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (unsigned i = 0; i < sizeof(w) / 16; ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (unsigned i = 0; i < sizeof(w) / 16; ++i) reinterpret_cast<uint4*>(p)[i] = w[i];
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (Elem<T>::kBf16) {
      const uint32_t x[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
      return __uint_as_float(i % 2 ? x[i / 2] & 0xffff0000u : x[i / 2] << 16);
    } else {
      const uint4 v = w[i / 4];
      const uint32_t x[4] = {v.x, v.y, v.z, v.w};
      return __uint_as_float(x[i % 4]);
    }
  }
  __device__ __forceinline__ void set(const float (&x)[8]) {
    if constexpr (Elem<T>::kBf16) {
      w[0] = __builtin_bit_cast(uint4, bf16x8{(bf16)x[0], (bf16)x[1], (bf16)x[2], (bf16)x[3],
                                              (bf16)x[4], (bf16)x[5], (bf16)x[6], (bf16)x[7]});
    } else {
      w[0] = __builtin_bit_cast(uint4, f32x4{x[0], x[1], x[2], x[3]});
      w[1] = __builtin_bit_cast(uint4, f32x4{x[4], x[5], x[6], x[7]});
    }
  }
};

// x: chunk u (dimensions 8u .. 8u+7) of a row; y: the chunk of its partners,
// rot / 2 dimensions away (not used interleaved); c, s: the cosines and sines
// of its pairs. The products and the sum are rounded one by one (no fused
// multiply-add), so that equal inputs give equal bits wherever a row is
// rotated.
template <typename T>
__device__ __forceinline__ void rotate(bool interleaved, bool low, const Chunk<T>& y,
                                       const float (&c)[8], const float (&s)[8], float (&x)[8]) {
#pragma clang fp contract(off)
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p = x[2 * i], q = x[2 * i + 1];
      x[2 * i] = p * c[i] - q * s[i];
      x[2 * i + 1] = q * c[i] + p * s[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float p = x[i] * c[i], q = y.get(i) * s[i];
      x[i] = low ? p - q : p + q;
    }
  }
}

// Queries and keys of one token: pieces of 512 / D heads, the queries' first.
template <typename T, int D, bool FP4>
__device__ __forceinline__ void append_rows(const AppendArgs& a) {
  constexpr int LPR = D / 8, HPS = kWave / LPR;  // lanes per row, heads per piece
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(block_of() * kWaves + threadIdx.x / kWave);
  const int t = wave / a.groups;
  if (t >= a.tok.T) return;
  const int first = wave % a.groups * a.steps;
  int pos = 0;
  const int s = place<false>(a.tok, t, lane, pos);
  if (s < 0 || (a.rot && pos >= a.n_pos)) return;
  const int u = lane % LPR, hl = lane / LPR;
  const int half = a.rot / 2;
  const bool turn = 8 * u < a.rot, low = 8 * u < half;
  const int other = low ? 8 * u + half : 8 * u - half;
  const T* q_row = static_cast<const T*>(a.Q) + t * a.q_stride;
  const T* k_row = static_cast<const T*>(a.K) + t * a.k_stride;
  // piece i: queries or keys, and the lane's head in it
  auto piece = [&](int i, bool& keys, int& h) {
    keys = i >= a.q_steps;
    h = (keys ? i - a.q_steps : i) * HPS + hl;
    return i < a.q_steps + a.k_steps && h < (keys ? a.cache.Hkv : a.Hq);
  };
  Chunk<T> own[kRowSteps], partner[kRowSteps];
#pragma unroll
  for (int k = 0; k < kRowSteps; ++k) {
    bool keys;
    int h;
    if (k < a.steps && piece(first + k, keys, h)) {
      const T* p = (keys ? k_row : q_row) + h * D;
      own[k].load(p + 8 * u);
      if (turn && !a.interleaved) partner[k].load(p + other);
    }
  }
  float c[8], sn[8];
  if (turn) {  // 4 pairs of the chunk, or the 8 its dimensions belong to
    const int at = a.interleaved ? 4 * u : low ? 8 * u : 8 * u - half;
    const float* cp = a.cos + (size_t)pos * half + at;
    const float* sp = a.sin + (size_t)pos * half + at;
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      if (i == 0 || !a.interleaved) {
        const f32x4 cv = *reinterpret_cast<const f32x4*>(cp + i);
        const f32x4 sv = *reinterpret_cast<const f32x4*>(sp + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) c[i + e] = cv[e], sn[i + e] = sv[e];
      }
    }
  }
  const PageLayout L = page_layout(FP4, sizeof(T), 1 << a.cache.ps_log2, D);
  unsigned char* page = page_of(a.cache, L.bytes, s, pos, 0);
  const int slot = pos & ((1 << a.cache.ps_log2) - 1);
#pragma unroll
  for (int k = 0; k < kRowSteps; ++k) {
    bool keys;
    int h;
    if (k >= a.steps || !piece(first + k, keys, h)) continue;  // a row's lanes together
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = own[k].get(i);
    if (turn) rotate<T>(a.interleaved, low, partner[k], c, sn, x);
    Chunk<T> out;
    out.set(x);
    T* dense = static_cast<T*>(keys ? a.K_out : a.Q_out);
    if (dense)
      out.store(dense + ((size_t)t * (keys ? a.cache.Hkv : a.Hq) + h) * D + 8 * u);
    if (!keys || !page) continue;
    unsigned char* dst = page + (size_t)h * L.bytes;
    if constexpr (FP4) {
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(x[i]));
      m = fmaxf(m, xor16<1>(m));  // the 4 lanes of 32 dimensions
      m = fmaxf(m, xor16<2>(m));
      const uint32_t e = fp4_scale(m);
      const float scale = __uint_as_float(e << 23);
      uint32_t code = 0;
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[0], x[1], scale, 0);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[2], x[3], scale, 1);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[4], x[5], scale, 2);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[6], x[7], scale, 3);
      *reinterpret_cast<uint32_t*>(dst + slot * (D / 2) + 4 * u) = code;
      if (u % 4 == 0) dst[L.ks + slot * (D / 32) + u / 4] = (unsigned char)e;
    } else {
      out.store(reinterpret_cast<T*>(dst) + slot * D + 8 * u);
    }
  }
}

// An octet of positions of one sequence, and which of its positions are among
// the call's tokens.
struct Octet {
  int s, pos0, t0;  // sequence, first position (at most kNoPlace), its packed row
  unsigned mask;    // bit j: position pos0 + j is a token of this call
};
template <bool kAll>
__device__ __forceinline__ Octet find_octet(const TokenArgs& a, long long slot, int lane) {
  Octet o;
  o.mask = 0;
  int b, e;
  long long first = 0;
  if (a.cu) {
    o.s = find_sequence(a.S, slot, lane, [&](int s) {
      return (long long)min(max(a.cu[s], 0), a.T) / 8 + 2LL * s;
    });
    packed_range(a.cu, o.s, a.T, b, e);
    first = b / 8 + 2LL * o.s;
  } else {
    o.s = (int)slot;
    b = o.s;
    e = b + 1;
    first = slot;
  }
  const int p0 = start_of<kAll>(a, o.s);
  if (p0 < 0) return o;
  const long long pos0 = (p0 / 8 + (slot - first)) * 8;
  if (pos0 >= (long long)p0 + (e - b)) return o;
  o.pos0 = (int)min(pos0, (long long)kNoPlace);
  o.t0 = (int)(b + (pos0 - p0));
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (o.t0 + j >= b && o.t0 + j < e) o.mask |= 1u << j;
  return o;
}

__host__ __device__ inline long long slots_of(const TokenArgs& a) {
  return a.cu ? octet_slots(a.T, a.S) : a.T;
}

// Values: one wave per octet slot and 512 / D heads
template <typename T, int D, bool FP4>
__device__ __forceinline__ void append_values(const AppendArgs& a) {
  constexpr int LPR = D / 8, HPS = kWave / LPR;
  const int lane = threadIdx.x % kWave;
  const long long wave = (long long)(block_of() - a.row_blocks) * kWaves +
                         __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int Hkv = a.cache.Hkv, HG = (Hkv + HPS - 1) / HPS;
  const long long slot = wave / HG;
  if (slot >= slots_of(a.tok)) return;
  const int u = lane % LPR, h = (int)(wave % HG) * HPS + lane / LPR;
  const Octet o = find_octet<false>(a.tok, slot, lane);
  unsigned mask = o.mask;
  if (a.rot && mask) {  // positions past the table are not written
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (o.pos0 >= a.n_pos - j) mask &= ~(1u << j);
  }
  if (mask == 0 || h >= Hkv) return;
  const PageLayout L = page_layout(FP4, sizeof(T), 1 << a.cache.ps_log2, D);
  unsigned char* page = page_of(a.cache, L.bytes, o.s, o.pos0, h);
  if (!page) return;
  const int oct = (o.pos0 & ((1 << a.cache.ps_log2) - 1)) / 8;
  Chunk<T> x[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    x[j] = Chunk<T>{};
    if (mask >> j & 1)
      x[j].load(static_cast<const T*>(a.V) + (o.t0 + j) * a.v_stride + h * D + 8 * u);
  }
  if constexpr (FP4) {
    uint32_t code[4][2], exps[2] = {0, 0};  // pairs of columns x halves of the octet
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float v[8], m = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i] = x[j].get(i);
        m = fmaxf(m, fabsf(v[i]));
      }
      m = fmaxf(m, xor16<1>(m));  // the 4 lanes of 32 dimensions
      m = fmaxf(m, xor16<2>(m));
      const uint32_t e = fp4_scale(m);
      const float scale = __uint_as_float(e << 23);
      exps[j / 4] |= e << (8 * (j % 4));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t& w = code[i][j / 4];
        if (j % 4 == 0) w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[2 * i], v[2 * i + 1], scale, 0);
        if (j % 4 == 1) w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2 * i], v[2 * i + 1], scale, 1);
        if (j % 4 == 2) w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2 * i], v[2 * i + 1], scale, 2);
        if (j % 4 == 3) w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2 * i], v[2 * i + 1], scale, 3);
      }
    }
    unsigned char* vc = page + L.v + (oct * (D / 2) + 4 * u) * 8;
    unsigned char* vs = page + L.vs + (oct * (D / 32) + u / 4) * 8;
    if (mask == 0xffu) {
      *reinterpret_cast<uint4*>(vc) = make_uint4(code[0][0], code[0][1], code[1][0], code[1][1]);
      *reinterpret_cast<uint4*>(vc + 16) = make_uint4(code[2][0], code[2][1], code[3][0], code[3][1]);
      if (u % 4 == 0) *reinterpret_cast<uint2*>(vs) = make_uint2(exps[0], exps[1]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (mask >> j & 1) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            vc[8 * i + j] = (unsigned char)(code[i][j / 4] >> (8 * (j % 4)));
          if (u % 4 == 0) vs[j] = (unsigned char)(exps[j / 4] >> (8 * (j % 4)));
        }
    }
  } else {
    T* v = reinterpret_cast<T*>(page + L.v) + (oct * D + 8 * u) * 8;
    if (mask == 0xffu) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float col[8] = {x[0].get(i), x[1].get(i), x[2].get(i), x[3].get(i),
                              x[4].get(i), x[5].get(i), x[6].get(i), x[7].get(i)};
        Chunk<T> out;
        out.set(col);
        out.store(v + 8 * i);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (mask >> j & 1) {
#pragma unroll
          for (int i = 0; i < 8; ++i) v[8 * i + j] = (T)x[j].get(i);
        }
    }
  }
}

template <typename T, int D, bool FP4>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a) {
  if (block_of() < a.row_blocks)
    append_rows<T, D, FP4>(a);
  else
    append_values<T, D, FP4>(a);
}

struct GatherArgs {
  CacheArgs cache;
  TokenArgs tok;
  void *K, *V;
  int groups, steps, row_blocks;  // as in AppendArgs
  int tokens;                     // per wave
};

// two decoded values of byte B of w
template <int B>
__device__ __forceinline__ void decode2(uint32_t w, float scale, float& a, float& b) {
  const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, B);
  a = v[0];
  b = v[1];
}
// The one decoded value that neither type holds, 4 at a scale of 2^126 (2^128),
// becomes the type's largest finite one. In a branch: 4945 tokens of 6 heads of
// 64 take 6.5 us, 7.3 with every value clamped.
template <typename T>
__device__ __forceinline__ void saturate(float scale, float (&x)[8]) {
  constexpr float kTop = Elem<T>::kBf16 ? 0x1.fep127f : 0x1.fffffep127f;
  if (__any(scale >= 0x1p126f)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_fmed3f(x[i], -kTop, kTop);
  }
}
__device__ __forceinline__ float scale_of(uint32_t w, int byte) {
  return __uint_as_float((w >> (8 * byte) & 0xffu) << 23);
}

template <typename T, int D, bool FP4>
__device__ __forceinline__ void gather_keys(const GatherArgs& a) {
  constexpr int LPR = D / 8, HPS = kWave / LPR;
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(block_of() * kWaves + threadIdx.x / kWave);
  const int t0 = wave / a.groups * a.tokens;
  if (t0 >= a.tok.T) return;
  const int first = wave % a.groups * a.steps;
  const int u = lane % LPR, Hkv = a.cache.Hkv;
  const PageLayout L = page_layout(FP4, sizeof(T), 1 << a.cache.ps_log2, D);
  // kRowSteps pieces: a.tokens tokens of a.steps pieces each
  uint32_t code[kRowSteps], scale[kRowSteps];
  Chunk<T> out[kRowSteps];
  T* dst[kRowSteps];
#pragma unroll
  for (int k = 0; k < kRowSteps; ++k) {
    const int t = t0 + k / a.steps, h = (first + k % a.steps) * HPS + lane / LPR;
    code[k] = scale[k] = 0;
    out[k] = Chunk<T>{};
    dst[k] = nullptr;
    int pos = 0, s = -1;
    if (k < a.steps * a.tokens && t < a.tok.T) s = place<true>(a.tok, t, lane, pos);
    if (s >= 0 && h < Hkv) {
      dst[k] = static_cast<T*>(a.K) + ((size_t)t * Hkv + h) * D + 8 * u;
      const unsigned char* src = page_of(a.cache, L.bytes, s, pos, h);
      const int slot = pos & ((1 << a.cache.ps_log2) - 1);
      if (src) {
        if constexpr (FP4) {
          code[k] = *reinterpret_cast<const uint32_t*>(src + slot * (D / 2) + 4 * u);
          scale[k] = src[L.ks + slot * (D / 32) + u / 4];
        } else {
          out[k].load(reinterpret_cast<const T*>(src) + slot * D + 8 * u);
        }
      }
    }
  }
#pragma unroll
  for (int k = 0; k < kRowSteps; ++k) {
    if constexpr (FP4) {
      float x[8];
      const float sc = scale_of(scale[k], 0);
      decode2<0>(code[k], sc, x[0], x[1]);
      decode2<1>(code[k], sc, x[2], x[3]);
      decode2<2>(code[k], sc, x[4], x[5]);
      decode2<3>(code[k], sc, x[6], x[7]);
      saturate<T>(sc, x);
      out[k].set(x);
    }
    if (dst[k]) out[k].store(dst[k]);
  }
}

template <typename T, int D, bool FP4>
__device__ __forceinline__ void gather_values(const GatherArgs& a) {
  constexpr int LPR = D / 8, HPS = kWave / LPR;
  const int lane = threadIdx.x % kWave;
  const long long wave = (long long)(block_of() - a.row_blocks) * kWaves +
                         __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int Hkv = a.cache.Hkv, HG = (Hkv + HPS - 1) / HPS;
  const long long slot = wave / HG;
  if (slot >= slots_of(a.tok)) return;
  const int u = lane % LPR, h = (int)(wave % HG) * HPS + lane / LPR;
  const Octet o = find_octet<true>(a.tok, slot, lane);
  if (o.mask == 0 || h >= Hkv) return;
  const PageLayout L = page_layout(FP4, sizeof(T), 1 << a.cache.ps_log2, D);
  const unsigned char* page = page_of(a.cache, L.bytes, o.s, o.pos0, h);
  const int oct = (o.pos0 & ((1 << a.cache.ps_log2) - 1)) / 8;
  T* dst = static_cast<T*>(a.V) + h * D + 8 * u;
  const size_t stride = (size_t)Hkv * D;
  if constexpr (FP4) {
    uint4 w[2] = {};
    uint2 e = {};
    if (page) {
      w[0] = *reinterpret_cast<const uint4*>(page + L.v + (oct * (D / 2) + 4 * u) * 8);
      w[1] = *reinterpret_cast<const uint4*>(page + L.v + (oct * (D / 2) + 4 * u) * 8 + 16);
      e = *reinterpret_cast<const uint2*>(page + L.vs + (oct * (D / 32) + u / 4) * 8);
    }
    const uint32_t code[4][2] = {{w[0].x, w[0].y}, {w[0].z, w[0].w}, {w[1].x, w[1].y}, {w[1].z, w[1].w}};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float scale = scale_of(j < 4 ? e.x : e.y, j % 4);
      float x[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t c = code[i][j / 4];
        if (j % 4 == 0) decode2<0>(c, scale, x[2 * i], x[2 * i + 1]);
        if (j % 4 == 1) decode2<1>(c, scale, x[2 * i], x[2 * i + 1]);
        if (j % 4 == 2) decode2<2>(c, scale, x[2 * i], x[2 * i + 1]);
        if (j % 4 == 3) decode2<3>(c, scale, x[2 * i], x[2 * i + 1]);
      }
      saturate<T>(scale, x);
      Chunk<T> out;
      out.set(x);
      if (o.mask >> j & 1) out.store(dst + (o.t0 + j) * stride);
    }
  } else {
    Chunk<T> col[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      col[i] = Chunk<T>{};
      if (page) col[i].load(reinterpret_cast<const T*>(page + L.v) + (oct * D + 8 * u + i) * 8);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float x[8] = {col[0].get(j), col[1].get(j), col[2].get(j), col[3].get(j),
                          col[4].get(j), col[5].get(j), col[6].get(j), col[7].get(j)};
      Chunk<T> out;
      out.set(x);
      if (o.mask >> j & 1) out.store(dst + (o.t0 + j) * stride);
    }
  }
}

template <typename T, int D, bool FP4>
__global__ __launch_bounds__(kThreads) void gather_kernel(GatherArgs a) {
  if (block_of() < a.row_blocks)
    gather_keys<T, D, FP4>(a);
  else
    gather_values<T, D, FP4>(a);
}

int log2_of(int x) { return 31 - __builtin_clz((unsigned)x); }

CacheArgs cache_args(const CacheShape& c, const void* pool, const int32_t* table) {
  return {static_cast<unsigned char*>(const_cast<void*>(pool)), table, c.n_pages, c.max_pages,
          log2_of(c.page_size), c.Hkv};
}

// pieces of H heads
template <int D>
int steps_of(int H) {
  return (H + 512 / D - 1) / (512 / D);
}
// Waves per token and pieces per wave: even shares of at most kRowSteps, one
// piece each where that gives fewer than 1024 waves (a step of 64 sequences
// with 40 heads of 128: 5.8 us with four pieces per wave, 5.0 with one).
template <typename Args>
void share_rows(Args& a, int pieces) {
  const int most = (long long)a.tok.T * pieces < 1024 ? 1 : kRowSteps;
  a.groups = (pieces + most - 1) / most;
  a.steps = (pieces + a.groups - 1) / a.groups;
}
dim3 grid_of(long long blocks) {
  return dim3((unsigned)std::min(blocks, kGridRow), (unsigned)((blocks + kGridRow - 1) / kGridRow));
}
template <int D>
long long octet_blocks(const TokenArgs& t, int Hkv) {
  return (slots_of(t) * steps_of<D>(Hkv) + kWaves - 1) / kWaves;
}

}  // namespace

template <typename T, int D>
hipError_t launch_cache_append(const CacheShape& c, int S, int T_, int Hq, int rot, int n_pos,
                               int interleaved, const void* Q, int64_t q_stride, const void* K,
                               int64_t k_stride, const void* V, int64_t v_stride,
                               const int32_t* cu, const int32_t* start, const int32_t* table,
                               const float* cos, const float* sin, void* cache, void* Q_out,
                               void* K_out, hipStream_t stream) {
  AppendArgs a;
  a.cache = cache_args(c, cache, table);
  a.tok = {cu, start, S, T_};
  a.Q = Q, a.K = K, a.V = V;
  a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride;
  a.Q_out = Q_out, a.K_out = K_out;
  a.cos = cos, a.sin = sin;
  a.n_pos = n_pos, a.rot = rot, a.interleaved = interleaved, a.Hq = Hq;
  a.q_steps = Q ? steps_of<D>(Hq) : 0;
  a.k_steps = steps_of<D>(c.Hkv);
  share_rows(a, a.q_steps + a.k_steps);
  const long long rows = ((long long)T_ * a.groups + kWaves - 1) / kWaves;
  const long long grid = rows + octet_blocks<D>(a.tok, c.Hkv);
  if ((grid + kGridRow) * kWaves > 0x7fffffff) return hipErrorInvalidConfiguration;
  a.row_blocks = (int)rows;
  if (c.fp4)
    hipLaunchKernelGGL((append_kernel<T, D, true>), grid_of(grid), dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((append_kernel<T, D, false>), grid_of(grid), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_cache_gather(const CacheShape& c, int S, int T_, const void* cache,
                               const int32_t* cu, const int32_t* start, const int32_t* table,
                               void* K, void* V, hipStream_t stream) {
  GatherArgs a;
  a.cache = cache_args(c, cache, table);
  a.tok = {cu, start, S, T_};
  a.K = K, a.V = V;
  share_rows(a, steps_of<D>(c.Hkv));
  // several tokens per wave where there are waves enough without (20685 tokens
  // of 4 heads of 128 in 4 bits: 12.6 us, 14.8 one by one; 4945 of 6 of 64: 6.9
  // and 6.4)
  a.tokens = (long long)T_ * a.groups < 16384 ? 1 : kRowSteps / a.steps;
  const long long rows = (((long long)T_ + a.tokens - 1) / a.tokens * a.groups + kWaves - 1) / kWaves;
  const long long grid = rows + octet_blocks<D>(a.tok, c.Hkv);
  if ((grid + kGridRow) * kWaves > 0x7fffffff) return hipErrorInvalidConfiguration;
  a.row_blocks = (int)rows;
  if (c.fp4)
    hipLaunchKernelGGL((gather_kernel<T, D, true>), grid_of(grid), dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((gather_kernel<T, D, false>), grid_of(grid), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

#define AVQ_CACHE_INSTANCES(T, D)                                                                 \
  template hipError_t launch_cache_append<T, D>(                                                  \
      const CacheShape&, int, int, int, int, int, int, const void*, int64_t, const void*, int64_t, \
      const void*, int64_t, const int32_t*, const int32_t*, const int32_t*, const float*,         \
      const float*, void*, void*, void*, hipStream_t);                                            \
  template hipError_t launch_cache_gather<T, D>(const CacheShape&, int, int, const void*,         \
                                                const int32_t*, const int32_t*, const int32_t*,   \
                                                void*, void*, hipStream_t);
AVQ_CACHE_INSTANCES(bf16, 64)
AVQ_CACHE_INSTANCES(bf16, 128)
AVQ_CACHE_INSTANCES(float, 64)
AVQ_CACHE_INSTANCES(float, 128)
#undef AVQ_CACHE_INSTANCES

}  // namespace avq
