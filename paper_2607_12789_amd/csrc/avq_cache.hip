// The paged cache: appending rotated keys, values (and rotating the queries)
// and reading cached positions back.
//
// Rotation: for pairs (a, b) of dimensions, a' = a cos - b sin, b' = b cos + a
// sin in fp32 from a table of the caller's (position x pair), each product
// rounded by itself; rotated queries and keys are rounded once to the element
// type, the 4-bit codes are taken from the fp32 values.
//
// Both kernels only move bytes. Queries and keys go row by row, 8 elements
// (one chunk) per lane; a rotation whose pairs are rot/2 apart loads the
// partner's chunk too, from the cache line its own row brings in. Values go
// by octets of positions, one wave per octet of 128 columns, 2 columns per
// lane: 8 positions of a column are written as one piece (bf16 16 bytes, 4
// bits 8 bytes per pair of columns), and only octets that the call covers in
// part are written position by position.
#include "avq_cache.hpp"
#include "avq_launch.hpp"

#include <type_traits>

namespace avq {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;

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
  int n_pos, rot, interleaved, Hq, q_blocks, k_blocks;
};

// Sequence and position of packed token t (-1: of no sequence).
__device__ __forceinline__ int place(const TokenArgs& a, int t, int& pos) {
  int s = t, i = 0;
  if (a.cu) {
    int lo = 0, hi = a.S;  // cu[lo] <= t < cu[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.cu[mid] <= t) lo = mid; else hi = mid;
    }
    int b, e;
    packed_range(a.cu, lo, a.T, b, e);
    if (t < b || t >= e) return -1;
    s = lo;
    i = t - b;
  }
  const int p0 = a.start[s];
  if (p0 < 0 || p0 > 0x7fffffff - i) return -1;
  pos = p0 + i;
  return s;
}

// 8 elements as fp32
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  if constexpr (Elem<T>::kBf16) {
    const bf16x8 v = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
  } else {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  if constexpr (Elem<T>::kBf16) {
    bf16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (bf16)x[i];
    *reinterpret_cast<bf16x8*>(p) = v;
  } else {
    *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
  }
}

// Chunk u (dimensions 8u .. 8u+7) of a row, rotated to position pos. The
// products and the sum are rounded one by one (no fused multiply-add), so
// that equal inputs give equal bits wherever the row is rotated.
template <typename T>
__device__ __forceinline__ void rotated(const AppendArgs& a, const T* row, int u, int pos,
                                        float (&x)[8]) {
#pragma clang fp contract(off)
  load8(row + 8 * u, x);
  if (8 * u >= a.rot) return;
  const int half = a.rot / 2;
  const float* cs = a.cos + (size_t)pos * half;
  const float* sn = a.sin + (size_t)pos * half;
  if (a.interleaved) {
    const f32x4 c = *reinterpret_cast<const f32x4*>(cs + 4 * u);
    const f32x4 s = *reinterpret_cast<const f32x4*>(sn + 4 * u);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p = x[2 * i], q = x[2 * i + 1];
      x[2 * i] = p * c[i] - q * s[i];
      x[2 * i + 1] = q * c[i] + p * s[i];
    }
  } else {
    const bool low = 8 * u < half;
    float y[8], c[8], s[8];
    load8(row + (low ? 8 * u + half : 8 * u - half), y);
    const int i0 = low ? 8 * u : 8 * u - half;
    load8(cs + i0, c);
    load8(sn + i0, s);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float p = x[i] * c[i], q = y[i] * s[i];
      x[i] = low ? p - q : p + q;
    }
  }
}

// Queries: rows t * Hq + h
template <typename T, int D>
__device__ __forceinline__ void rotate_queries(const AppendArgs& a, int block) {
  constexpr int LPR = D / 8;
  const long long r = ((long long)block * kThreads + threadIdx.x) / LPR;
  const int u = threadIdx.x % LPR;
  if (r >= (long long)a.tok.T * a.Hq) return;
  const int t = (int)(r / a.Hq), h = (int)(r % a.Hq);
  int pos = 0;
  if (place(a.tok, t, pos) < 0 || (a.rot && pos >= a.n_pos)) return;
  float x[8];
  rotated(a, static_cast<const T*>(a.Q) + t * a.q_stride + h * D, u, pos, x);
  store8(static_cast<T*>(a.Q_out) + r * D + 8 * u, x);
}

// Keys: rows t * Hkv + h, into the cache and, rotated, into K_out
template <typename T, int D, bool FP4>
__device__ __forceinline__ void append_keys(const AppendArgs& a, int block) {
  constexpr int LPR = D / 8;
  const int Hkv = a.cache.Hkv;
  const long long r = ((long long)block * kThreads + threadIdx.x) / LPR;
  const int u = threadIdx.x % LPR;
  if (r >= (long long)a.tok.T * Hkv) return;
  const int t = (int)(r / Hkv), h = (int)(r % Hkv);
  int pos = 0;
  const int s = place(a.tok, t, pos);
  if (s < 0 || (a.rot && pos >= a.n_pos)) return;
  const PageLayout L = page_layout(FP4, sizeof(T), 1 << a.cache.ps_log2, D);
  unsigned char* page = page_of(a.cache, L.bytes, s, pos, h);
  const int slot = pos & ((1 << a.cache.ps_log2) - 1);
  float x[8];
  rotated(a, static_cast<const T*>(a.K) + t * a.k_stride + h * D, u, pos, x);
  if (a.K_out) store8(static_cast<T*>(a.K_out) + r * D + 8 * u, x);
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
    if (!page) return;
    *reinterpret_cast<uint32_t*>(page + slot * (D / 2) + 4 * u) = code;
    if (u % 4 == 0) page[L.ks + slot * (D / 32) + u / 4] = (unsigned char)e;
  } else {
    if (page) store8(reinterpret_cast<T*>(page) + slot * D + 8 * u, x);
  }
}

// An octet of positions of one (sequence, head): its wave, and which of its
// positions are among the call's tokens.
struct Octet {
  int s, pos0, t0;  // sequence, first position, packed row of that position
  unsigned mask;    // bit j: position pos0 + j is a token of this call
};
__device__ __forceinline__ Octet find_octet(const TokenArgs& a, long long slot, int lane) {
  Octet o;
  o.mask = 0;
  int b, e, p0;
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
  p0 = a.start[o.s];
  if (p0 < 0 || p0 > 0x7fffffff - (e - b) - 8) return o;
  const long long k = p0 / 8 + (slot - first);
  if (k * 8 >= (long long)p0 + (e - b)) return o;
  o.pos0 = (int)(k * 8);
  o.t0 = b + (o.pos0 - p0);
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (o.t0 + j >= b && o.t0 + j < e) o.mask |= 1u << j;
  return o;
}

template <typename T>
__device__ __forceinline__ void load2(const T* p, float& a, float& b) {
  if constexpr (Elem<T>::kBf16) {
    const bf16x2 v = *reinterpret_cast<const bf16x2*>(p);
    a = (float)v[0];
    b = (float)v[1];
  } else {
    a = p[0];
    b = p[1];
  }
}

// Values: one wave per (octet slot, head); at D = 64 the upper half takes the
// next head
template <typename T, int D, bool FP4>
__device__ __forceinline__ void append_values(const AppendArgs& a, long long wave) {
  constexpr int HPW = 128 / D;  // heads per wave
  const int lane = threadIdx.x % kWave;
  const int Hkv = a.cache.Hkv, HG = (Hkv + HPW - 1) / HPW;
  const long long slots = a.tok.cu ? octet_slots(a.tok.T, a.tok.S) : a.tok.T;
  const long long slot = wave / HG;
  if (slot >= slots) return;
  const int h = (int)(wave % HG) * HPW + lane / (D / 2);
  const int i = lane % (D / 2);  // the lane's pair of columns
  const Octet o = find_octet(a.tok, slot, lane);
  if (o.mask == 0 || h >= Hkv) return;
  unsigned mask = o.mask;
  if (a.rot) {  // positions past the table are not written
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (o.pos0 + j >= a.n_pos) mask &= ~(1u << j);
  }
  const PageLayout L = page_layout(FP4, sizeof(T), 1 << a.cache.ps_log2, D);
  unsigned char* page = page_of(a.cache, L.bytes, o.s, o.pos0, h);
  if (!page) return;
  const int oct = (o.pos0 & ((1 << a.cache.ps_log2) - 1)) / 8;
  float x[8], y[8];
  const T* V = static_cast<const T*>(a.V) + h * D + 2 * i;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    x[j] = y[j] = 0.f;
    if (mask >> j & 1) load2(V + (o.t0 + j) * a.v_stride, x[j], y[j]);
  }
  if constexpr (FP4) {
    uint32_t code[2], exps[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      code[q] = exps[q] = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int j = 4 * q + k;
        float m = fmaxf(fabsf(x[j]), fabsf(y[j]));
        m = fmaxf(m, xor16<1>(m));  // the 16 lanes of 32 dimensions
        m = fmaxf(m, xor16<2>(m));
        m = fmaxf(m, xor16<4>(m));
        m = fmaxf(m, xor16<8>(m));
        const uint32_t e = fp4_scale(m);
        const uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(
            0u, x[j], y[j], __uint_as_float(e << 23), 0) & 0xffu;
        code[q] |= c << (8 * k);
        exps[q] |= e << (8 * k);
      }
    }
    unsigned char* vc = page + L.v + (oct * (D / 2) + i) * 8;
    unsigned char* vs = page + L.vs + (oct * (D / 32) + i / 16) * 8;
    if (mask == 0xffu) {
      *reinterpret_cast<uint2*>(vc) = make_uint2(code[0], code[1]);
      if (i % 16 == 0) *reinterpret_cast<uint2*>(vs) = make_uint2(exps[0], exps[1]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (mask >> j & 1) {
          vc[j] = (unsigned char)(code[j / 4] >> (8 * (j % 4)));
          if (i % 16 == 0) vs[j] = (unsigned char)(exps[j / 4] >> (8 * (j % 4)));
        }
    }
  } else {
    T* v = reinterpret_cast<T*>(page + L.v) + (oct * D + 2 * i) * 8;
    if (mask == 0xffu) {
      store8(v, x);
      store8(v + 8, y);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (mask >> j & 1) {
          v[j] = (T)x[j];
          v[8 + j] = (T)y[j];
        }
    }
  }
}

template <typename T, int D, bool FP4>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a) {
  const int b = blockIdx.x;
  if (b < a.q_blocks) {
    rotate_queries<T, D>(a, b);
  } else if (b < a.q_blocks + a.k_blocks) {
    append_keys<T, D, FP4>(a, b - a.q_blocks);
  } else {
    append_values<T, D, FP4>(
        a, (long long)(b - a.q_blocks - a.k_blocks) * kWaves + threadIdx.x / kWave);
  }
}

struct GatherArgs {
  CacheArgs cache;
  TokenArgs tok;
  void *K, *V;
  int k_blocks;
};

// two decoded values of byte B of w
template <int B>
__device__ __forceinline__ void decode2(uint32_t w, float scale, float& a, float& b) {
  const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, B);
  a = v[0];
  b = v[1];
}

template <typename T, int D, bool FP4>
__device__ __forceinline__ void gather_keys(const GatherArgs& a, int block) {
  constexpr int LPR = D / 8;
  const int Hkv = a.cache.Hkv;
  const long long r = ((long long)block * kThreads + threadIdx.x) / LPR;
  const int u = threadIdx.x % LPR;
  if (r >= (long long)a.tok.T * Hkv) return;
  const int t = (int)(r / Hkv), h = (int)(r % Hkv);
  int pos = 0;
  const int s = place(a.tok, t, pos);
  if (s < 0) return;
  const PageLayout L = page_layout(FP4, sizeof(T), 1 << a.cache.ps_log2, D);
  const unsigned char* page = page_of(a.cache, L.bytes, s, pos, h);
  const int slot = pos & ((1 << a.cache.ps_log2) - 1);
  float x[8] = {};
  if (page) {
    if constexpr (FP4) {
      const uint32_t code = *reinterpret_cast<const uint32_t*>(page + slot * (D / 2) + 4 * u);
      const float scale =
          __uint_as_float((uint32_t)page[L.ks + slot * (D / 32) + u / 4] << 23);
      decode2<0>(code, scale, x[0], x[1]);
      decode2<1>(code, scale, x[2], x[3]);
      decode2<2>(code, scale, x[4], x[5]);
      decode2<3>(code, scale, x[6], x[7]);
    } else {
      load8(reinterpret_cast<const T*>(page) + slot * D + 8 * u, x);
    }
  }
  store8(static_cast<T*>(a.K) + r * D + 8 * u, x);
}

template <typename T, int D, bool FP4>
__device__ __forceinline__ void gather_values(const GatherArgs& a, long long wave) {
  constexpr int HPW = 128 / D;
  const int lane = threadIdx.x % kWave;
  const int Hkv = a.cache.Hkv, HG = (Hkv + HPW - 1) / HPW;
  const long long slots = a.tok.cu ? octet_slots(a.tok.T, a.tok.S) : a.tok.T;
  const long long slot = wave / HG;
  if (slot >= slots) return;
  const int h = (int)(wave % HG) * HPW + lane / (D / 2);
  const int i = lane % (D / 2);
  const Octet o = find_octet(a.tok, slot, lane);
  if (o.mask == 0 || h >= Hkv) return;
  const PageLayout L = page_layout(FP4, sizeof(T), 1 << a.cache.ps_log2, D);
  const unsigned char* page = page_of(a.cache, L.bytes, o.s, o.pos0, h);
  const int oct = (o.pos0 & ((1 << a.cache.ps_log2) - 1)) / 8;
  float x[8] = {}, y[8] = {};
  if (page) {
    if constexpr (FP4) {
      const uint2 code = *reinterpret_cast<const uint2*>(page + L.v + (oct * (D / 2) + i) * 8);
      const uint2 e = *reinterpret_cast<const uint2*>(page + L.vs + (oct * (D / 32) + i / 16) * 8);
      auto scale = [](uint32_t w, int k) { return __uint_as_float((w >> (8 * k) & 0xffu) << 23); };
      decode2<0>(code.x, scale(e.x, 0), x[0], y[0]);
      decode2<1>(code.x, scale(e.x, 1), x[1], y[1]);
      decode2<2>(code.x, scale(e.x, 2), x[2], y[2]);
      decode2<3>(code.x, scale(e.x, 3), x[3], y[3]);
      decode2<0>(code.y, scale(e.y, 0), x[4], y[4]);
      decode2<1>(code.y, scale(e.y, 1), x[5], y[5]);
      decode2<2>(code.y, scale(e.y, 2), x[6], y[6]);
      decode2<3>(code.y, scale(e.y, 3), x[7], y[7]);
    } else {
      const T* v = reinterpret_cast<const T*>(page + L.v) + (oct * D + 2 * i) * 8;
      load8(v, x);
      load8(v + 8, y);
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (o.mask >> j & 1) {
      T* p = static_cast<T*>(a.V) + ((size_t)(o.t0 + j) * Hkv + h) * D + 2 * i;
      if constexpr (Elem<T>::kBf16)
        *reinterpret_cast<bf16x2*>(p) = bf16x2{(bf16)x[j], (bf16)y[j]};
      else
        *reinterpret_cast<float2*>(p) = make_float2(x[j], y[j]);
    }
}

template <typename T, int D, bool FP4>
__global__ __launch_bounds__(kThreads) void gather_kernel(GatherArgs a) {
  const int b = blockIdx.x;
  if (b < a.k_blocks)
    gather_keys<T, D, FP4>(a, b);
  else
    gather_values<T, D, FP4>(a, (long long)(b - a.k_blocks) * kWaves + threadIdx.x / kWave);
}

// workgroups for the rows of H heads, and for the value octets
template <int D>
long long row_blocks(long long T, int H) {
  return (T * H * (D / 8) + kThreads - 1) / kThreads;
}
template <int D>
long long octet_blocks(const TokenArgs& t, int Hkv) {
  constexpr int HPW = 128 / D;
  const long long slots = t.cu ? octet_slots(t.T, t.S) : t.T;
  return (slots * ((Hkv + HPW - 1) / HPW) + kWaves - 1) / kWaves;
}

int log2_of(int x) { return 31 - __builtin_clz((unsigned)x); }

CacheArgs cache_args(const CacheShape& c, const void* pool, const int32_t* table) {
  return {static_cast<unsigned char*>(const_cast<void*>(pool)), table, c.n_pages, c.max_pages,
          log2_of(c.page_size), c.Hkv};
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
  const long long qb = Q ? row_blocks<D>(T_, Hq) : 0, kb = row_blocks<D>(T_, c.Hkv);
  const long long grid = qb + kb + octet_blocks<D>(a.tok, c.Hkv);
  if (grid > 0x7fffffff) return hipErrorInvalidConfiguration;
  a.q_blocks = (int)qb;
  a.k_blocks = (int)kb;
  if (c.fp4)
    hipLaunchKernelGGL((append_kernel<T, D, true>), dim3((unsigned)grid), dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((append_kernel<T, D, false>), dim3((unsigned)grid), dim3(kThreads), 0, stream, a);
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
  const long long kb = row_blocks<D>(T_, c.Hkv);
  const long long grid = kb + octet_blocks<D>(a.tok, c.Hkv);
  if (grid > 0x7fffffff) return hipErrorInvalidConfiguration;
  a.k_blocks = (int)kb;
  if (c.fp4)
    hipLaunchKernelGGL((gather_kernel<T, D, true>), dim3((unsigned)grid), dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((gather_kernel<T, D, false>), dim3((unsigned)grid), dim3(kThreads), 0, stream, a);
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
