// Exact attention of whole prompts: packed sequences of different lengths,
// grouped heads, causal or not.
//
//   S_ij = scale q_i . k_j,  Y_i = sum_j exp(S_ij - lse_i) v_j,
//   lse_i = ln sum_j exp(S_ij), over the keys j of i's sequence, with the
//   causal mask those with j <= i + Lk - Lq (the queries are the last Lq of
//   the Lk positions).
//
// One pass over the keys with a running maximum and sum. A workgroup of four
// waves owns 128 queries of one head, 32 per wave; the keys and values of its
// head stream through LDS in tiles, double buffered, by direct global->LDS
// copies. Products are transposed, as in the codeword attention: S^T = K Q^T
// with 32x32x16 bf16 (32x32x2 fp32) MFMA, so that a lane owns one query (with
// its partner lane l ^ 32) and 16 of 32 keys; the weights that come out of
// exp2 are the B operand of Y^T = V^T P^T, whose contraction over the keys is
// taken in the order in which the lanes hold them. Its A operand, several
// keys at one column, is read from the row-major value tile with the LDS
// transpose read (bf16: 4 keys of 16 columns per 16 lanes; fp32 needs one key
// per lane and no transpose).
//
// Lengths are known on the device only: the grid has Tq / 128 + S tiles per
// head, at least as many as the sequences need, each workgroup finds its tile
// and those left over exit; or the tiles' keys are dealt out in equal runs.
#include "avq_cache.hpp"
#include "avq_launch.hpp"

#include <algorithm>
#include <type_traits>

namespace avq {

namespace {

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

struct PromptArgs {
  const void *Q, *K, *V;
  int64_t q_stride, k_stride, v_stride;  // elements between tokens
  const int32_t *cu_q, *cu_k;            // [S + 1]
  void* Y;
  float* lse;  // nullable
  int S, Tq, Tk, Hq, G, causal;
  int tiles;  // query tiles per head, at most
  float scale_log2;
  float lazy;  // kLazy / scale_log2
  // equal runs: see part_floats and Runs
  float* parts;
  int32_t* joins;  // [tiles][Hq][2]: first part, number of parts; before it, one
                   // entry that says whether joins is filled
};

template <typename T, int D>
struct PromptCfg {
  static constexpr bool kB = Elem<T>::kBf16;
  static constexpr int NW = 4;            // waves
  static constexpr int BM = 32 * NW;      // queries per workgroup
  // Keys per tile: 64, but 32 for bf16 at d = 128, where three workgroups then
  // fit a CU (168 registers, 32 KB of LDS) instead of two (18 packed prompts
  // 156 to 149 us, 16384 tokens 1026 to 1011; d = 64: 27.4 us with 64, 28.7 with
  // 32 for 8 x 784 patches), and for fp32 (LDS)
  static constexpr int BN = kB && D == 64 ? 64 : 32;
  // key tiles of a run where there are few: ceil(units / kLeast) runs, so that
  // each has at least half as many
  static constexpr int kLeast = (kB ? 256 : 128) / BN;
  static constexpr int kPerCu = kB && D == 128 ? 3 : 2;  // waves per SIMD, at least
  static constexpr int KT = BN / 32;
  static constexpr int DT = D / 32;
  static constexpr int ESZ = sizeof(T);
  static constexpr int U = D * ESZ / 16;       // 16-byte units per row
  static constexpr int TILE = BN * D * ESZ;    // bytes of a tile
  static constexpr int COPIES = TILE / 1024;   // wave copies per tile
  static constexpr int CPW = COPIES / NW;
  static constexpr int RPC = 64 / U;           // rows per wave copy
  static_assert(COPIES % NW == 0, "copies split evenly over the waves");
};

// ---- division of the work --------------------------------------------------------
// Whole tiles (one workgroup each) where there are enough of them; otherwise
// equal runs: the key tiles of all query tiles, in the order head, sequence,
// query tile, key tile, are cut into as many equal runs as workgroups run at
// once. A run covers parts of one or more query tiles: a whole one is stored, a
// part leaves its numerators, maxima and sums, and a second launch joins the
// parts. At most a run's first and last tile are parts.

// A part: numerators, maxima [BM], sums [BM]; run i has parts 2 i and 2 i + 1.
// The numerators lie as the lanes hold them, so that every store and load of a
// wave covers 1 KB: piece q = 4 i + j of wave w, [w][q][64 lanes][4], are the
// columns 32 i + 8 j + 4 (lane / 32) + 0 .. 3 of row 32 w + lane % 32.
__host__ __device__ constexpr size_t part_floats(int BM, int D) { return (size_t)BM * (D + 2); }

struct Tile {
  int s, lt;           // sequence, tile of its queries
  int qa, ka, Lq, Lk;  // its rows
  __device__ __forceinline__ void rows_of(const PromptArgs& a) {
    int b;
    packed_range(a.cu_q, s, a.Tq, qa, b);
    Lq = b - qa;
    packed_range(a.cu_k, s, a.Tk, ka, b);
    Lk = b - ka;
  }
};

// Key tiles that query tile lt reads.
template <int BM, int BN>
__device__ __forceinline__ int key_tiles(int lt, int Lq, int Lk, int causal) {
  const int keys = causal ? max(0, min(Lk, min((lt + 1) * BM, Lq) + Lk - Lq)) : Lk;
  return (keys + BN - 1) / BN;
}

// Whole tiles: tile of work item i, false if there is none. Up to one sequence
// per lane: by levels, the last tiles of the longest sequences first (under
// the causal mask a tile's work grows with its index, and a long tile that
// starts last runs alone): N(L) = sum over the sequences of max(0, tiles - L)
// tiles have level L or more, and the items of level L are those from N(L + 1)
// to N(L). More sequences: from the last tile back, found in the closed form
// cu / BM + s.
template <int BM>
__device__ __forceinline__ bool find_tile(const PromptArgs& a, int i, int lane, Tile& t) {
  if (a.S <= kWave) {
    Tile mine{lane, 0, 0, 0, 0, 0};  // the lane's sequence
    if (lane < a.S) mine.rows_of(a);
    const int nt = (mine.Lq + BM - 1) / BM;
    auto from = [&](int L) { return last_lane(wave_incl_scan(max(nt - L, 0))); };
    if (i >= from(0)) return false;
    int lo = 0, hi = a.tiles;  // N(lo) > i >= N(hi)
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (from(mid) > i) lo = mid; else hi = mid;
    }
    // the level's sequences in order: the one with i - N(lo + 1) before it
    const int rank = i - from(lo + 1);
    const unsigned long long in = __ballot(nt > lo);
    const unsigned long long at = __ballot(nt > lo && bits_below(in) == rank);
    t.s = (int)__builtin_ctzll(at);
    t.lt = lo;
    t.qa = __builtin_amdgcn_readlane(mine.qa, t.s);
    t.ka = __builtin_amdgcn_readlane(mine.ka, t.s);
    t.Lq = __builtin_amdgcn_readlane(mine.Lq, t.s);
    t.Lk = __builtin_amdgcn_readlane(mine.Lk, t.s);
    return true;
  }
  const int tile = a.tiles - 1 - i;
  t.s = find_sequence(a.S, tile, lane, [&](int k) {
    return (long long)min(max(a.cu_q[k], 0), a.Tq) / BM + k;
  });
  t.rows_of(a);
  t.lt = tile - (t.qa / BM + t.s);
  return t.lt >= 0 && (long long)t.lt * BM < t.Lq;
}

// Equal runs. A unit is a key tile of a query tile; a query tile that reads
// none has one unit too, so that its rows are stored.
template <int BM, int BN>
struct Runs {
  // Units of the tiles 0 .. n - 1 of a sequence: tile L reads the keys up to
  // BM (L + 1) + off (causal), so Q (L + 1) + o key tiles, but the last tile,
  // and every one without a mask, all.
  static __device__ __forceinline__ int before(int n, int Lq, int Lk, int causal) {
    constexpr int Q = BM / BN;
    const int nt = (Lq + BM - 1) / BM, all = max(1, (Lk + BN - 1) / BN);
    if (!causal) return n * all;
    const int off = Lk - Lq, o = off >= 0 ? (off + BN - 1) / BN : -(-off / BN);  // ceil(off / BN)
    const int m = min(n, nt - 1);
    // tiles below one have no key: Q (L + 1) + o < 1
    const int one = min(m, o >= 1 - Q ? 0 : (Q - o) / Q - 1);
    const int sum = one + Q * ((m * (m + 1) - one * (one + 1)) / 2) + o * (m - one);
    return n < nt || nt == 0 ? sum : sum + all;
  }
  static __device__ __forceinline__ int total(int Lq, int Lk, int causal) {
    return Lq > 0 ? before((Lq + BM - 1) / BM, Lq, Lk, causal) : 0;
  }
};

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

// The key tiles t_begin .. t_end - 1 of one query tile and head; part: where a
// part goes, null for a whole tile.
template <typename T, int D>
__device__ __forceinline__ void attend(const PromptArgs& a, const Tile& tile, int hq, int t_begin,
                                       int t_end, float* part, unsigned char* lds, int wave,
                                       int lane) {
  using Cfg = PromptCfg<T, D>;
  constexpr bool kB = Cfg::kB;
  constexpr int BM = Cfg::BM, BN = Cfg::BN, KT = Cfg::KT, DT = Cfg::DT, U = Cfg::U,
                ESZ = Cfg::ESZ, CPW = Cfg::CPW, RPC = Cfg::RPC, TILE = Cfg::TILE;
  constexpr int KQ = kB ? D / 16 : D / 2;
  using Frag = typename std::conditional<kB, bf16x8, float>::type;
  const int h = lane / 32, c = lane % 32;
  const int qa = tile.qa, ka = tile.ka, Lq = tile.Lq, Lk = tile.Lk, lt = tile.lt;
  const int hkv = hq / a.G;
  const int off = Lk - Lq;  // key of query 0 on the diagonal
  const int row0 = lt * BM + 32 * wave;
  const int row = row0 + c;
  const bool has_row = row < Lq;
  // keys that the row, some row of the wave, and all its rows see
  const int see = a.causal ? min(Lk, row + off + 1) : Lk;
  const int wave_see = row0 >= Lq ? 0 : a.causal ? min(Lk, min(row0 + 31, Lq - 1) + off + 1) : Lk;
  const int wave_all = a.causal ? min(Lk, row0 + off + 1) : Lk;
  const int n_tiles = t_end;

  // ---- query operand ---------------------------------------------------------
  Frag q[KQ];
  {
    const T* qp = static_cast<const T*>(a.Q) + (size_t)(qa + min(row, Lq - 1)) * a.q_stride +
                  (size_t)hq * D;
#pragma unroll
    for (int k = 0; k < KQ; ++k) {
      if constexpr (kB) {
        q[k] = *reinterpret_cast<const bf16x8*>(qp + 16 * k + 8 * h);
      } else if (k % 4 == 0) {  // step 4 i + e: column 8 i + 4 h + e
        const f32x4 v = *reinterpret_cast<const f32x4*>(qp + 2 * k + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) q[k + e] = v[e];
      }
    }
  }

  // ---- tiles to LDS ------------------------------------------------------------
  const T* kbase = static_cast<const T*>(a.K) + (size_t)ka * a.k_stride + (size_t)hkv * D;
  const T* vbase = static_cast<const T*>(a.V) + (size_t)ka * a.v_stride + (size_t)hkv * D;
  const int lrow = lane / U, lunit = lane % U;
  auto issue = [&](int t, int b) {
    const __amdgpu_buffer_rsrc_t rk = rsrc(kbase + (size_t)t * BN * a.k_stride);
    const __amdgpu_buffer_rsrc_t rv = rsrc(vbase + (size_t)t * BN * a.v_stride);
    const int last = Lk - 1 - t * BN;  // rows past the sequence read its last one
#pragma unroll
    for (int i = 0; i < CPW; ++i) {
      const int j = wave * CPW + i;
      const int r = RPC * j + lrow, rr = min(r, last);
      const uint32_t ko = (uint32_t)rr * (uint32_t)(a.k_stride * ESZ) +
                          16u * (lunit ^ key_swizzle<U>(r));
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rk, (__attribute__((address_space(3))) void*)(lds + b * TILE + 1024 * j), 16, ko, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < CPW; ++i) {
      const int j = wave * CPW + i;
      const int r = RPC * j + lrow, rr = min(r, last);
      const uint32_t vo = (uint32_t)rr * (uint32_t)(a.v_stride * ESZ) +
                          16u * (lunit ^ value_swizzle<U, kB>(r));
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rv, (__attribute__((address_space(3))) void*)(lds + (2 + b) * TILE + 1024 * j), 16, vo, 0,
          0, 0);
    }
  };

  // m: the running max of s. The weights exp2((s - m) scale) are one fma with
  // ms = m scale and exp2. It leaves the rounding error of ms, up to |ms| / 2^24,
  // in the exponent: one factor for all weights of a row while that is at most
  // 1, but beyond float's range for the largest s. Once a row has such a max
  // its wave subtracts m first, in the branch of the new max (which is then
  // taken for every tile), and ms is 0: the usual path has no more work.
  float m = kMaxFloor, ms = kMaxFloor, limit = kMaxFloor, l = 0.f;
  bool fused = true;
  f32x16 o[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) o[i] = f32x16{};

  if (t_begin < n_tiles) issue(t_begin, t_begin & 1);
  for (int t = t_begin; t < n_tiles; ++t) {
    const int b = t & 1;
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();  // tile t has landed, tile t - 1 is read
    if (t + 1 < n_tiles) issue(t + 1, b ^ 1);
    const int k0 = t * BN;
    if (k0 >= wave_see) continue;
    const unsigned char* kt = lds + b * TILE;
    const unsigned char* vt = lds + (2 + b) * TILE;

    // ---- S^T -------------------------------------------------------------------
    f32x16 sc[KT];
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      sc[i] = f32x16{};
      const int r = 32 * i + c;
      const unsigned char* rowp = kt + r * (D * ESZ);
#pragma unroll
      for (int k = 0; k < U / 2; ++k) {
        const unsigned char* p = rowp + 16 * ((2 * k + h) ^ key_swizzle<U>(r));
        if constexpr (kB) {
          sc[i] = mfma32(*reinterpret_cast<const bf16x8*>(p), q[k], sc[i]);
        } else {
          const f32x4 v = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[i] = mfma32(v[e], q[4 * k + e], sc[i]);
        }
      }
    }
    if (k0 + BN > wave_all) {
#pragma unroll
      for (int i = 0; i < KT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (k0 + 32 * i + 8 * (r / 4) + 4 * h + r % 4 >= see) sc[i][r] = -INFINITY;
    }

    // ---- running max, weights -----------------------------------------------------
    float mx = sc[0][0];
#pragma unroll
    for (int i = 0; i < KT; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[i][r]);
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
      limit = fused ? mn + a.lazy : -INFINITY;
      if (!fused) {
#pragma unroll
        for (int i = 0; i < KT; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) sc[i][r] -= m;
      }
      l *= f;
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] *= f;
    }
#pragma unroll
    for (int i = 0; i < KT; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        sc[i][r] = exp2_hw(fmaf(sc[i][r], a.scale_log2, -ms));
        l += sc[i][r];
      }

    // ---- Y^T += V^T P^T ---------------------------------------------------------------
    // bf16: the matrix product takes the weights rounded to bf16 (by at most half
    // a step, 2^-8; their sum l is of the unrounded ones). The errors of a row's
    // weights are independent and leave about as much as rounding Y does: for
    // 16384 tokens 0.0022 of Y's norm with both, 0.0017 with Y's alone.
    if constexpr (kB) {
#pragma unroll
      for (int k = 0; k < BN / 16; ++k) {  // 16 keys: 4 h + 0..3 and 8 + 4 h + 0..3 per lane
        bf16x8 p;
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = (bf16)sc[k / 2][8 * (k % 2) + e];
        const int key = 16 * k + 4 * h + lane % 16 / 4;
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          const int unit = 4 * i + lane / 16 % 2 * 2 + lane % 4 / 2;
          bf16x8 v;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int r = key + 8 * e;
            const bf16x4 part = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
                (__attribute__((address_space(3))) bf16x4*)(
                    vt + r * (D * ESZ) + 16 * (unit ^ value_swizzle<U, kB>(r)) + 8 * (lane % 2)));
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * e + j] = part[j];
          }
          o[i] = mfma32(v, p, o[i]);
        }
      }
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int key = 8 * (r / 4) + 4 * h + r % 4;
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          const float v = *reinterpret_cast<const float*>(
              vt + key * (D * ESZ) + 16 * ((8 * i + c / 4) ^ value_swizzle<U, kB>(key)) +
              4 * (c % 4));
          o[i] = mfma32(v, sc[0][r], o[i]);
        }
      }
    }
  }

  l = add_xor<32>(l);
  if (!fused) ms = m * a.scale_log2;
  if (part) {
    const int r0 = 32 * wave + c;
    if (h == 0) {
      part[BM * D + r0] = ms;
      part[BM * D + BM + r0] = l;
    }
    if (has_row) {
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          *reinterpret_cast<f32x4*>(part + ((wave * (D / 8) + 4 * i + r / 4) * kWave + lane) * 4) =
              f32x4{o[i][r], o[i][r + 1], o[i][r + 2], o[i][r + 3]};
    }
    return;
  }
  // ---- Y = O / l -----------------------------------------------------------------------
  const float inv = l > 0.f ? 1.f / l : 0.f;
  if (!has_row) return;
  const size_t at = (size_t)(qa + row) * a.Hq + hq;
  T* y = static_cast<T*>(a.Y) + at * D;
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const int d0 = 32 * i + 2 * r + 4 * h;
      if constexpr (kB)
        *reinterpret_cast<bf16x4*>(y + d0) = bf16x4{(bf16)(o[i][r] * inv), (bf16)(o[i][r + 1] * inv),
                                                    (bf16)(o[i][r + 2] * inv),
                                                    (bf16)(o[i][r + 3] * inv)};
      else
        *reinterpret_cast<f32x4*>(y + d0) =
            f32x4{o[i][r] * inv, o[i][r + 1] * inv, o[i][r + 2] * inv, o[i][r + 3] * inv};
    }
  if (a.lse && h == 0) a.lse[at] = l > 0.f ? (ms + log2_hw(l)) * kLn2 : -INFINITY;
}

template <typename T, int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(PromptCfg<T, D>::kPerCu)))
void prompt_kernel(PromptArgs a) {
  using Cfg = PromptCfg<T, D>;
  __shared__ __attribute__((aligned(16))) unsigned char lds[4 * Cfg::TILE];  // K0 K1 V0 V1
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  int hq = blockIdx.x % a.Hq;
  // workgroup i runs on XCD i % 8: each XCD takes consecutive heads, which
  // share keys, of every tile
  if (a.Hq % 8 == 0) hq = hq % 8 * (a.Hq / 8) + hq / 8;
  Tile t;
  if (!find_tile<Cfg::BM>(a, blockIdx.x / a.Hq, lane, t)) return;
  attend<T, D>(a, t, hq, 0, key_tiles<Cfg::BM, Cfg::BN>(t.lt, t.Lq, t.Lk, a.causal), nullptr, lds,
               wave, lane);
}

template <typename T, int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(PromptCfg<T, D>::kPerCu)))
void prompt_runs_kernel(PromptArgs a) {
  using Cfg = PromptCfg<T, D>;
  constexpr int BM = Cfg::BM, BN = Cfg::BN;
  using R = Runs<BM, BN>;
  __shared__ __attribute__((aligned(16))) unsigned char lds[4 * Cfg::TILE];  // K0 K1 V0 V1
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);

  // units of the lane's sequences (consecutive ones) and of those before them
  const int per = (a.S + kWave - 1) / kWave;
  Tile t;
  int mine = 0;
  bool fine = true;
  for (int i = 0; i < per; ++i) {
    t.s = lane * per + i;
    if (t.s >= a.S) break;
    t.rows_of(a);
    mine += R::total(t.Lq, t.Lk, a.causal);
    fine = fine && a.cu_q[t.s] <= a.cu_q[t.s + 1];
  }
  // sequences that overlap would have more tiles than joins has room for
  fine = __all(fine);
  if (blockIdx.x == 0 && threadIdx.x == 0) a.joins[-1] = fine;
  if (!fine) return;
  const int incl = wave_incl_scan(mine);
  const int per_head = last_lane(incl);
  const long long U = (long long)per_head * a.Hq;
  // runs of about kLeast units where there are few (at least half as many);
  // consecutive runs on one XCD (workgroup i runs on XCD i % 8), so that it takes
  // consecutive heads, which share keys, and every XCD has its share of the runs
  // there are
  const int W = (int)min((long long)gridDim.x, (U + Cfg::kLeast - 1) / Cfg::kLeast);
  if ((int)blockIdx.x >= W) return;
  const int xcd = blockIdx.x % 8;
  const int w = xcd * (W / 8) + min(xcd, W % 8) + blockIdx.x / 8;
  long long u = U * w / W;
  const long long u_first = u, u_end = U * (w + 1) / W;

  // head, sequence and tile of the run's first unit
  int hq = __builtin_amdgcn_readfirstlane((int)(u / per_head));
  int x = __builtin_amdgcn_readfirstlane((int)(u % per_head));  // units before it in the head
  const int owner = __popcll(__ballot(incl <= x));  // the first lane with more units up to it
  x -= __builtin_amdgcn_readlane(incl - mine, owner);
  t.s = owner * per;
  t.rows_of(a);
  for (int n = R::total(t.Lq, t.Lk, a.causal); x >= n && t.s + 1 < a.S;
       n = R::total(t.Lq, t.Lk, a.causal)) {
    x -= n;
    ++t.s;
    t.rows_of(a);
  }
  int lo = 0, hi = (t.Lq + BM - 1) / BM;  // before(lo) <= x < before(hi)
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (R::before(mid, t.Lq, t.Lk, a.causal) <= x) lo = mid; else hi = mid;
  }
  t.lt = lo;
  x -= R::before(lo, t.Lq, t.Lk, a.causal);

  while (true) {
    const int tiles = key_tiles<BM, BN>(t.lt, t.Lq, t.Lk, a.causal), units = max(1, tiles);
    const int x_end = (int)min((long long)units, x + (u_end - u));
    const int slot = u == u_first ? 0 : 1;
    const bool whole = x == 0 && x_end == units;
    if (x == 0 && threadIdx.x == 0) {
      // the run that holds unit v is ((v + 1) W - 1) / U
      const long long w_last = ((u + units) * W - 1) / U;
      int32_t* join = a.joins + 2 * ((size_t)(t.qa / BM + t.s + t.lt) * a.Hq + hq);
      join[0] = 2 * w + slot;
      join[1] = whole ? 1 : (int)(w_last - w) + 1;
    }
    attend<T, D>(a, t, hq, x, min(x_end, tiles),
                 whole ? nullptr : a.parts + (size_t)(2 * w + slot) * part_floats(BM, D), lds, wave,
                 lane);
    u += x_end - x;
    if (u >= u_end) break;
    __syncthreads();  // the tiles in LDS are read
    x = 0;
    if ((++t.lt) * BM >= t.Lq) {  // the next sequence that has queries
      t.lt = 0;
      do {
        if (++t.s == a.S) {
          t.s = 0;
          ++hq;
        }
        t.rows_of(a);
      } while (t.Lq == 0);
    }
  }
}

// Joins the parts of a tile's rows (one piece of 4 columns per thread): the
// first part is the one that joins names, the others are the first ones of the
// runs that follow.
template <typename T, int D>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptArgs a) {
  constexpr int BM = PromptCfg<T, D>::BM;
  const int tile = blockIdx.x / a.Hq, hq = blockIdx.x % a.Hq;
  Tile t;  // tile qa / BM + s + lt; ids that belong to none have no entry in joins
  t.s = find_sequence(a.S, tile, threadIdx.x % kWave, [&](int k) {
    return (long long)min(max(a.cu_q[k], 0), a.Tq) / BM + k;
  });
  t.rows_of(a);
  t.lt = tile - (t.qa / BM + t.s);
  if (t.lt < 0 || (long long)t.lt * BM >= t.Lq) return;
  if (a.joins[-1] == 0) return;
  const int first = a.joins[2 * (size_t)blockIdx.x], n = a.joins[2 * (size_t)blockIdx.x + 1];
  if (n == 1) return;
  const int piece = blockIdx.y * 256 + threadIdx.x, q = piece / kWave % (D / 8);
  const int r = 32 * (piece / kWave / (D / 8)) + piece % 32;
  const int d0 = 8 * q + 4 * (piece % kWave / 32);
  const int row = t.lt * BM + r;
  if (row >= t.Lq) return;
  auto part = [&](int i) {
    return a.parts + (size_t)(i == 0 ? first : 2 * (first / 2 + i)) * part_floats(BM, D);
  };
  float m = kMaxFloor, l = 0.f;
#pragma unroll 8
  for (int i = 0; i < n; ++i) m = fmaxf(m, part(i)[BM * D + r]);
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int i = 0; i < n; ++i) {
    const float* p = part(i);
    const float f = exp2_hw(p[BM * D + r] - m);
    l = fmaf(f, p[BM * D + BM + r], l);
    acc += f * *reinterpret_cast<const f32x4*>(p + 4 * piece);
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  const size_t at = (size_t)(t.qa + row) * a.Hq + hq;
  T* y = static_cast<T*>(a.Y) + at * D + d0;
  if constexpr (Elem<T>::kBf16)
    *reinterpret_cast<bf16x4*>(y) = bf16x4{(bf16)(acc[0] * inv), (bf16)(acc[1] * inv),
                                           (bf16)(acc[2] * inv), (bf16)(acc[3] * inv)};
  else
    *reinterpret_cast<f32x4*>(y) = acc * inv;
  if (a.lse && d0 == 0) a.lse[at] = l > 0.f ? (m + log2_hw(l)) * kLn2 : -INFINITY;
}

long long tiles_of(long long Tq, int S, int BM) { return Tq / BM + S; }

// Equal runs (workgroups), or 0 for whole tiles. With whole tiles the longest
// tile's chain of keys bounds the time; with runs it is the mean work, and the
// parts, which are written and joined. So runs are taken where the chain exceeds
// the mean by enough keys, the sequences' mean lengths standing for all.
// * More tiles than CUs share these, so the chain is slower: the mean is tiles /
//   1024 of it under the causal mask (tiles / 512 without one), the parts cost 15
//   to 20 us. Measured, us whole / runs (d = 128): one sequence of 8192 tokens and
//   8 heads 188 / 170, 4096 and 16 98 / 100, 6144 and 16 173 / 190, 2048 and 32
//   53 / 68; fp32, d = 64, 2048 and 8 146 / 52, 256 and 16 22 / 19, and without a
//   mask 1024 and 32 79 / 86.
// * bf16 tiles with a CU each (0.6 us per 32 keys of a chain, 0.5 per unit of a
//   CU): a run has about 256 keys at least, and a second launch and the parts cost
//   by their rows: as much as 500 keys up to 16384 rows, 900 up to 32768, 1250 for
//   all 768 runs. Measured, us whole / runs (d = 128): 32 queries behind 992 keys,
//   4, 16, 32 heads 23 / 15, 22 / 15, 22 / 15; behind 480 13 / 13 each; 128 behind
//   896 25 / 16, 25 / 18, 25 / 20; 128 behind 1920 43 / 16, 44 / 19, 44 / 25; a
//   prompt of 2048, 4 and 16 heads 44 / 29, 45 / 45, of 1024 25 / 21, 25 / 31;
//   chunks of 512 and 300 behind 15872 and 4001, 16 heads 300 / 116.
// fp32's products alone nearly fill the matrix units: one run per CU and half the
// parts, but two where a run is then still 16 key tiles long (by the mean
// lengths). Measured, us one / two: 1024 tokens and 16 heads 60 / 65, 2048 and 8
// 95 / 96, 4096 and 16 587 / 560 (d = 64: 318 / 295), 56 queries of three
// sequences behind 10848 keys, 42 heads 174 / 120.
template <typename T, int D>
int runs_of(int S, int Tq, int Tk, int Hq, int causal) {
  using Cfg = PromptCfg<T, D>;
  const long long tiles = tiles_of(Tq, S, Cfg::BM) * Hq, full = causal ? 1024 : 512;
  const long long excess = (full - tiles) * (Tk / S) / full;
  if (Cfg::kB) {
    constexpr int kRuns = 768;
    const long long Lq = std::max(1, Tq / S), Lk = Tk / S;  // mean lengths
    const long long own = (Lq + Cfg::BM - 1) / Cfg::BM * S * Hq;
    if (own > 256) return excess < 2500 ? 0 : kRuns;
    const long long keys = own * (Lk - (causal ? std::min(Lq, Lk) / 2 : 0));
    const long long mean = std::max(256LL, keys * 5 / 6 / 256);
    const long long rows = std::min(keys / 256, (long long)kRuns) * std::min<long long>(Lq, Cfg::BM);
    if (Lk - mean < (rows <= 16384 ? 500 : rows <= 32768 ? 900 : 1250)) return 0;
    // room for twice the runs that the mean lengths give (ragged tiles): 64 runs'
    // parts are 8 MB, those of 768 100 MB
    return (int)std::min<long long>(kRuns, (keys / 128 + 63) / 64 * 64);
  }
  if (excess < (causal ? 200 : 600)) return 0;
  const long long units = tiles * (Tk - (causal ? Tq / 2 : 0)) / S / Cfg::BN;
  return units < 512 * 16 ? 256 : 512;
}

}  // namespace

template <typename T, int D>
size_t prompt_attention_workspace(int S, int Tq, int Tk, int Hq, int causal) {
  using Cfg = PromptCfg<T, D>;
  const int runs = runs_of<T, D>(S, Tq, Tk, Hq, causal);
  if (runs == 0) return 0;
  return 2 * (size_t)runs * part_floats(Cfg::BM, D) * sizeof(float) +
         ((size_t)tiles_of(Tq, S, Cfg::BM) * Hq * 2 + 4) * sizeof(int32_t);
}

template <typename T, int D>
hipError_t launch_prompt_attention(int S, int Tq, int Tk, int Hq, int Hkv, float scale, int causal,
                                   const void* Q, int64_t q_stride, const void* K,
                                   int64_t k_stride, const void* V, int64_t v_stride,
                                   const int32_t* cu_q, const int32_t* cu_k, void* Y, float* lse,
                                   void* workspace, hipStream_t stream) {
  using Cfg = PromptCfg<T, D>;
  const long long tiles = tiles_of(Tq, S, Cfg::BM);
  const int runs = runs_of<T, D>(S, Tq, Tk, Hq, causal);
  float* parts = static_cast<float*>(workspace);
  PromptArgs a{Q, K, V, q_stride, k_stride, v_stride, cu_q, cu_k, Y, lse,
               S, Tq, Tk, Hq, Hq / Hkv, causal, (int)tiles, scale * kLog2e,
               kLazy / (scale * kLog2e), parts,
               reinterpret_cast<int32_t*>(parts + 2 * (size_t)runs * part_floats(Cfg::BM, D)) + 4};
  const unsigned grid = (unsigned)(tiles * Hq), threads = 64 * Cfg::NW;
  if (runs == 0) {
    hipLaunchKernelGGL((prompt_kernel<T, D>), dim3(grid), dim3(threads), 0, stream, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((prompt_runs_kernel<T, D>), dim3(runs), dim3(threads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((prompt_join_kernel<T, D>), dim3(grid, Cfg::BM * D / 4 / 256), dim3(256), 0,
                     stream, a);
  return hipGetLastError();
}

#define AVQ_INSTANCE(T, D)                                                                        \
  template hipError_t launch_prompt_attention<T, D>(                                              \
      int, int, int, int, int, float, int, const void*, int64_t, const void*, int64_t, const void*, \
      int64_t, const int32_t*, const int32_t*, void*, float*, void*, hipStream_t);                \
  template size_t prompt_attention_workspace<T, D>(int, int, int, int, int);
AVQ_INSTANCE(bf16, 64)
AVQ_INSTANCE(bf16, 128)
AVQ_INSTANCE(float, 64)
AVQ_INSTANCE(float, 128)
#undef AVQ_INSTANCE

}  // namespace avq
