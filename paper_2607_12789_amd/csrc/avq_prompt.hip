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
// Lengths are known on the device only, so the grid has Tq / 128 + S tiles per
// head, at least as many as the sequences need, and each workgroup finds its
// sequence; those left over exit. Where the tiles are too few to fill the
// device (a chunk behind a long prefix), several workgroups share a tile's
// keys and a second launch joins their sums.
#include "avq_cache.hpp"
#include "avq_launch.hpp"

#include <algorithm>
#include <type_traits>

namespace avq {

namespace {

constexpr int kMaxSplits = 16;

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
  int tiles;   // query tiles per head, at most
  int splits;  // workgroups that share a tile's keys
  float scale_log2;
  float* parts;  // with splits: see part_floats
};

// What one of a tile's workgroups leaves when its keys are shared: numerators
// [BM][D], maxima [BM], sums [BM]; tile t of head h has parts (t Hq + h) splits
// + z.
__host__ __device__ constexpr size_t part_floats(int BM, int D) { return (size_t)BM * (D + 2); }

// Sequence and query tile of work item i. Up to one sequence per lane: by
// levels, the last tiles of the longest sequences first (under the causal mask
// a tile's work grows with its index, and a long tile that starts last runs
// alone): N(L) = sum over the sequences of max(0, tiles - L) tiles have level
// L or more, and the items of level L are those from N(L + 1) to N(L). More
// sequences: from the last tile back, found in the closed form cu / BM + s.
// Returns false if there is no such item.
__device__ __forceinline__ bool find_tile(const int32_t* cu, int S, int T, int BM, int tiles, int i,
                                          int lane, int& s, int& lt) {
  if (S <= kWave) {
    int nt = 0;
    if (lane < S) {
      int a, b;
      packed_range(cu, lane, T, a, b);
      nt = (b - a + BM - 1) / BM;
    }
    auto from = [&](int L) { return last_lane(wave_incl_scan(max(nt - L, 0))); };
    if (i >= from(0)) return false;
    int lo = 0, hi = tiles;  // N(lo) > i >= N(hi)
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (from(mid) > i) lo = mid; else hi = mid;
    }
    // the level's sequences in order: the one with i - N(lo + 1) before it
    const int rank = i - from(lo + 1);
    const unsigned long long in = __ballot(nt > lo);
    const unsigned long long at = __ballot(nt > lo && bits_below(in) == rank);
    s = (int)__builtin_ctzll(at);
    lt = lo;
    return true;
  }
  const int tile = tiles - 1 - i;
  s = find_sequence(S, tile, lane, [&](int k) {
    return (long long)min(max(cu[k], 0), T) / BM + k;
  });
  int a, b;
  packed_range(cu, s, T, a, b);
  lt = tile - (a / BM + s);
  return lt >= 0 && (long long)lt * BM < b - a;
}

template <typename T, int D>
struct PromptCfg {
  static constexpr bool kB = Elem<T>::kBf16;
  static constexpr int NW = 4;            // waves
  static constexpr int BM = 32 * NW;      // queries per workgroup
  static constexpr int BN = kB ? 64 : 32;  // keys per tile
  static constexpr int KT = BN / 32;
  static constexpr int DT = D / 32;
  static constexpr int ESZ = sizeof(T);
  static constexpr int U = D * ESZ / 16;       // 16-byte units per row
  static constexpr int TILE = BN * D * ESZ;    // bytes of a tile
  static constexpr int COPIES = TILE / 1024;   // wave copies per tile
  static constexpr int CPW = COPIES / NW;
  static constexpr int RPC = 64 / U;           // rows per wave copy
  static constexpr int LDS_BYTES = 4 * TILE;   // K and V, two buffers
  static_assert(COPIES % NW == 0, "copies split evenly over the waves");
};

// Positions of the 16-byte units of a staged row. Keys: 32 rows read one unit
// each, so consecutive rows permute their units. Values: the transpose read
// takes 32 bytes (a pair of units) of 4 consecutive keys per 16 lanes, so
// those keys permute their pairs, and keys 4 apart swap halves of the row.
template <int U>
__device__ __forceinline__ int key_swizzle(int r) {
  return U >= 16 ? r & 15 : (r >> 1) & 7;
}
template <int U, bool kB>
__device__ __forceinline__ int value_swizzle(int r) {
  if constexpr (!kB) return (r >> 2 & 1) << 3;
  return ((r & 3) << 1) | (U >= 16 ? (r >> 2 & 1) << 3 : 0);
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const void* p) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, 0x7fffffff, 0x00020000);
}

template <typename T, int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
void prompt_kernel(PromptArgs a) {
  using Cfg = PromptCfg<T, D>;
  constexpr bool kB = Cfg::kB;
  constexpr int BM = Cfg::BM, BN = Cfg::BN, KT = Cfg::KT, DT = Cfg::DT, U = Cfg::U,
                ESZ = Cfg::ESZ, CPW = Cfg::CPW, RPC = Cfg::RPC, TILE = Cfg::TILE;
  constexpr int KQ = kB ? D / 16 : D / 2;
  using Frag = typename std::conditional<kB, bf16x8, float>::type;
  constexpr float kLazy = 8.f, kMaxFloor = -1e30f, kLn2 = 0.6931471805599453f;

  __shared__ __attribute__((aligned(16))) unsigned char lds[Cfg::LDS_BYTES];  // K0 K1 V0 V1

  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int h = lane / 32, c = lane % 32;

  const int item = blockIdx.x / a.Hq;
  int hq = blockIdx.x % a.Hq;
  // workgroup i runs on XCD i % 8: each XCD takes consecutive heads, which
  // share keys, of every tile
  if (a.Hq % 8 == 0) hq = hq % 8 * (a.Hq / 8) + hq / 8;
  const int hkv = hq / a.G;

  int s, lt;
  if (!find_tile(a.cu_q, a.S, a.Tq, BM, a.tiles, item, lane, s, lt)) return;
  int qa, qb, ka, kb;
  packed_range(a.cu_q, s, a.Tq, qa, qb);
  packed_range(a.cu_k, s, a.Tk, ka, kb);
  const int Lq = qb - qa, Lk = kb - ka;
  const int off = Lk - Lq;  // key of query 0 on the diagonal
  const int row0 = lt * BM + 32 * wave;
  const int row = row0 + c;
  const bool has_row = row < Lq;
  // keys that the row, the wave's last row and the workgroup's last row see
  const int see = a.causal ? min(Lk, row + off + 1) : Lk;
  const int wave_see = row0 >= Lq ? 0 : a.causal ? min(Lk, min(row0 + 31, Lq - 1) + off + 1) : Lk;
  const int wave_all = a.causal ? min(Lk, row0 + off + 1) : Lk;  // seen by all its rows
  const int tile_see = a.causal ? min(Lk, min(lt * BM + BM, Lq) + off) : Lk;
  const int all_tiles = tile_see > 0 ? (tile_see + BN - 1) / BN : 0;
  // key tiles of this workgroup's share
  const int t_begin = (int)((long long)all_tiles * blockIdx.y / a.splits);
  const int n_tiles = (int)((long long)all_tiles * (blockIdx.y + 1) / a.splits);

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

  float m = kMaxFloor, l = 0.f;
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
    mx *= a.scale_log2;
    if (__any(mx > m + kLazy)) {
      const float mn = fmaxf(m, max_xor<32>(mx));
      const float f = exp2_hw(m - mn);
      m = mn;
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
        sc[i][r] = exp2_hw(fmaf(sc[i][r], a.scale_log2, -m));
        l += sc[i][r];
      }

    // ---- Y^T += V^T P^T ---------------------------------------------------------------
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
  if (a.splits > 1) {  // a part: nothing but the sum 0 for a row that saw no key
    float* part = a.parts + (((size_t)item * a.Hq + hq) * a.splits + blockIdx.y) * part_floats(BM, D);
    const int r0 = 32 * wave + c;
    if (h == 0) {
      part[BM * D + r0] = m;
      part[BM * D + BM + r0] = l;
    }
    if (has_row && l > 0.f) {
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          *reinterpret_cast<f32x4*>(part + r0 * D + 32 * i + 2 * r + 4 * h) =
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
  if (a.lse && h == 0) a.lse[at] = l > 0.f ? (m + log2_hw(l)) * kLn2 : -INFINITY;
}

// Joins the parts of a tile's rows: D / 4 threads per row, 4 columns each.
template <typename T, int D>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptArgs a) {
  constexpr int BM = PromptCfg<T, D>::BM;
  constexpr int TPR = D / 4, RPW = 256 / TPR;  // threads per row, rows per workgroup
  constexpr float kLn2 = 0.6931471805599453f;
  const int item = blockIdx.x / a.Hq, hq = blockIdx.x % a.Hq;
  int s, lt, qa, qb;
  if (!find_tile(a.cu_q, a.S, a.Tq, BM, a.tiles, item, threadIdx.x % kWave, s, lt)) return;
  packed_range(a.cu_q, s, a.Tq, qa, qb);
  const int r = blockIdx.y * RPW + threadIdx.x / TPR, d0 = threadIdx.x % TPR * 4;
  const int row = lt * BM + r;
  if (row >= qb - qa) return;
  const size_t step = part_floats(BM, D);
  const float* part = a.parts + ((size_t)item * a.Hq + hq) * a.splits * step;
  float m = -1e30f, ms[kMaxSplits], ls[kMaxSplits];
#pragma unroll
  for (int z = 0; z < kMaxSplits; ++z) {
    ls[z] = 0.f;
    if (z < a.splits) {
      ms[z] = part[z * step + BM * D + r];
      ls[z] = part[z * step + BM * D + BM + r];
    }
  }
#pragma unroll
  for (int z = 0; z < kMaxSplits; ++z)
    if (ls[z] > 0.f) m = fmaxf(m, ms[z]);
  float l = 0.f;
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int z = 0; z < kMaxSplits; ++z)
    if (ls[z] > 0.f) {
      const float f = exp2_hw(ms[z] - m);
      l = fmaf(f, ls[z], l);
      acc += f * *reinterpret_cast<const f32x4*>(part + z * step + r * D + d0);
    }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  const size_t at = (size_t)(qa + row) * a.Hq + hq;
  T* y = static_cast<T*>(a.Y) + at * D + d0;
  if constexpr (Elem<T>::kBf16)
    *reinterpret_cast<bf16x4*>(y) = bf16x4{(bf16)(acc[0] * inv), (bf16)(acc[1] * inv),
                                           (bf16)(acc[2] * inv), (bf16)(acc[3] * inv)};
  else
    *reinterpret_cast<f32x4*>(y) = acc * inv;
  if (a.lse && d0 == 0) a.lse[at] = l > 0.f ? (m + log2_hw(l)) * kLn2 : -INFINITY;
}

long long tiles_of(long long Tq, int S, int BM) { return Tq / BM + S; }

// Workgroups per tile: its keys are shared where the tiles leave more than
// half of the device's workgroup slots (two per CU) idle, and the sequences'
// mean length leaves each enough keys to pay for the joining launch.
template <typename T, int D>
int splits_of(int S, int Tq, int Tk, int Hq) {
  using Cfg = PromptCfg<T, D>;
  constexpr int kSlots = 512;
  const long long n = tiles_of(Tq, S, Cfg::BM) * Hq;
  const long long room = kSlots / n, keys = Tk / S / (4 * Cfg::BN);
  return (int)std::max(1LL, std::min({room, keys, (long long)kMaxSplits}));
}

}  // namespace

template <typename T, int D>
size_t prompt_attention_workspace(int S, int Tq, int Tk, int Hq) {
  using Cfg = PromptCfg<T, D>;
  const int splits = splits_of<T, D>(S, Tq, Tk, Hq);
  if (splits == 1) return 0;
  return (size_t)tiles_of(Tq, S, Cfg::BM) * Hq * splits * part_floats(Cfg::BM, D) * sizeof(float);
}

template <typename T, int D>
hipError_t launch_prompt_attention(int S, int Tq, int Tk, int Hq, int Hkv, float scale, int causal,
                                   const void* Q, int64_t q_stride, const void* K,
                                   int64_t k_stride, const void* V, int64_t v_stride,
                                   const int32_t* cu_q, const int32_t* cu_k, void* Y, float* lse,
                                   void* workspace, hipStream_t stream) {
  using Cfg = PromptCfg<T, D>;
  const long long tiles = tiles_of(Tq, S, Cfg::BM);
  const int splits = splits_of<T, D>(S, Tq, Tk, Hq);
  if (tiles * Hq > 0x7fffffff) return hipErrorInvalidConfiguration;
  PromptArgs a{Q, K, V, q_stride, k_stride, v_stride, cu_q, cu_k, Y, lse,
               S, Tq, Tk, Hq, Hq / Hkv, causal, (int)tiles, splits, scale * kLog2e,
               static_cast<float*>(workspace)};
  const unsigned grid = (unsigned)(tiles * Hq);
  hipLaunchKernelGGL((prompt_kernel<T, D>), dim3(grid, (unsigned)splits), dim3(64 * Cfg::NW), 0,
                     stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || splits == 1) return e;
  hipLaunchKernelGGL((prompt_join_kernel<T, D>), dim3(grid, Cfg::BM * D / 4 / 256), dim3(256), 0,
                     stream, a);
  return hipGetLastError();
}

#define AVQ_INSTANCE(T, D)                                                                        \
  template hipError_t launch_prompt_attention<T, D>(                                              \
      int, int, int, int, int, float, int, const void*, int64_t, const void*, int64_t, const void*, \
      int64_t, const int32_t*, const int32_t*, void*, float*, void*, hipStream_t);                \
  template size_t prompt_attention_workspace<T, D>(int, int, int, int);
AVQ_INSTANCE(bf16, 64)
AVQ_INSTANCE(bf16, 128)
AVQ_INSTANCE(float, 64)
AVQ_INSTANCE(float, 128)
#undef AVQ_INSTANCE

}  // namespace avq
