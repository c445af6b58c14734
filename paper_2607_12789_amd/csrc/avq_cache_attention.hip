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
#include "avq_cache_attention.hpp"
#include "avq_launch.hpp"

#include <algorithm>

namespace avq {

namespace {

template <typename T, int D, bool FP4, int NT>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(kPerCu<T, D, FP4, NT>)))
void cache_attention_kernel(CacheAttnArgs a) {
  __shared__ __attribute__((aligned(16))) Exchange<D> s_o;
  cache_attention_run<T, D, FP4, NT, false>(a, blockIdx.x, gridDim.x, s_o);
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
  CacheAttnArgs a{};
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
