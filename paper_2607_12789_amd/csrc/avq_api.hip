// C ABI of the AVQ-Attention forward pass: argument validation on the host,
// then dispatch to the gfx950 kernels. Nothing here allocates device memory or
// synchronises; no exception crosses the boundary.
#include <float.h>
#include <stdarg.h>
#include <stdio.h>

#include <atomic>

#include "../../include/avq.h"
#include "avq_cache.hpp"
#include "avq_common.hpp"
#include "avq_packed.hpp"

#include "avq_launch.hpp"

namespace avq {

constexpr int kMaxDevices = 64;
constexpr int kMaxSlots = 256;

hipError_t device_info(DeviceInfo* out) {
  static DeviceInfo cache[kMaxDevices];
  static std::atomic<int> ready[kMaxDevices];
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return hipErrorInvalidDevice;
  if (ready[dev].load(std::memory_order_acquire) == 0) {
    DeviceInfo info;
    e = hipDeviceGetAttribute(&info.lds_max, hipDeviceAttributeMaxSharedMemoryPerBlock, dev);
    if (e != hipSuccess) return e;
    e = hipDeviceGetAttribute(&info.cus, hipDeviceAttributeMultiprocessorCount, dev);
    if (e != hipSuccess) return e;
    cache[dev] = info;
    ready[dev].store(1, std::memory_order_release);
  }
  *out = cache[dev];
  return hipSuccess;
}

hipError_t ensure_dynamic_lds(const void* kernel, int bytes, int slot) {
  // largest limit already set for (device, slot)
  static std::atomic<int> done[kMaxDevices][kMaxSlots];
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices || slot < 0 || slot >= kMaxSlots) return hipErrorInvalidValue;
  if (done[dev][slot].load(std::memory_order_acquire) >= bytes) return hipSuccess;
  e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != hipSuccess) return e;
  int prev = done[dev][slot].load(std::memory_order_relaxed);
  while (prev < bytes && !done[dev][slot].compare_exchange_weak(prev, bytes)) {
  }
  return hipSuccess;
}

}  // namespace avq

namespace {

thread_local char g_err[512] = "";

avq_status_t fail(avq_status_t st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return st;
}

avq_status_t ok() {
  g_err[0] = '\0';
  return AVQ_OK;
}

avq_status_t from_hip(hipError_t e, const char* what) {
  if (e == hipSuccess) return ok();
  return fail(AVQ_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

// Shared shape checks. Everything is validated before any HIP call.
avq_status_t check_common(avq_dtype_t dtype, int32_t B, int32_t H, int32_t N, int32_t d,
                          int32_t M0, int32_t Ch) {
  if (dtype != AVQ_F32 && dtype != AVQ_BF16)
    return fail(AVQ_ERR_INVALID_ARG, "unknown dtype %d", (int)dtype);
  if (B < 1 || H < 1 || N < 1 || d < 1 || M0 < 1 || Ch < 0)
    return fail(AVQ_ERR_INVALID_ARG,
                "sizes must be positive, Ch not negative (B=%d H=%d N=%d d=%d M0=%d Ch=%d)", B, H,
                N, d, M0, Ch);
  if (d != 64 && d != 128) return fail(AVQ_ERR_UNSUPPORTED, "d=%d: only 64 and 128", d);
  if (Ch != 0 && Ch != 1 && Ch != 2 && Ch != 4 && Ch != 8 && Ch != 16)
    return fail(AVQ_ERR_UNSUPPORTED, "Ch=%d: only 0 (flat codebook), 1, 2, 4, 8, 16", Ch);
  if (M0 > 512) return fail(AVQ_ERR_UNSUPPORTED, "M0=%d: at most 512", M0);
  if (N > (1 << 24)) return fail(AVQ_ERR_UNSUPPORTED, "N=%d: at most 2^24 keys per head", N);
  const long long elems = (long long)B * H * N * d;
  if (elems >= (1LL << 31))
    return fail(AVQ_ERR_UNSUPPORTED, "B*H*N*d=%lld: must stay below 2^31", elems);
  return AVQ_OK;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace

extern "C" {

int avq_version(void) { return 202; }

const char* avq_last_error(void) { return g_err; }

int64_t avq_packed_bytes(avq_dtype_t dtype, int32_t M0, int32_t Ch, int32_t d) {
  if (dtype != AVQ_F32 && dtype != AVQ_BF16) return -1;
  if (M0 < 1 || Ch < 0 || d < 1 || M0 > 512 || Ch > 16 || d > 128) return -1;
  return (int64_t)avq::packed_layout(M0, Ch, d, dtype == AVQ_BF16 ? 2 : 4).bytes;
}

avq_status_t avq_assign(avq_dtype_t dtype, int32_t B, int32_t H, int32_t N, int32_t d,
                        int32_t M0, int32_t Ch, const void* K, const void* Cp, const void* Cc,
                        int32_t* parent_idx, int32_t* code_idx, void* stream) {
  avq_status_t st = check_common(dtype, B, H, N, d, M0, Ch);
  if (st != AVQ_OK) return st;
  if (!K || !Cp || (!Cc && Ch > 0) || !parent_idx || !code_idx)
    return fail(AVQ_ERR_INVALID_ARG, "avq_assign: null pointer argument");
  if (!aligned16(K) || !aligned16(Cp) || !aligned16(Cc) || !aligned16(parent_idx) ||
      !aligned16(code_idx))
    return fail(AVQ_ERR_INVALID_ARG, "avq_assign: arrays must be 16-byte aligned");
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int BH = B * H;
  hipError_t e;
  if (dtype == AVQ_BF16)
    e = d == 64 ? avq::launch_assign<avq::bf16, 64>(BH, H, N, M0, Ch, K, Cp, Cc, parent_idx, code_idx, true, s)
                : avq::launch_assign<avq::bf16, 128>(BH, H, N, M0, Ch, K, Cp, Cc, parent_idx, code_idx, true, s);
  else
    e = d == 64 ? avq::launch_assign<float, 64>(BH, H, N, M0, Ch, K, Cp, Cc, parent_idx, code_idx, true, s)
                : avq::launch_assign<float, 128>(BH, H, N, M0, Ch, K, Cp, Cc, parent_idx, code_idx, true, s);
  return from_hip(e, "avq_assign launch");
}

avq_status_t avq_aggregate(avq_dtype_t dtype, int32_t B, int32_t H, int32_t N, int32_t d,
                           int32_t M0, int32_t Ch, const void* V, const int32_t* code_idx,
                           float* Vbar, int32_t* counts, void* packed, void* stream) {
  avq_status_t st = check_common(dtype, B, H, N, d, M0, Ch);
  if (st != AVQ_OK) return st;
  if (!V || !code_idx || !counts)
    return fail(AVQ_ERR_INVALID_ARG, "avq_aggregate: null pointer argument");
  if (!Vbar && !packed)
    return fail(AVQ_ERR_INVALID_ARG, "avq_aggregate: Vbar and packed are both null");
  if (!aligned16(V) || !aligned16(code_idx) || !aligned16(Vbar) || !aligned16(counts) ||
      !aligned16(packed))
    return fail(AVQ_ERR_INVALID_ARG, "avq_aggregate: arrays must be 16-byte aligned");
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int BH = B * H;
  hipError_t e =
      dtype == AVQ_BF16
          ? avq::launch_aggregate<avq::bf16>(BH, N, d, M0, Ch, V, code_idx, Vbar, counts, packed, s)
          : avq::launch_aggregate<float>(BH, N, d, M0, Ch, V, code_idx, Vbar, counts, packed, s);
  return from_hip(e, "avq_aggregate launch");
}

avq_status_t avq_assign_aggregate(avq_dtype_t dtype, int32_t B, int32_t H, int32_t N,
                                  int32_t d, int32_t M0, int32_t Ch, const void* K,
                                  const void* V, const void* Cp, const void* Cc,
                                  int32_t* parent_idx, int32_t* code_idx, float* Vbar,
                                  int32_t* counts, void* packed, void* stream) {
  avq_status_t st = check_common(dtype, B, H, N, d, M0, Ch);
  if (st != AVQ_OK) return st;
  if (!K || !V || !Cp || (!Cc && Ch > 0) || !parent_idx || !code_idx || !counts)
    return fail(AVQ_ERR_INVALID_ARG, "avq_assign_aggregate: null pointer argument");
  if (!Vbar && !packed)
    return fail(AVQ_ERR_INVALID_ARG, "avq_assign_aggregate: Vbar and packed are both null");
  if (!aligned16(K) || !aligned16(V) || !aligned16(Cp) || !aligned16(Cc) ||
      !aligned16(parent_idx) || !aligned16(code_idx) || !aligned16(Vbar) || !aligned16(counts) ||
      !aligned16(packed))
    return fail(AVQ_ERR_INVALID_ARG, "avq_assign_aggregate: arrays must be 16-byte aligned");
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int BH = B * H;
  hipError_t e =
      dtype == AVQ_BF16
          ? avq::launch_assign_aggregate<avq::bf16>(BH, H, N, d, M0, Ch, K, V, Cp, Cc, parent_idx,
                                                    code_idx, Vbar, counts, packed, s)
          : avq::launch_assign_aggregate<float>(BH, H, N, d, M0, Ch, K, V, Cp, Cc, parent_idx,
                                                code_idx, Vbar, counts, packed, s);
  return from_hip(e, "avq_assign_aggregate launch");
}

avq_status_t avq_pack_aggregates(avq_dtype_t dtype, int32_t B, int32_t H, int32_t d,
                                 int32_t M0, int32_t Ch, const float* Vbar,
                                 const int32_t* counts, void* packed, void* stream) {
  avq_status_t st = check_common(dtype, B, H, 1, d, M0, Ch);
  if (st != AVQ_OK) return st;
  if (!Vbar || !counts || !packed)
    return fail(AVQ_ERR_INVALID_ARG, "avq_pack_aggregates: null pointer argument");
  if (!aligned16(Vbar) || !aligned16(counts) || !aligned16(packed))
    return fail(AVQ_ERR_INVALID_ARG, "avq_pack_aggregates: arrays must be 16-byte aligned");
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int BH = B * H;
  hipError_t e = dtype == AVQ_BF16
                     ? avq::launch_pack<avq::bf16>(BH, M0, Ch, d, Vbar, counts, packed, s)
                     : avq::launch_pack<float>(BH, M0, Ch, d, Vbar, counts, packed, s);
  return from_hip(e, "avq_pack_aggregates launch");
}

}  // extern "C"

namespace {

// avq_attention_fwd and avq_attention_fwd_tiled: the same checks and launch;
// tiled selects the App. B importance.
avq_status_t attention(const char* name, bool tiled, const int32_t* order, avq_dtype_t dtype,
                       int32_t B, int32_t H, int32_t N, int32_t d, int32_t M0, int32_t Ch,
                       int32_t P, int32_t block_q, const void* Q, const void* Cp, const void* Cc,
                       const void* packed, void* Y, int32_t* topp_idx, float* importance,
                       void* stream) {
  avq_status_t st = check_common(dtype, B, H, N, d, M0, Ch);
  if (st != AVQ_OK) return st;
  if (P < 0 || P > M0) return fail(AVQ_ERR_INVALID_ARG, "P=%d outside [0, M0=%d]", P, M0);
  if (Ch == 0 && P != 0)
    return fail(AVQ_ERR_INVALID_ARG, "P=%d with a flat codebook (Ch=0): must be 0", P);
  if (block_q < 1) return fail(AVQ_ERR_INVALID_ARG, "block_q=%d must be positive", block_q);
  if (block_q > 256) return fail(AVQ_ERR_UNSUPPORTED, "block_q=%d: at most 256", block_q);
  if (!Q || !Cp || (!Cc && Ch > 0) || !packed || !Y)
    return fail(AVQ_ERR_INVALID_ARG, "%s: null pointer argument", name);
  if (!aligned16(Q) || !aligned16(Cp) || !aligned16(Cc) || !aligned16(packed) ||
      !aligned16(Y) || !aligned16(topp_idx) || !aligned16(importance) || !aligned16(order))
    return fail(AVQ_ERR_INVALID_ARG, "%s: arrays must be 16-byte aligned", name);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int BH = B * H;
  hipError_t e;
  if (dtype == AVQ_BF16)
    e = d == 64 ? avq::launch_attention<avq::bf16, 64>(BH, H, N, M0, Ch, P, block_q, Q, Cp, Cc,
                                                       packed, Y, topp_idx, importance, tiled, order, s)
                : avq::launch_attention<avq::bf16, 128>(BH, H, N, M0, Ch, P, block_q, Q, Cp, Cc,
                                                        packed, Y, topp_idx, importance, tiled, order, s);
  else
    e = d == 64 ? avq::launch_attention<float, 64>(BH, H, N, M0, Ch, P, block_q, Q, Cp, Cc,
                                                   packed, Y, topp_idx, importance, tiled, order, s)
                : avq::launch_attention<float, 128>(BH, H, N, M0, Ch, P, block_q, Q, Cp, Cc,
                                                    packed, Y, topp_idx, importance, tiled, order, s);
  return from_hip(e, "attention launch");
}

}  // namespace

extern "C" {

avq_status_t avq_attention_fwd(avq_dtype_t dtype, int32_t B, int32_t H, int32_t N, int32_t d,
                               int32_t M0, int32_t Ch, int32_t P, int32_t block_q,
                               const void* Q, const void* Cp, const void* Cc,
                               const void* packed, void* Y,
                               int32_t* topp_idx, float* importance, void* stream) {
  return attention("avq_attention_fwd", false, nullptr, dtype, B, H, N, d, M0, Ch, P, block_q, Q, Cp, Cc,
                   packed, Y, topp_idx, importance, stream);
}

avq_status_t avq_attention_fwd_tiled(avq_dtype_t dtype, int32_t B, int32_t H, int32_t N,
                                     int32_t d, int32_t M0, int32_t Ch, int32_t P,
                                     int32_t block_q, const void* Q, const void* Cp,
                                     const void* Cc, const void* packed, void* Y,
                                     int32_t* topp_idx, float* importance, void* stream) {
  return attention("avq_attention_fwd_tiled", true, nullptr, dtype, B, H, N, d, M0, Ch, P, block_q, Q, Cp,
                   Cc, packed, Y, topp_idx, importance, stream);
}

avq_status_t avq_codebook_update(avq_dtype_t dtype, int32_t B, int32_t H, int32_t d,
                                 int32_t M0, int32_t Ch, float lambda, const float* sums,
                                 const int32_t* counts, float* S, float* Nema, void* Cp_out,
                                 void* Cc_out, void* stream) {
  avq_status_t st = check_common(dtype, B, H, 1, d, M0, Ch);
  if (st != AVQ_OK) return st;
  if (!(lambda > 0.f && lambda <= 1.f))
    return fail(AVQ_ERR_INVALID_ARG, "lambda=%g outside (0, 1]", (double)lambda);
  if (!sums || !counts || !S || !Nema || !Cp_out || (!Cc_out && Ch > 0))
    return fail(AVQ_ERR_INVALID_ARG, "avq_codebook_update: null pointer argument");
  if (!aligned16(sums) || !aligned16(counts) || !aligned16(S) || !aligned16(Nema) ||
      !aligned16(Cp_out) || !aligned16(Cc_out))
    return fail(AVQ_ERR_INVALID_ARG, "avq_codebook_update: arrays must be 16-byte aligned");
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e =
      dtype == AVQ_BF16
          ? avq::launch_codebook_update<avq::bf16>(B, H, d, M0, Ch, lambda, sums, counts, S, Nema,
                                                   Cp_out, Cc_out, s)
          : avq::launch_codebook_update<float>(B, H, d, M0, Ch, lambda, sums, counts, S, Nema,
                                               Cp_out, Cc_out, s);
  return from_hip(e, "avq_codebook_update launch");
}

avq_status_t avq_attention_fwd_ordered(avq_dtype_t dtype, int32_t B, int32_t H, int32_t N,
                                       int32_t d, int32_t M0, int32_t Ch, int32_t P,
                                       int32_t block_q, const int32_t* query_order,
                                       int32_t tiled_importance, const void* Q, const void* Cp,
                                       const void* Cc, const void* packed, void* Y,
                                       int32_t* topp_idx, float* importance, void* stream) {
  if (!query_order)
    return fail(AVQ_ERR_INVALID_ARG, "avq_attention_fwd_ordered: null query_order");
  if (tiled_importance != 0 && tiled_importance != 1)
    return fail(AVQ_ERR_INVALID_ARG, "tiled_importance=%d: must be 0 or 1", tiled_importance);
  return attention("avq_attention_fwd_ordered", tiled_importance == 1, query_order, dtype, B, H,
                   N, d, M0, Ch, P, block_q, Q, Cp, Cc, packed, Y, topp_idx, importance, stream);
}

avq_status_t avq_gilbert_order(int32_t width, int32_t height, int32_t* order, int32_t* rank) {
  if (width < 1 || height < 1)
    return fail(AVQ_ERR_INVALID_ARG, "grid %d x %d: sizes must be positive", width, height);
  if ((long long)width * height > (1LL << 24))
    return fail(AVQ_ERR_UNSUPPORTED, "grid %d x %d: at most 2^24 cells", width, height);
  if (!order) return fail(AVQ_ERR_INVALID_ARG, "avq_gilbert_order: null order");
  const long long n = avq::gilbert_order(width, height, order);
  if (n != (long long)width * height)
    return fail(AVQ_ERR_INVALID_ARG, "avq_gilbert_order: internal count mismatch");
  if (rank)
    for (long long k = 0; k < n; ++k) rank[order[k]] = (int32_t)k;
  return ok();
}

}  // extern "C"

// ---- exact attention of packed prompts and the paged cache -------------------------------

namespace {

constexpr int64_t kMaxStride = 1 << 22;  // elements between tokens: 64 rows stay below 2^31 bytes
constexpr int kMaxHeads = 1024;
constexpr int kMaxDrafts = 16;

// Workgroups of 256 threads along one dimension of a launch: less than this.
constexpr int64_t kMaxBlocks = 1 << 24;
int64_t cache_segments(int32_t S, int32_t n_q, int32_t Hq, int32_t Hkv) {
  return (int64_t)S * Hkv * ((n_q * (Hq / Hkv) + 15) / 16);
}

avq_status_t check_heads(const char* name, avq_dtype_t dtype, int32_t S, int32_t Hq, int32_t Hkv,
                         int32_t d) {
  if (dtype != AVQ_F32 && dtype != AVQ_BF16)
    return fail(AVQ_ERR_INVALID_ARG, "%s: unknown dtype %d", name, (int)dtype);
  if (S < 1 || Hq < 1 || Hkv < 1 || d < 1)
    return fail(AVQ_ERR_INVALID_ARG, "%s: sizes must be positive (S=%d Hq=%d Hkv=%d d=%d)", name, S,
                Hq, Hkv, d);
  if (Hq % Hkv != 0)
    return fail(AVQ_ERR_INVALID_ARG, "%s: Hq=%d must be a multiple of Hkv=%d", name, Hq, Hkv);
  if (d != 64 && d != 128) return fail(AVQ_ERR_UNSUPPORTED, "%s: d=%d: only 64 and 128", name, d);
  if (Hq > kMaxHeads) return fail(AVQ_ERR_UNSUPPORTED, "%s: Hq=%d: at most %d", name, Hq, kMaxHeads);
  if (S > (1 << 20)) return fail(AVQ_ERR_UNSUPPORTED, "%s: S=%d: at most 2^20 sequences", name, S);
  return AVQ_OK;
}

avq_status_t check_stride(const char* name, const char* what, avq_dtype_t dtype, int64_t stride,
                          int32_t H, int32_t d) {
  const int unit = dtype == AVQ_BF16 ? 8 : 4;
  if (stride < (int64_t)H * d || stride % unit != 0)
    return fail(AVQ_ERR_INVALID_ARG,
                "%s: %s=%lld must be at least heads * d = %lld and a multiple of 16 bytes", name,
                what, (long long)stride, (long long)H * d);
  if (stride > kMaxStride)
    return fail(AVQ_ERR_UNSUPPORTED, "%s: %s=%lld: at most 2^22", name, what, (long long)stride);
  return AVQ_OK;
}

avq_status_t check_scale(const char* name, float scale) {
  // the kernels multiply by scale log2(e): infinite, it would make 0 logits NaN
  if (!(scale > 0.f && scale * avq::kLog2e <= FLT_MAX))
    return fail(AVQ_ERR_INVALID_ARG, "%s: scale=%g must be positive, and finite times log2(e)", name,
                (double)scale);
  return AVQ_OK;
}

avq_status_t check_cache(const char* name, avq_cache_t format, int32_t n_pages, int32_t page_size,
                         int32_t max_pages) {
  if (format != AVQ_CACHE_NATIVE && format != AVQ_CACHE_FP4)
    return fail(AVQ_ERR_INVALID_ARG, "%s: unknown cache format %d", name, (int)format);
  if (n_pages < 1 || max_pages < 1)
    return fail(AVQ_ERR_INVALID_ARG, "%s: n_pages=%d and max_pages=%d must be positive", name,
                n_pages, max_pages);
  if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1)) != 0)
    return fail(AVQ_ERR_UNSUPPORTED, "%s: page_size=%d: only 16, 32, 64, 128, 256", name, page_size);
  if ((int64_t)max_pages * page_size > (1LL << 30))
    return fail(AVQ_ERR_UNSUPPORTED, "%s: max_pages * page_size = %lld: at most 2^30 positions", name,
                (long long)max_pages * page_size);
  return AVQ_OK;
}

avq_status_t misaligned(const char* name) {
  return fail(AVQ_ERR_INVALID_ARG, "%s: arrays must be 16-byte aligned", name);
}
avq_status_t null_pointer(const char* name) {
  return fail(AVQ_ERR_INVALID_ARG, "%s: null pointer argument", name);
}

// calls launch<T, D> for the dtype and head width
#define AVQ_BY_TYPE(launch, ...)                                                        \
  (dtype == AVQ_BF16 ? (d == 64 ? avq::launch<avq::bf16, 64>(__VA_ARGS__)               \
                                : avq::launch<avq::bf16, 128>(__VA_ARGS__))             \
                     : (d == 64 ? avq::launch<float, 64>(__VA_ARGS__)                   \
                                : avq::launch<float, 128>(__VA_ARGS__)))

}  // namespace

extern "C" {

int64_t avq_prompt_attention_workspace(avq_dtype_t dtype, int32_t S, int32_t Tq, int32_t Tk,
                                       int32_t Hq, int32_t d, int32_t causal) {
  if ((dtype != AVQ_F32 && dtype != AVQ_BF16) || (d != 64 && d != 128) || S < 1 ||
      S > (1 << 20) || Hq < 1 || Hq > kMaxHeads || Tq < 0 || Tk < 0 || Tq > (1 << 24) ||
      Tk > (1 << 24) || (causal != 0 && causal != 1) ||
      ((int64_t)Tq / 128 + S) * Hq >= kMaxBlocks)
    return -1;
  return (int64_t)AVQ_BY_TYPE(prompt_attention_workspace, S, Tq, Tk, Hq, causal);
}

avq_status_t avq_prompt_attention_fwd(avq_dtype_t dtype, int32_t S, int32_t Tq, int32_t Tk,
                                      int32_t Hq, int32_t Hkv, int32_t d, float scale,
                                      int32_t causal, const void* Q, int64_t q_stride,
                                      const void* K, int64_t k_stride, const void* V,
                                      int64_t v_stride, const int32_t* cu_q, const int32_t* cu_k,
                                      void* Y, float* lse, void* workspace,
                                      int64_t workspace_bytes, void* stream) {
  const char* name = "avq_prompt_attention_fwd";
  avq_status_t st = check_heads(name, dtype, S, Hq, Hkv, d);
  if (st == AVQ_OK) st = check_stride(name, "q_stride", dtype, q_stride, Hq, d);
  if (st == AVQ_OK) st = check_stride(name, "k_stride", dtype, k_stride, Hkv, d);
  if (st == AVQ_OK) st = check_stride(name, "v_stride", dtype, v_stride, Hkv, d);
  if (st == AVQ_OK) st = check_scale(name, scale);
  if (st != AVQ_OK) return st;
  if (Tq < 0 || Tk < 0)
    return fail(AVQ_ERR_INVALID_ARG, "%s: Tq=%d and Tk=%d must not be negative", name, Tq, Tk);
  if (Tq > (1 << 24) || Tk > (1 << 24))
    return fail(AVQ_ERR_UNSUPPORTED, "%s: Tq=%d, Tk=%d: at most 2^24 tokens", name, Tq, Tk);
  if (((int64_t)Tq / 128 + S) * Hq >= kMaxBlocks)
    return fail(AVQ_ERR_UNSUPPORTED, "%s: Tq=%d tokens of S=%d sequences and Hq=%d heads: too many",
                name, Tq, S, Hq);
  if (causal != 0 && causal != 1)
    return fail(AVQ_ERR_INVALID_ARG, "%s: causal=%d: must be 0 or 1", name, causal);
  if (!cu_q || !cu_k || (Tq > 0 && (!Q || !Y)) || (Tk > 0 && (!K || !V))) return null_pointer(name);
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(cu_q) || !aligned16(cu_k) ||
      !aligned16(Y) || !aligned16(lse) || !aligned16(workspace))
    return misaligned(name);
  const int64_t need = avq_prompt_attention_workspace(dtype, S, Tq, Tk, Hq, d, causal);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return fail(AVQ_ERR_INVALID_ARG, "%s: workspace of %lld bytes, %lld are needed", name,
                workspace ? (long long)workspace_bytes : 0LL, (long long)need);
  if (Tq == 0) return ok();
  hipStream_t s = static_cast<hipStream_t>(stream);
  return from_hip(AVQ_BY_TYPE(launch_prompt_attention, S, Tq, Tk, Hq, Hkv, scale, causal, Q,
                              q_stride, K, k_stride, V, v_stride, cu_q, cu_k, Y, lse, workspace, s),
                  "avq_prompt_attention_fwd launch");
}

int64_t avq_cache_page_bytes(avq_dtype_t dtype, avq_cache_t format, int32_t page_size, int32_t d) {
  if ((dtype != AVQ_F32 && dtype != AVQ_BF16) || (d != 64 && d != 128)) return -1;
  if (format != AVQ_CACHE_NATIVE && format != AVQ_CACHE_FP4) return -1;
  if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1)) != 0) return -1;
  return (int64_t)avq::page_layout(format == AVQ_CACHE_FP4, dtype == AVQ_BF16 ? 2 : 4, page_size, d)
      .bytes;
}

avq_status_t avq_cache_append(avq_dtype_t dtype, avq_cache_t format, int32_t S, int32_t T,
                              int32_t Hq, int32_t Hkv, int32_t d, int32_t n_pages,
                              int32_t page_size, int32_t max_pages, int32_t rot, int32_t n_pos,
                              int32_t interleaved, const void* Q, int64_t q_stride, const void* K,
                              int64_t k_stride, const void* V, int64_t v_stride,
                              const int32_t* cu, const int32_t* start, const int32_t* block_table,
                              const float* cos, const float* sin, void* cache, void* Q_out,
                              void* K_out, void* stream) {
  const char* name = "avq_cache_append";
  avq_status_t st = check_heads(name, dtype, S, Q ? Hq : Hkv, Hkv, d);
  if (st == AVQ_OK) st = check_cache(name, format, n_pages, page_size, max_pages);
  if (st == AVQ_OK && Q) st = check_stride(name, "q_stride", dtype, q_stride, Hq, d);
  if (st == AVQ_OK) st = check_stride(name, "k_stride", dtype, k_stride, Hkv, d);
  if (st == AVQ_OK) st = check_stride(name, "v_stride", dtype, v_stride, Hkv, d);
  if (st != AVQ_OK) return st;
  if (T < 0) return fail(AVQ_ERR_INVALID_ARG, "%s: T=%d must not be negative", name, T);
  if (T > (1 << 24)) return fail(AVQ_ERR_UNSUPPORTED, "%s: T=%d: at most 2^24 tokens", name, T);
  if (!cu && T != S)
    return fail(AVQ_ERR_INVALID_ARG, "%s: without cu, T=%d must be S=%d (one token each)", name, T, S);
  if (rot < 0 || rot > d || rot % 16 != 0)
    return fail(AVQ_ERR_INVALID_ARG, "%s: rot=%d must be a multiple of 16 in [0, d=%d]", name, rot, d);
  if (rot > 0 && (!cos || !sin || n_pos < 1))
    return fail(AVQ_ERR_INVALID_ARG, "%s: rot=%d needs cos, sin and n_pos >= 1", name, rot);
  if (interleaved != 0 && interleaved != 1)
    return fail(AVQ_ERR_INVALID_ARG, "%s: interleaved=%d: must be 0 or 1", name, interleaved);
  if ((T > 0 && (!K || !V)) || !start || !block_table || !cache || (!Q != !Q_out))
    return null_pointer(name);
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(cu) || !aligned16(start) ||
      !aligned16(block_table) || !aligned16(cos) || !aligned16(sin) || !aligned16(cache) ||
      !aligned16(Q_out) || !aligned16(K_out))
    return misaligned(name);
  if (T == 0) return ok();
  const avq::CacheShape c{format == AVQ_CACHE_FP4, n_pages, page_size, max_pages, Hkv};
  hipStream_t s = static_cast<hipStream_t>(stream);
  return from_hip(AVQ_BY_TYPE(launch_cache_append, c, S, T, Hq, rot, n_pos, interleaved, Q, q_stride,
                              K, k_stride, V, v_stride, cu, start, block_table, cos, sin, cache,
                              Q_out, K_out, s),
                  "avq_cache_append launch");
}

avq_status_t avq_cache_gather(avq_dtype_t dtype, avq_cache_t format, int32_t S, int32_t T,
                              int32_t Hkv, int32_t d, int32_t n_pages, int32_t page_size,
                              int32_t max_pages, const void* cache, const int32_t* cu,
                              const int32_t* start, const int32_t* block_table, void* K, void* V,
                              void* stream) {
  const char* name = "avq_cache_gather";
  avq_status_t st = check_heads(name, dtype, S, Hkv, Hkv, d);
  if (st == AVQ_OK) st = check_cache(name, format, n_pages, page_size, max_pages);
  if (st != AVQ_OK) return st;
  if (T < 0) return fail(AVQ_ERR_INVALID_ARG, "%s: T=%d must not be negative", name, T);
  if (T > (1 << 24)) return fail(AVQ_ERR_UNSUPPORTED, "%s: T=%d: at most 2^24 tokens", name, T);
  if (!cache || !cu || !start || !block_table || (T > 0 && (!K || !V))) return null_pointer(name);
  if (!aligned16(cache) || !aligned16(cu) || !aligned16(start) || !aligned16(block_table) ||
      !aligned16(K) || !aligned16(V))
    return misaligned(name);
  if (T == 0) return ok();
  const avq::CacheShape c{format == AVQ_CACHE_FP4, n_pages, page_size, max_pages, Hkv};
  hipStream_t s = static_cast<hipStream_t>(stream);
  return from_hip(AVQ_BY_TYPE(launch_cache_gather, c, S, T, cache, cu, start, block_table, K, V, s),
                  "avq_cache_gather launch");
}

int64_t avq_cache_attention_workspace(int32_t S, int32_t n_q, int32_t Hq, int32_t Hkv, int32_t d) {
  if (S < 1 || S > (1 << 20) || n_q < 1 || n_q > kMaxDrafts || Hq < 1 || Hkv < 1 ||
      Hq > kMaxHeads || Hq % Hkv != 0 || (d != 64 && d != 128) ||
      cache_segments(S, n_q, Hq, Hkv) >= kMaxBlocks)
    return -1;
  return (int64_t)avq::cache_attention_workspace(S, n_q, Hq, Hkv, d);
}

avq_status_t avq_cache_attention_fwd(avq_dtype_t dtype, avq_cache_t format, int32_t S, int32_t n_q,
                                     int32_t Hq, int32_t Hkv, int32_t d, int32_t n_pages,
                                     int32_t page_size, int32_t max_pages, float scale,
                                     const void* Q, int64_t q_stride, const void* cache,
                                     const int32_t* lens, const int32_t* block_table, void* Y,
                                     float* lse, void* workspace, int64_t workspace_bytes,
                                     void* stream) {
  const char* name = "avq_cache_attention_fwd";
  avq_status_t st = check_heads(name, dtype, S, Hq, Hkv, d);
  if (st == AVQ_OK) st = check_cache(name, format, n_pages, page_size, max_pages);
  if (st == AVQ_OK) st = check_stride(name, "q_stride", dtype, q_stride, Hq, d);
  if (st == AVQ_OK) st = check_scale(name, scale);
  if (st != AVQ_OK) return st;
  if (n_q < 1) return fail(AVQ_ERR_INVALID_ARG, "%s: n_q=%d must be positive", name, n_q);
  if (n_q > kMaxDrafts)
    return fail(AVQ_ERR_UNSUPPORTED, "%s: n_q=%d: at most %d tokens per sequence", name, n_q,
                kMaxDrafts);
  if (cache_segments(S, n_q, Hq, Hkv) >= kMaxBlocks)
    return fail(AVQ_ERR_UNSUPPORTED, "%s: S=%d sequences of Hq=%d, Hkv=%d heads: too many", name, S,
                Hq, Hkv);
  if ((int64_t)S * (((int64_t)max_pages * page_size + 127) / 128) > (1LL << 30))
    return fail(AVQ_ERR_UNSUPPORTED, "%s: S * max_pages * page_size: at most 2^37 positions", name);
  const bool divided = (int64_t)max_pages * page_size > AVQ_CACHE_UNDIVIDED;
  if (!Q || !cache || !lens || !block_table || !Y || (divided && !workspace))
    return null_pointer(name);
  if (!aligned16(Q) || !aligned16(cache) || !aligned16(lens) || !aligned16(block_table) ||
      !aligned16(Y) || !aligned16(lse) || !aligned16(workspace))
    return misaligned(name);
  const int64_t need = workspace ? avq_cache_attention_workspace(S, n_q, Hq, Hkv, d) : 0;
  if (workspace_bytes < need)
    return fail(AVQ_ERR_INVALID_ARG, "%s: workspace of %lld bytes, %lld are needed", name,
                (long long)workspace_bytes, (long long)need);
  const avq::CacheShape c{format == AVQ_CACHE_FP4, n_pages, page_size, max_pages, Hkv};
  hipStream_t s = static_cast<hipStream_t>(stream);
  return from_hip(AVQ_BY_TYPE(launch_cache_attention, c, S, n_q, Hq, scale, Q, q_stride, cache, lens,
                              block_table, Y, lse, workspace, s),
                  "avq_cache_attention_fwd launch");
}

}  // extern "C"
