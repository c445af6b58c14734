// Rotary positions with several axes (time, height, width): pair i of a token's
// head is rotated by the angle of the token's position on the pair's axis.
//
//   a' = a cos - b sin,  b' = b cos + a sin,  cos, sin of (pos[t][axis_i], i)
//
// and back, with -sin: the gradient of the rotation, since it is orthogonal.
//
// Bound by the rows' bytes, each read once and written once. A wave takes one
// token and all its heads, queries' and keys': its lanes hold two 16-byte pieces
// of a head each (the a's and the b's of 8 bf16 or 4 fp32 pairs) and the angles of
// these pairs, the same for all heads. The angles are looked up by pairs, one per lane
// in any order of the axes, and handed over in LDS: two loads a lane, where looking up
// a lane's own eight pairs takes up to 16 (20003 tokens of 16 heads of 128, half of
// the dimensions rotated, axes in turn: 37.1 us so, 35.3 now, 4.7 TB/s; 16384 tokens of
// 40 heads of 128 63 us, 5.3 TB/s, the rate of a large copy).
#include "avq_launch.hpp"
#include "avq_common.hpp"

namespace avq {

namespace {

struct RotateArgs {
  const void *Q, *K;
  int64_t q_stride, k_stride;  // elements between tokens
  const int32_t* pos;          // [T][n_axes]
  const float *cos, *sin;      // [n_pos][rot / 2]
  void *Q_out, *K_out;
  int T, Hq, H, rot, n_axes, n_pos;  // H: heads of queries and keys
  uint32_t axes[4];                  // axis of each pair, 2 bits
  float sign;                        // of the sines
};

constexpr int kWavesPerGroup = 4;
constexpr int kAhead = 4;  // heads a lane has in flight

template <typename T, int D, bool kInterleaved>
__global__ __launch_bounds__(64 * kWavesPerGroup) void rotate_kernel(RotateArgs a) {
  constexpr int P = 16 / (int)sizeof(T);  // elements of a piece, pairs of a lane
  constexpr int C = D / (2 * P);          // lanes per head
  constexpr int HP = kWave / C;           // heads per step of the wave
  const int lane = threadIdx.x % kWave;
  const int t = __builtin_amdgcn_readfirstlane(blockIdx.x * kWavesPerGroup + threadIdx.x / kWave);
  if (t >= a.T) return;
  // the token's positions; one outside the tables: nothing is written
  int at[4] = {0, 0, 0, 0};
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < a.n_axes) {
      at[i] = a.pos[(size_t)t * a.n_axes + i];
      bad = bad || (unsigned)at[i] >= (unsigned)a.n_pos;
    }
  if (bad) return;

  const int chunk = lane % C, i0 = chunk * P, half = a.rot / 2;
  const bool turns = i0 < half;
  const int d_a = turns && !kInterleaved ? i0 : 2 * i0;
  const int d_b = turns && !kInterleaved ? half + i0 : 2 * i0 + P;

  typedef T Piece __attribute__((ext_vector_type(P)));
  const T* q_in = static_cast<const T*>(a.Q) + (size_t)t * a.q_stride;
  const T* k_in = static_cast<const T*>(a.K) + (size_t)t * a.k_stride;
  T* q_out = static_cast<T*>(a.Q_out) + (size_t)t * a.Hq * D;
  T* k_out = static_cast<T*>(a.K_out) + (size_t)t * (a.H - a.Hq) * D;
  Piece x[kAhead], y[kAhead];
  auto load = [&](int h0) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int h = h0 + HP * i;
      if (h < a.H) {
        const T* p = h < a.Hq ? q_in + (size_t)h * D : k_in + (size_t)(h - a.Hq) * D;
        x[i] = *reinterpret_cast<const Piece*>(p + d_a);
        y[i] = *reinterpret_cast<const Piece*>(p + d_b);
      }
    }
  };
  load(lane / C);

  // the angle of pair `lane`, then those of the lane's pairs
  __shared__ __attribute__((aligned(16))) float s_angle[kWavesPerGroup][2][kWave];
  float(&angle)[2][kWave] = s_angle[threadIdx.x / kWave];
  if (lane < half) {
    const int w = lane / 16;
    const uint32_t word = w == 0 ? a.axes[0] : w == 1 ? a.axes[1] : w == 2 ? a.axes[2] : a.axes[3];
    const int axis = word >> (2 * (lane % 16)) & 3;
    const int row = axis == 0 ? at[0] : axis == 1 ? at[1] : axis == 2 ? at[2] : at[3];
    angle[0][lane] = a.cos[(size_t)row * half + lane];
    angle[1][lane] = a.sin[(size_t)row * half + lane] * a.sign;
  }
  __builtin_amdgcn_wave_barrier();  // only this wave reads them: its LDS accesses stay in order
  float c[P], s[P];
  if (turns) {
#pragma unroll
    for (int j = 0; j < P; ++j) c[j] = angle[0][i0 + j], s[j] = angle[1][i0 + j];
  }

  for (int h0 = lane / C; h0 < a.H; h0 += HP * kAhead) {
    if (h0 >= HP * kAhead) load(h0);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int h = h0 + HP * i;
      if (h >= a.H) continue;
      if (turns) {
        if constexpr (kInterleaved) {
#pragma unroll
          for (int j = 0; j < P; j += 2) {
            const float u = (float)x[i][j], v = (float)x[i][j + 1];
            x[i][j] = (T)(u * c[j / 2] - v * s[j / 2]);
            x[i][j + 1] = (T)(v * c[j / 2] + u * s[j / 2]);
            const float w = (float)y[i][j], z = (float)y[i][j + 1];
            y[i][j] = (T)(w * c[(P + j) / 2] - z * s[(P + j) / 2]);
            y[i][j + 1] = (T)(z * c[(P + j) / 2] + w * s[(P + j) / 2]);
          }
        } else {
#pragma unroll
          for (int j = 0; j < P; ++j) {
            const float u = (float)x[i][j], v = (float)y[i][j];
            x[i][j] = (T)(u * c[j] - v * s[j]);
            y[i][j] = (T)(v * c[j] + u * s[j]);
          }
        }
      }
      T* p = h < a.Hq ? q_out + (size_t)h * D : k_out + (size_t)(h - a.Hq) * D;
      *reinterpret_cast<Piece*>(p + d_a) = x[i];
      *reinterpret_cast<Piece*>(p + d_b) = y[i];
    }
  }
}

}  // namespace

template <typename T, int D>
hipError_t launch_rotate_axes(int T_, int Hq, int Hkv, int rot, int n_axes, const uint8_t* axis,
                              int n_pos, int interleaved, int inverse, const void* Q,
                              int64_t q_stride, const void* K, int64_t k_stride,
                              const int32_t* pos, const float* cos, const float* sin, void* Q_out,
                              void* K_out, hipStream_t stream) {
  RotateArgs a{Q, K, q_stride, k_stride, pos, cos, sin, Q_out, K_out, T_, Hq, K ? Hq + Hkv : Hq,
               rot, n_axes, n_pos, {0, 0, 0, 0}, inverse ? -1.f : 1.f};
  for (int i = 0; i < rot / 2; ++i) a.axes[i / 16] |= (uint32_t)axis[i] << (2 * (i % 16));
  const unsigned grid = (unsigned)((T_ + kWavesPerGroup - 1) / kWavesPerGroup);
  if (interleaved)
    hipLaunchKernelGGL((rotate_kernel<T, D, true>), dim3(grid), dim3(64 * kWavesPerGroup), 0,
                       stream, a);
  else
    hipLaunchKernelGGL((rotate_kernel<T, D, false>), dim3(grid), dim3(64 * kWavesPerGroup), 0,
                       stream, a);
  return hipGetLastError();
}

#define AVQ_INSTANCE(T, D)                                                                       \
  template hipError_t launch_rotate_axes<T, D>(int, int, int, int, int, const uint8_t*, int, int, \
                                               int, const void*, int64_t, const void*, int64_t,  \
                                               const int32_t*, const float*, const float*, void*, \
                                               void*, hipStream_t);
AVQ_INSTANCE(bf16, 64)
AVQ_INSTANCE(bf16, 128)
AVQ_INSTANCE(float, 64)
AVQ_INSTANCE(float, 128)
#undef AVQ_INSTANCE

}  // namespace avq
