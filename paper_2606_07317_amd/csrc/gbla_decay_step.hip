// gbla_decay_step.hip -- the decay attention for one new token of each row
// (gfx950):  state = lam state + k v^T,  out = scale state^T q.
//
// Nothing but the states moves: each is read and written once, 8 d^2 bytes a key
// head, with two multiply-adds an element.  A workgroup takes one row, one key head
// and a slice of W value channels; a thread holds four value channels of every R-th
// key channel in registers, all its loads in flight at once.  The sums over the key
// channels go over lanes, then over the waves in LDS, in a fixed order.
// Bound by memory: 256 rows, K = 4, d = 128 134 MB in 28 us, 4.8 TB/s; 64 rows, K = 16, d =
// 64 34 MB in 10 us, 3.4 TB/s; one row 4 us, the launch and its chain of loads and sums.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gbla_decay_tiles.h"

namespace gbla {
namespace {

constexpr int kGroup = 4;  // query heads of a pass over the registers

template <typename T, int D, int W>
__global__ void __launch_bounds__(kThreads)
step_kernel(int rows, int heads, int kv_heads, float scale, const T* q, const T* k, const T* v,
            const float* log_decay, const int32_t* indices, int slots, float* state, T* out) {
  constexpr int L = W / 4;             // lanes of a row of the slice
  constexpr int R = kThreads / L;      // key channels of a pass
  constexpr int N = (D + R - 1) / R;   // of a thread
  __shared__ float red[kThreads / 64][kGroup][W];
  __shared__ int same[2];
  const int n0 = blockIdx.x, h = blockIdx.y, e0 = blockIdx.z * W;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int e = (threadIdx.x % L) * 4, c0 = threadIdx.x / L;
  const int group = heads / kv_heads;
  const int slot = indices ? indices[n0] : n0;
  if (slot < 0 || slot >= slots) return;
  const Decay decay(log_decay[h]);
  const float lam = decay(1);
  const bool forgets = decay.forgets();
  float* S = state + ((int64_t)slot * kv_heads + h) * (D * D) + e0 + e;
  f32x4_t s[N];
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (c0 + i * R < D) s[i] = *reinterpret_cast<const f32x4_t*>(S + (c0 + i * R) * D);
  bool more = false;
  if (indices && rows > 1) {  // rows of one slot: the first row's workgroup does them all
    if (threadIdx.x < 2) same[threadIdx.x] = 0;
    __syncthreads();
    for (int m = threadIdx.x; m < rows; m += kThreads)
      if (m != n0 && indices[m] == slot) same[m > n0] = 1;
    __syncthreads();
    if (same[0]) return;
    more = same[1] != 0;
  }
  for (int n = n0; n < rows; ++n) {
    if (n != n0 && indices[n] != slot) continue;
    const T* kk = k + ((int64_t)n * kv_heads + h) * D;
    const T* vv = v + ((int64_t)n * kv_heads + h) * D + e0 + e;
    float vx[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) vx[r] = widen1(vv[r]);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = c0 + i * R;
      const float kx = c < D ? widen1(kk[c]) : 0.0f;
#pragma unroll
      for (int r = 0; r < 4; ++r) s[i][r] = fmaf(kx, vx[r], forgets ? 0.0f : lam * s[i][r]);
    }
    for (int g0 = 0; g0 < group; g0 += kGroup) {
      f32x4_t acc[kGroup];
#pragma unroll
      for (int j = 0; j < kGroup; ++j) {
        acc[j] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
        if (g0 + j >= group) continue;
        const T* qq = q + ((int64_t)n * heads + h * group + g0 + j) * D;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int c = c0 + i * R;
          const float qx = c < D ? widen1(qq[c]) : 0.0f;
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[j][r] = fmaf(qx, s[i][r], acc[j][r]);
        }
#pragma unroll
        for (int o = L; o < 64; o <<= 1)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[j][r] += __shfl_xor(acc[j][r], o);
        if (lane < L) *reinterpret_cast<f32x4_t*>(&red[wave][j][e]) = acc[j];
      }
      __syncthreads();
      const int gs = min(kGroup, group - g0);
      for (int i = threadIdx.x; i < gs * W; i += kThreads) {
        const int j = i / W, x = i % W;
        float y = red[0][j][x];
#pragma unroll
        for (int u = 1; u < kThreads / 64; ++u) y += red[u][j][x];
        y *= scale;
        const int64_t at = ((int64_t)n * heads + h * group + g0 + j) * D + e0 + x;
        if constexpr (sizeof(T) == 2) out[at] = (T)(pack_bf16x2(y, 0.0f) & 0xffffu);
        else out[at] = y;
      }
      if (g0 + kGroup < group || more) __syncthreads();
    }
    if (!more) break;
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (c0 + i * R < D) *reinterpret_cast<f32x4_t*>(S + (c0 + i * R) * D) = s[i];
}

}  // namespace

gbla_status launch_decay_step(const gbla_decay_shape& s, const void* q, const void* k,
                              const void* v, const float* log_decay, const int32_t* indices,
                              int32_t slots, float* state, void* out, hipStream_t st) {
#define GBLA_STEP(T, D, W)                                                                         \
  hipLaunchKernelGGL((step_kernel<T, D, W>), dim3(s.batch, s.kv_heads, D / W), dim3(kThreads), 0,  \
                     st, s.batch, s.heads, s.kv_heads, s.scale, (const T*)q, (const T*)k,          \
                     (const T*)v, log_decay, indices, slots, state, (T*)out)
  const bool half = s.dtype == GBLA_BF16;
  if (s.head_dim == 32) {
    if (half) GBLA_STEP(uint16_t, 32, 32);
    else GBLA_STEP(float, 32, 32);
  } else if (s.head_dim == 64) {
    if (half) GBLA_STEP(uint16_t, 64, 64);
    else GBLA_STEP(float, 64, 64);
  } else {
    if (half) GBLA_STEP(uint16_t, 128, 64);
    else GBLA_STEP(float, 128, 64);
  }
#undef GBLA_STEP
  return hipGetLastError() == hipSuccess ? GBLA_OK : GBLA_ERR_HIP;
}

}  // namespace gbla
