// gbla_norm.hip -- the residual's addition and the RMS norm over the width, with an output
// in the activations' type or in eight bits with scales, and its backward (gfx950).
//
//   s = x + residual (rounded to its type),  y = s / sqrt(mean s^2 + eps) w
// A row lies in the registers of its lanes (8 to 64 lanes of a wave, or a workgroup), eight
// channels a piece, so everything is read once and written once, and the sums over the row are
// lane exchanges (and one round through LDS for rows of a workgroup).  Both directions are
// bound by HBM: 32768 rows of 1024 into eight bits 51 us (236 MB at 4.6 TB/s), 5001 rows of 1288
// fp32 19 us (5.4, partly from the cache); backward, 16384 rows of 1024 27 + 5 us (134 MB, the
// sums of the weights' gradient behind), 4097 rows of 4096 fp32 55 + 5 us (268 MB at 4.9).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "gbla_device.h"
#include "gbla_norm.h"

namespace gbla {
namespace {

template <typename T>
__device__ __forceinline__ void load8(const T* p, float* x) {
  if constexpr (sizeof(T) == 2) {
    const u32x4_t v = load16(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = bf16_lo(v[i]), x[2 * i + 1] = bf16_hi(v[i]);
  } else {
    const f32x4_t a = *reinterpret_cast<const f32x4_t*>(p), b = *reinterpret_cast<const f32x4_t*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float* x) {
  if constexpr (sizeof(T) == 2) {
    u32x4_t v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
    *reinterpret_cast<u32x4_t*>(p) = v;
  } else {
    *reinterpret_cast<f32x4_t*>(p) = (f32x4_t){x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4_t*>(p + 4) = (f32x4_t){x[4], x[5], x[6], x[7]};
  }
}
// x as its type holds it
template <typename T>
__device__ __forceinline__ void round8(float* x) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t v = pack_bf16x2(x[2 * i], x[2 * i + 1]);
      x[2 * i] = bf16_lo(v);
      x[2 * i + 1] = bf16_hi(v);
    }
  }
}

// Sum (or maximum) over the L lanes of a row.  Rows of a workgroup: `red` has a place for
// each wave; the calls of a row take different ones.
template <int L, bool Max>
__device__ __forceinline__ float row_reduce(float x, float* red) {
  auto join = [](float a, float b) { return Max ? fmaxf(a, b) : a + b; };
#pragma unroll
  for (int o = 1; o < (L < 64 ? L : 64); o <<= 1) x = join(x, __shfl_xor(x, o));
  if constexpr (L == kThreads) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    x = red[0];
#pragma unroll
    for (int i = 1; i < kThreads / 64; ++i) x = join(x, red[i]);
  }
  return x;
}

// fmaxf passes over NaN: a row's largest magnitude that is NaN where one of its values is.
__device__ __forceinline__ float magnitude8(const float* x, float most, bool& nan) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    most = fmaxf(most, fabsf(x[i]));
    nan |= x[i] != x[i];
  }
  return most;
}

template <typename T, int L, int N, bool Bits8>
__global__ void __launch_bounds__(kThreads)
norm_kernel(NormPlan P, const T* x, const T* residual, const float* w, T* sum, void* out, float* scales) {
  constexpr int kRows = kThreads / L;
  __shared__ float red[2][2][kThreads / 64];
  const int l = threadIdx.x % L;
  int flip = 0;
  for (int64_t first = (int64_t)blockIdx.x * kRows; first < P.rows; first += (int64_t)gridDim.x * kRows, flip ^= 1) {
    const int64_t row = first + threadIdx.x / L;
    const bool live = row < P.rows;
    float s[N][8], ss = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = 8 * (l + i * L);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[i][j] = 0.0f;
      if (live && c < P.width) {
        load8(x + row * P.width + c, s[i]);
        if (residual) {
          float r[8];
          load8(residual + row * P.width + c, r);
#pragma unroll
          for (int j = 0; j < 8; ++j) s[i][j] += r[j];
          round8<T>(s[i]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) ss = fmaf(s[i][j], s[i][j], ss);
      }
    }
    ss = row_reduce<L, false>(ss, red[flip][0]);
    const float r = rsqrtf(fmaf(ss, P.inv_width, P.eps));
    float most = 0.0f;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = 8 * (l + i * L);
      if (!live || c >= P.width) continue;
      if (sum) store8(sum + row * P.width + c, s[i]);
      float ww[8];
      load8(w + c, ww);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[i][j] = s[i][j] * r * ww[j];
      if constexpr (Bits8) most = P.group ? 0.0f : magnitude8(s[i], most, nan);
      else store8(static_cast<T*>(out) + row * P.width + c, s[i]);
    }
    if constexpr (Bits8) {
      constexpr float kLargest = 448.0f;  // of e4m3
      if (!P.group) {
        most = row_reduce<L, true>(nan ? INFINITY : most, red[flip][1]);
        if (live && l == 0) scales[row] = fmaxf(most / kLargest, 0x1p-126f);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int c = 8 * (l + i * L);
        if (P.group) {  // 128 channels are sixteen lanes' pieces
          bool bad = false;
          const float m = magnitude8(s[i], 0.0f, bad);
          most = row_reduce<16, true>(bad ? INFINITY : m, nullptr);
        }
        if (!live || c >= P.width) continue;
        const float scale = fmaxf(most / kLargest, 0x1p-126f);
        if (P.group && (l & 15) == 0) scales[row * (P.width / 128) + c / 128] = scale;
        // (a scale that is infinite leaves NaN of infinite values and 0 of the others, whose
        // product with it is NaN too)
        int v[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float* y = &s[i][4 * j];
          v[j] = __builtin_amdgcn_cvt_pk_fp8_f32(y[0] / scale, y[1] / scale, v[j], false);
          v[j] = __builtin_amdgcn_cvt_pk_fp8_f32(y[2] / scale, y[3] / scale, v[j], true);
        }
        *reinterpret_cast<u32x2_t*>(static_cast<unsigned char*>(out) + row * P.width + c) =
            (u32x2_t){(uint32_t)v[0], (uint32_t)v[1]};
      }
    }
  }
}

// part[block][width]: the workgroup's sum of dout n.
template <typename T, int L, int N>
__global__ void __launch_bounds__(kThreads)
norm_back_kernel(NormPlan P, const T* sum, const float* w, const T* dout, const T* dsum, T* dx, float* part) {
  constexpr int kRows = kThreads / L;
  __shared__ float red[2][2][kThreads / 64];
  __shared__ float all[kRows > 1 ? kRows * 8 * L * N : 1];
  const int l = threadIdx.x % L;
  float dw[N][8];
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[i][j] = 0.0f;
  int flip = 0;
  for (int64_t first = (int64_t)blockIdx.x * kRows; first < P.rows; first += (int64_t)gridDim.x * kRows, flip ^= 1) {
    const int64_t row = first + threadIdx.x / L;
    const bool live = row < P.rows;
    float s[N][8], u[N][8], ss = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = 8 * (l + i * L);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[i][j] = u[i][j] = 0.0f;
      if (live && c < P.width) {
        load8(sum + row * P.width + c, s[i]);
        load8(dout + row * P.width + c, u[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) ss = fmaf(s[i][j], s[i][j], ss);
      }
    }
    const float r = rsqrtf(fmaf(row_reduce<L, false>(ss, red[flip][0]), P.inv_width, P.eps));
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = 8 * (l + i * L);
      if (!live || c >= P.width) continue;
      float ww[8];
      load8(w + c, ww);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        s[i][j] *= r;
        dw[i][j] = fmaf(u[i][j], s[i][j], dw[i][j]);
        u[i][j] *= ww[j];
        m = fmaf(u[i][j], s[i][j], m);
      }
    }
    m = row_reduce<L, false>(m, red[flip][1]) * P.inv_width;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = 8 * (l + i * L);
      if (!live || c >= P.width) continue;
      float d[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) d[j] = 0.0f;
      if (dsum) load8(dsum + row * P.width + c, d);
#pragma unroll
      for (int j = 0; j < 8; ++j) d[j] = fmaf(r, fmaf(-s[i][j], m, u[i][j]), d[j]);
      store8(dx + row * P.width + c, d);
    }
  }
  float* to = part + (int64_t)blockIdx.x * P.width;
  if constexpr (kRows == 1) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (8 * (l + i * L) < P.width) store8(to + 8 * (l + i * L), dw[i]);
  } else {
    float* mine = all + threadIdx.x / L * (8 * L * N);
#pragma unroll
    for (int i = 0; i < N; ++i) store8(mine + 8 * (l + i * L), dw[i]);
    __syncthreads();
    for (int c = threadIdx.x; c < P.width; c += kThreads) {
      float x = 0.0f;
#pragma unroll
      for (int i = 0; i < kRows; ++i) x += all[i * (8 * L * N) + c];
      to[c] = x;
    }
  }
}

// Sums of the partials over the workgroups: 64 columns by 16 strided parts of a block, each
// compensated, then the parts in order.
constexpr int kSumThreads = 1024;
__global__ void __launch_bounds__(kSumThreads)
norm_sum_kernel(int blocks, int width, const float* part, float* dw) {
  constexpr int parts = kSumThreads / 64;
  __shared__ float red[parts][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = blockIdx.x * 64 + lane;
  float sum = 0.0f, comp = 0.0f;
  if (col < width) {
    int b = w;
    for (; b + 7 * parts < blocks; b += 8 * parts) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = part[(int64_t)(b + i * parts) * width + col];
#pragma unroll
      for (int i = 0; i < 8; ++i) kahan_add(sum, comp, x[i]);
    }
    for (; b < blocks; b += parts) kahan_add(sum, comp, part[(int64_t)b * width + col]);
  }
  red[w][lane] = sum;
  __syncthreads();
  if (w == 0 && col < width) {
    sum = comp = 0.0f;
#pragma unroll
    for (int i = 0; i < parts; ++i) kahan_add(sum, comp, red[i][lane]);
    dw[col] = sum;
  }
}

// f(type, lanes, pieces) of a plan.
template <typename F>
gbla_status by_size(const NormPlan& p, F f) {
  auto sizes = [&](auto t) {
    using std::integral_constant;
    if (p.lanes == 8) f(t, integral_constant<int, 8>{}, integral_constant<int, 1>{});
    else if (p.lanes == 16) f(t, integral_constant<int, 16>{}, integral_constant<int, 1>{});
    else if (p.lanes == 32) f(t, integral_constant<int, 32>{}, integral_constant<int, 1>{});
    else if (p.lanes == 64 && p.pieces == 1) f(t, integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else if (p.lanes == 64 && p.pieces == 2) f(t, integral_constant<int, 64>{}, integral_constant<int, 2>{});
    else if (p.lanes == 64) f(t, integral_constant<int, 64>{}, integral_constant<int, 4>{});
    else if (p.pieces == 2) f(t, integral_constant<int, kThreads>{}, integral_constant<int, 2>{});
    else if (p.pieces == 4) f(t, integral_constant<int, kThreads>{}, integral_constant<int, 4>{});
    else f(t, integral_constant<int, kThreads>{}, integral_constant<int, 8>{});
  };
  if (p.dtype == GBLA_BF16) sizes(uint16_t{});
  else sizes(float{});
  return hipGetLastError() == hipSuccess ? GBLA_OK : GBLA_ERR_HIP;
}

}  // namespace

gbla_status launch_norm(const NormPlan& p, const void* x, const void* residual, const float* w,
                        void* sum, void* out, float* scales, hipStream_t st) {
  if (p.rows == 0) return GBLA_OK;
  return by_size(p, [&](auto t, auto lanes, auto pieces) {
    using T = decltype(t);
    constexpr int L = decltype(lanes)::value, N = decltype(pieces)::value;
    const auto kernel = p.out_dtype == GBLA_E4M3 ? norm_kernel<T, L, N, true> : norm_kernel<T, L, N, false>;
    hipLaunchKernelGGL(kernel, dim3(p.blocks), dim3(kThreads), 0, st, p, (const T*)x, (const T*)residual, w,
                       (T*)sum, out, scales);
  });
}

gbla_status launch_norm_backward(const NormPlan& p, const void* sum, const float* w,
                                 const void* dout, const void* dsum, void* ws, void* dx, float* dw,
                                 hipStream_t st) {
  const bool one = p.rows > 0 && p.blocks == 1;  // whose partial sum is all there is
  float* part = one ? dw : static_cast<float*>(ws);
  return by_size(p, [&](auto t, auto lanes, auto pieces) {
    using T = decltype(t);
    constexpr int L = decltype(lanes)::value, N = decltype(pieces)::value;
    if (p.rows > 0)
      hipLaunchKernelGGL((norm_back_kernel<T, L, N>), dim3(p.blocks), dim3(kThreads), 0, st, p, (const T*)sum, w,
                         (const T*)dout, (const T*)dsum, (T*)dx, part);
    if (!one)
      hipLaunchKernelGGL(norm_sum_kernel, dim3((p.width + 63) / 64), dim3(kSumThreads), 0, st,
                         p.rows > 0 ? p.blocks : 0, p.width, part, dw);
  });
}

}  // namespace gbla
