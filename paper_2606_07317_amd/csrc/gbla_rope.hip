// gbla_rope.hip -- RMS norm of every head's queries and keys and the rotation by
// position, one pass over the data each way (gfx950).
//
// A lane holds eight channels of one token: four rotating pairs (a_i, b_i) with
// frequencies 4 t + i, t the lane's place in the row, or eight channels past the
// rotary ones.  D / 8 lanes make a row, so the norm's sum is a few lane exchanges
// and no LDS.  A lane computes its four angles once and uses them for every head of
// its workgroup: an angle is position * turns reduced to a fraction of a turn in 64
// bits (a position of 2^31 leaves an error of 4e-8 turns), its sine and cosine in 32.
//
// Both directions are bound by HBM (B = 1, n = 32768, H = K = 8, d = 64 bf16: 134 MB in
// 26 us, 5.2 TB/s).  The backward also sums u * xn over the tokens for each (head,
// channel): over a wave's rows by lane exchanges, over a workgroup's waves and passes in
// LDS, over the workgroups in a second launch (B = 8, n = 2048, H = K = 16, d = 64: 201 MB
// in 48 us, 4.2 TB/s; 57 with seven instead of eight waves a SIMD, whose grid then takes
// two rounds; 62 with whole sums instead of halving exchanges too).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "gbla_decay.h"
#include "gbla_device.h"
#include "gbla_split.h"

namespace gbla {
namespace {

constexpr int kHeadsEach = 8;  // heads of a workgroup, at most

// Eight channels of a row for lane t: [4t, 4t + 4) and [R/2 + 4t, + 4) as a and b
// where they rotate in halves, else [8t, 8t + 8).
template <typename T, bool Pairs>
struct Row8 {
  static __device__ __forceinline__ bool halves(int t, int R) { return !Pairs && 8 * t < R; }
  static __device__ __forceinline__ void load(const T* row, int t, int R, float* x) {
    const int c0 = halves(t, R) ? 4 * t : 8 * t, c1 = halves(t, R) ? R / 2 + 4 * t : 8 * t + 4;
    float f[8];
    if constexpr (sizeof(T) == 2) {
      const u32x2_t a = *reinterpret_cast<const u32x2_t*>(row + c0);
      const u32x2_t b = *reinterpret_cast<const u32x2_t*>(row + c1);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f[2 * i] = bf16_lo(a[i]), f[2 * i + 1] = bf16_hi(a[i]);
        f[4 + 2 * i] = bf16_lo(b[i]), f[4 + 2 * i + 1] = bf16_hi(b[i]);
      }
    } else {
      const f32x4_t a = *reinterpret_cast<const f32x4_t*>(row + c0);
      const f32x4_t b = *reinterpret_cast<const f32x4_t*>(row + c1);
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = a[i], f[4 + i] = b[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = Pairs ? f[i < 4 ? 2 * i : 2 * (i - 4) + 1] : f[i];
  }
  static __device__ __forceinline__ void store(T* row, int t, int R, const float* y) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = Pairs ? y[(i >> 1) + 4 * (i & 1)] : y[i];
    const int c0 = halves(t, R) ? 4 * t : 8 * t, c1 = halves(t, R) ? R / 2 + 4 * t : 8 * t + 4;
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<u32x2_t*>(row + c0) = (u32x2_t){pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
      *reinterpret_cast<u32x2_t*>(row + c1) = (u32x2_t){pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
    } else {
      *reinterpret_cast<f32x4_t*>(row + c0) = (f32x4_t){x[0], x[1], x[2], x[3]};
      *reinterpret_cast<f32x4_t*>(row + c1) = (f32x4_t){x[4], x[5], x[6], x[7]};
    }
  }
};

// Sum over the D / 8 lanes of a row.
template <int D>
__device__ __forceinline__ float row_sum(float s) {
  s += dpp<0xB1>(s);
  s += dpp<0x4E>(s);
  if constexpr (D >= 64) s += dpp<0x141>(s);
  if constexpr (D >= 128) s += dpp<0x140>(s);
  return s;
}

// Sums over a wave's 64 / L rows of a lane's eight values: halving exchanges while a lane
// has more than one value (4 + 2 + 1 instead of 8 a step), then whole ones.  On return
// v[0 .. N) are the sums of values first .. first + N - 1 of lane t's row place.
template <int L>
struct RowSums {
  static constexpr int N = L == 16 ? 2 : 1;
  template <int Width, int O>
  static __device__ __forceinline__ void halve(float* v, int lane, int& first) {
    const bool high = lane & O;
    first += high ? Width : 0;
#pragma unroll
    for (int i = 0; i < Width; ++i) {
      const float keep = high ? v[i + Width] : v[i], give = high ? v[i] : v[i + Width];
      v[i] = keep + __shfl_xor(give, O);
    }
  }
  static __device__ __forceinline__ int reduce(float* v, int lane) {
    int first = 0;
    halve<4, 32>(v, lane, first);
    halve<2, 16>(v, lane, first);
    if constexpr (L <= 8) halve<1, 8>(v, lane, first);
    if constexpr (L == 4) v[0] += __shfl_xor(v[0], 4);
    return first;
  }
};

// A lane's token: where its row starts in a head of q and of k, or none.
struct Token {
  bool live;
  int64_t row;  // dense: batch and index below; ragged: the packed row
  int64_t b, i;
  int position;
};

__device__ __forceinline__ Token token_at(const RopePlan& P, int64_t tok, const int32_t* pos,
                                          const int32_t* cu) {
  Token t;
  if (P.ragged) {
    t.live = tok < P.tokens && tok < cu[P.nseq];
    t.b = 0;
    t.i = tok;
    t.position = 0;
    if (t.live && !pos) {  // the last sequence that starts at or before the token
      int lo = 0, hi = P.nseq;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid] <= tok) lo = mid;
        else hi = mid;
      }
      t.position = (int)(tok - cu[lo]);
    }
  } else {
    t.live = tok < P.tokens;
    t.b = t.live ? tok / P.rows : 0;
    t.i = tok - t.b * P.rows;
    t.position = (int)t.i;
  }
  if (t.live && pos) t.position = pos[tok];
  return t;
}

// Whether lane t's channels rotate (all of them, or none: R is a multiple of 8).
__device__ __forceinline__ bool rotates(const RopePlan& P, int t) { return 8 * t < P.rotary; }

// cos and sin of the lane's four pairs.
__device__ __forceinline__ void angles(const RopePlan& P, int t, int position, float* c, float* s) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    c[i] = 1.0f;
    s[i] = 0.0f;
  }
  if (!rotates(P, t)) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const double turn = (double)position * P.turns[4 * t + i];
    sincospif(2.0f * (float)(turn - rint(turn)), &s[i], &c[i]);
  }
}

template <typename T>
__device__ __forceinline__ T* head_row(const RopePlan& P, T* base, const Token& t, int heads, int h) {
  if (P.ragged) return base + ((int64_t)h * P.rows + t.i) * P.d;
  return base + ((t.b * heads + h) * P.rows + t.i) * P.d;
}

template <typename T, int D, bool Pairs>
__global__ void __launch_bounds__(kThreads)
rope_kernel(RopePlan P, const T* q, const T* k, const float* q_w, const float* k_w,
            const int32_t* pos, const int32_t* cu, T* q_out, T* k_out) {
  constexpr int L = D / 8;
  const int t = threadIdx.x % L;
  const Token tok = token_at(P, (int64_t)blockIdx.x * P.tile + threadIdx.x / L, pos, cu);
  if (!tok.live) return;
  float c[4], s[4];
  angles(P, t, tok.position, c, s);
  const int h0 = blockIdx.y * P.heads_each, h1 = min(h0 + P.heads_each, P.heads + P.kv_heads);
  const bool turn = rotates(P, t);
  const bool norm = !(P.flags & GBLA_NO_NORM);
  for (int hh = h0; hh < h1; ++hh) {
    const bool isq = hh < P.heads;
    const int h = isq ? hh : hh - P.heads, heads = isq ? P.heads : P.kv_heads;
    float x[8];
    Row8<T, Pairs>::load(head_row(P, isq ? q : k, tok, heads, h), t, P.rotary, x);
    if (norm) {
      float w[8];
      Row8<float, Pairs>::load((isq ? q_w : k_w) + h * D, t, P.rotary, w);
      float ss = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
      const float r = rsqrtf(row_sum<D>(ss) * (1.0f / D) + P.eps);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = x[i] * r * w[i];
    }
    float y[8];
    // by selects: 0 times an infinite or NaN neighbour is no part of a channel that stays
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[i] = turn ? x[i] * c[i] - x[4 + i] * s[i] : x[i];
      y[4 + i] = turn ? x[i] * s[i] + x[4 + i] * c[i] : x[4 + i];
    }
    Row8<T, Pairs>::store(head_row(P, isq ? q_out : k_out, tok, heads, h), t, P.rotary, y);
  }
}

// part[block][head of H + K][D]: the workgroup's sum of u * xn.
template <typename T, int D, bool Pairs>
__global__ void __launch_bounds__(kThreads, 8)
rope_back_kernel(RopePlan P, const T* q, const T* k, const float* q_w, const float* k_w,
                 const int32_t* pos, const int32_t* cu, const T* dq_out, const T* dk_out,
                 T* dq, T* dk, float* part) {
  constexpr int L = D / 8;
  __shared__ float sums[kHeadsEach][kThreads / 64][D];
  const int t = threadIdx.x % L, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int all = P.heads + P.kv_heads;
  const int h0 = blockIdx.y * P.heads_each, h1 = min(h0 + P.heads_each, all);
  const bool turn = rotates(P, t);
  const bool norm = !(P.flags & GBLA_NO_NORM);
  if (norm) {
    for (int i = threadIdx.x; i < kHeadsEach * (kThreads / 64) * D; i += kThreads)
      (&sums[0][0][0])[i] = 0.0f;
    __syncthreads();
  }
  for (int pass = 0; pass < P.passes; ++pass) {
    const Token tok = token_at(
        P, ((int64_t)blockIdx.x * P.passes + pass) * P.tile + threadIdx.x / L, pos, cu);
    float c[4], s[4];
    angles(P, t, tok.position, c, s);
    for (int hh = h0; hh < h1; ++hh) {
      const bool isq = hh < P.heads;
      const int h = isq ? hh : hh - P.heads, heads = isq ? P.heads : P.kv_heads;
      float dw[8], x[8], dy[8], u[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = dy[i] = 0.0f;
      if (tok.live) {
        Row8<T, Pairs>::load(head_row(P, isq ? dq_out : dk_out, tok, heads, h), t, P.rotary, dy);
        if (norm) Row8<T, Pairs>::load(head_row(P, isq ? q : k, tok, heads, h), t, P.rotary, x);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u[i] = turn ? dy[i] * c[i] + dy[4 + i] * s[i] : dy[i];
        u[4 + i] = turn ? dy[4 + i] * c[i] - dy[i] * s[i] : dy[4 + i];
      }
      if (norm) {
        float w[8], ss = 0.0f, uw = 0.0f;
        Row8<float, Pairs>::load((isq ? q_w : k_w) + h * D, t, P.rotary, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
        const float r = rsqrtf(row_sum<D>(ss) * (1.0f / D) + P.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] *= r;
          dw[i] = tok.live ? u[i] * x[i] : 0.0f;
          u[i] *= w[i];
          uw = fmaf(u[i], x[i], uw);
        }
        const float m = row_sum<D>(uw) * (1.0f / D);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = r * (u[i] - x[i] * m);
        const int first = RowSums<L>::reduce(dw, lane);
        if (L > 4 || !(lane & 4)) {
#pragma unroll
          for (int i = 0; i < RowSums<L>::N; ++i) sums[hh - h0][wave][8 * t + first + i] += dw[i];
        }
      }
      if (tok.live)
        Row8<T, Pairs>::store(head_row(P, isq ? dq : dk, tok, heads, h), t, P.rotary, u);
    }
  }
  if (!norm) return;
  __syncthreads();
  // slot 8 t + i of a row holds a_i (i < 4) or b_i of lane t
  for (int i = threadIdx.x; i < (h1 - h0) * D; i += kThreads) {
    const int hh = i / D, slot = i % D, at = slot >> 3, j = slot & 7;
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) sum += sums[hh][w][slot];
    int ch;
    if (Pairs) ch = 8 * at + 2 * (j & 3) + (j >> 2);
    else if (8 * at < P.rotary) ch = (j < 4 ? 0 : P.rotary / 2) + 4 * at + (j & 3);
    else ch = 8 * at + j;
    part[((int64_t)blockIdx.x * all + h0 + hh) * D + ch] = sum;
  }
}

// Sums of the partials over the workgroups: 64 columns by 16 strided parts of a
// block, each compensated, then the parts in order.
constexpr int kSumThreads = 1024;
__global__ void __launch_bounds__(kSumThreads)
rope_sum_kernel(int blocks, int columns, int q_columns, const float* part, float* dq_w, float* dk_w) {
  constexpr int parts = kSumThreads / 64;
  __shared__ float red[parts][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, col = blockIdx.x * 64 + lane;
  float sum = 0.0f, comp = 0.0f;
  if (col < columns) {
    int b = w;
    for (; b + 7 * parts < blocks; b += 8 * parts) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = part[(int64_t)(b + i * parts) * columns + col];
#pragma unroll
      for (int i = 0; i < 8; ++i) kahan_add(sum, comp, x[i]);
    }
    for (; b < blocks; b += parts) kahan_add(sum, comp, part[(int64_t)b * columns + col]);
  }
  red[w][lane] = sum;
  __syncthreads();
  if (w == 0 && col < columns) {
    sum = comp = 0.0f;
#pragma unroll
    for (int i = 0; i < parts; ++i) kahan_add(sum, comp, red[i][lane]);
    if (col < q_columns) dq_w[col] = sum;
    else dk_w[col - q_columns] = sum;
  }
}

template <typename F>
gbla_status by_type(const RopePlan& p, F f) {
  auto dims = [&](auto t) {
    if (p.d == 32) f(t, std::integral_constant<int, 32>{});
    else if (p.d == 64) f(t, std::integral_constant<int, 64>{});
    else f(t, std::integral_constant<int, 128>{});
  };
  if (p.dtype == GBLA_BF16) dims(uint16_t{});
  else dims(float{});
  return hipGetLastError() == hipSuccess ? GBLA_OK : GBLA_ERR_HIP;
}

}  // namespace

gbla_status launch_rope(const RopePlan& p, const void* q, const void* k, const float* q_w,
                        const float* k_w, const int32_t* pos, const int32_t* cu, void* q_out,
                        void* k_out, hipStream_t st) {
  if (p.tokens == 0) return GBLA_OK;
  return by_type(p, [&](auto t, auto dim) {
    using T = decltype(t);
    constexpr int D = decltype(dim)::value;
    const auto run = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3(p.blocks, p.head_blocks), dim3(kThreads), 0, st, p,
                         (const T*)q, (const T*)k, q_w, k_w, pos, cu, (T*)q_out, (T*)k_out);
    };
    if (p.flags & GBLA_ROPE_PAIRS) run(rope_kernel<T, D, true>);
    else run(rope_kernel<T, D, false>);
  });
}

gbla_status launch_rope_backward(const RopePlan& p, const void* q, const void* k, const float* q_w,
                                 const float* k_w, const int32_t* pos, const int32_t* cu,
                                 const void* dq_out, const void* dk_out, void* ws, void* dq,
                                 void* dk, float* dq_w, float* dk_w, hipStream_t st) {
  float* part = static_cast<float*>(ws);
  return by_type(p, [&](auto t, auto dim) {
    using T = decltype(t);
    constexpr int D = decltype(dim)::value;
    const auto run = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3(p.blocks, p.head_blocks), dim3(kThreads), 0, st, p,
                         (const T*)q, (const T*)k, q_w, k_w, pos, cu, (const T*)dq_out,
                         (const T*)dk_out, (T*)dq, (T*)dk, part);
    };
    if (p.tokens > 0) {
      if (p.flags & GBLA_ROPE_PAIRS) run(rope_back_kernel<T, D, true>);
      else run(rope_back_kernel<T, D, false>);
    }
    if (!(p.flags & GBLA_NO_NORM)) {
      const int columns = (p.heads + p.kv_heads) * D;
      hipLaunchKernelGGL(rope_sum_kernel, dim3((columns + 63) / 64), dim3(kSumThreads), 0, st,
                         p.tokens > 0 ? p.blocks : 0, columns, p.heads * D, part, dq_w, dk_w);
    }
  });
}

}  // namespace gbla
