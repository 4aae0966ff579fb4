// gbla_delta_grads.hip -- the gated delta rule's backward, tile by tile in any order (gfx950):
// the gradients of q, k, v and log_decay.
//
// With S the state before the tile, N the gradient of the state after it, u = beta e, dv =
// beta f, and D_ts = e^(c_t - c_s):
//   dq_t = scale (e^c_t S do_t + sum_{s <= t} D_ts (do_t u_s) k_s)
//   dk_t = e^(c_L - c_t) N u_t - e^c_t S dv_t + scale sum_{r >= t} D_rt (do_r u_t) q_r
//          - sum_{s < t} D_ts (dv_t u_s) k_s - sum_{r > t} D_rt (dv_r u_t) k_r
// summed over the value heads that share the query and key head.
//
// The decay's gradient <dZ_t, Z_t> (Z_t = e^g_t S_{t-1}, dZ_t its gradient) goes on from token
// to token: dg_{t+1} = dg_t + dv_t v_t - do_t o_t.  It is anchored where both states are at
// hand, at the start of every unit, and summed from there in 64 bits.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gbla_delta_tiles.h"

namespace gbla {
namespace {

// Two parts of what is computed in fp32: 2^-16 of a term, below the bf16 rounding of the
// gradients that they form.
constexpr int kParts = 2;

// One value of a row-major tile of `live` rows (zero behind them).
template <typename T>
__device__ __forceinline__ float value_at(__amdgpu_buffer_rsrc_t r, int at) {
  if constexpr (sizeof(T) == 2)
    return __uint_as_float((uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, (uint32_t)(2 * at), 0, 0) << 16);
  else
    return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, (uint32_t)(4 * at), 0, 0));
}
template <typename T>
__device__ __forceinline__ Parts<T, 1> exact(const float* x) {
  Parts<T, 1> p;
  p.set(x);
  return p;
}

// Wave w takes the tokens row_of(w, ..) of a tile as its own.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
grads_kernel(DeltaPlan P, TileSpans tiles, const T* q, const T* k, const T* dout, const int32_t* cu,
             const Gates* gates, const float* S, const float* N, const float* E, const float* F, T* dq, T* dk, T* dv) {
  using C = DS<T, D, 4, 1>;
  __shared__ __attribute__((aligned(16))) Gates G;
  Span sp;
  if (!find_span<kThreads>(tiles, cu, blockIdx.x, &sp)) return;
  const int hk = blockIdx.y, lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), own = row_of(w, n);
  const int live = sp.end - sp.begin;
  if (live <= 0) return;
  const int64_t krow = first_row(P, sp, P.heads, hk) + sp.begin;
  const uint32_t bytes = (uint32_t)(live * C::kRow);
  const __amdgpu_buffer_rsrc_t rk = make_rsrc(k + krow * D, bytes), rq = make_rsrc(q + krow * D, bytes);
  f32x4_t aq[C::NB], ak[C::NB];  // channels 16 c + 4 g + r of the own token
#pragma unroll
  for (int c = 0; c < C::NB; ++c) aq[c] = ak[c] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
  for (int gi = 0; gi < P.group; ++gi) {
    const int h = hk * P.group + gi;
    const size_t slot = (size_t)h * P.tiles + sp.slot;
    const int64_t vrow = first_row(P, sp, P.value_heads, h) + sp.begin;
    const __amdgpu_buffer_rsrc_t ro = make_rsrc(dout + vrow * D, bytes);
    __syncthreads();
    if (threadIdx.x < kGateBytes / 16)
      reinterpret_cast<u32x4_t*>(&G)[threadIdx.x] = reinterpret_cast<const u32x4_t*>(gates + slot)[threadIdx.x];
    __syncthreads();
    const float *St = S + slot * (D * D), *Nt = N + slot * (D * D);
    const float *Et = E + slot * (D * kDeltaTile), *Ft = F + slot * (D * kDeltaTile);
    auto vectors = [&](const float* X, int t, int ks, float f, float* x) {  // f X[32 ks + 8 g + j][t]
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = f * X[(32 * ks + 8 * g + j) * kDeltaTile + t];
    };
    auto gradient = [&](int t, int ks, float* x) {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = value_at<T>(ro, t * D + 32 * ks + 8 * g + j);
    };
    Parts<T, kParts> u[C::KS], v[C::KS];
    Parts<T, 1> o[C::KS];
    const float beta = G.beta[own];
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) {
      float x[8];
      vectors(Et, own, ks, beta, x);
      u[ks].set(x);
      vectors(Ft, own, ks, beta, x);
      v[ks].set(x);
      if (own < live) {
#pragma unroll
        for (int j = 0; j < 8; ++j) dv[(vrow + own) * D + 32 * ks + 8 * g + j] = narrow1<T>(x[j]);
      }
      gradient(own, ks, x);
      o[ks] = exact<T>(x);
    }
    const float into = G.into[own], rest = G.rest[own];
#pragma unroll
    for (int c = 0; c < C::NB; ++c) {
      f32x4_t so = {0.0f, 0.0f, 0.0f, 0.0f}, sv = so, nu = so;
#pragma unroll
      for (int ks = 0; ks < C::KS; ++ks) {
        float x[8];
        Parts<T, kParts> a;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = St[(32 * ks + 8 * g + j) * D + 16 * c + n];
        a.set(x);
        mma_parts<T>(so, a, o[ks]);
        mma_parts<T>(sv, a, v[ks]);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = Nt[(32 * ks + 8 * g + j) * D + 16 * c + n];
        a.set(x);
        mma_parts<T>(nu, a, u[ks]);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        aq[c][r] = fmaf(P.scale * into, so[r], aq[c][r]);
        ak[c][r] = fmaf(rest, nu[r], fmaf(-into, sv[r], ak[c][r]));
      }
    }
    // Pairs of an own token and another of the tile, [others][own].
    const float hi = G.hi[own], lo = G.lo[own];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      float x[8], y[8], z[8];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int b = 2 * kt + half, other = row_of(b, n);
        f32x4_t ou = {0.0f, 0.0f, 0.0f, 0.0f}, uo = ou, vu = ou, uv = ou;
        const float bo = G.beta[other];
#pragma unroll
        for (int ks = 0; ks < C::KS; ++ks) {
          float f[8];
          Parts<T, kParts> a;
          vectors(Et, other, ks, bo, f);
          a.set(f);
          mma_parts<T>(uo, a, o[ks]);
          mma_parts<T>(uv, a, v[ks]);
          vectors(Ft, other, ks, bo, f);
          a.set(f);
          mma_parts<T>(vu, a, u[ks]);
          gradient(other, ks, f);
          mma_parts<T>(ou, exact<T>(f), u[ks]);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int t = row_of(b, 4 * g + r), j = 4 * half + r;
          const float away = (hi - G.hi[t]) + (lo - G.lo[t]);
          const float f = __builtin_amdgcn_exp2f(t <= own ? away : -away);
          x[j] = t <= own ? P.scale * f * uo[r] : 0.0f;
          y[j] = t >= own ? P.scale * f * ou[r] : 0.0f;
          z[j] = t < own ? -f * uv[r] : t > own ? -f * vu[r] : 0.0f;
        }
      }
      Parts<T, kParts> xp, yp, zp;
      xp.set(x);
      yp.set(y);
      zp.set(z);
#pragma unroll
      for (int c = 0; c < C::NB; ++c) {
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = value_at<T>(rk, (32 * kt + 8 * g + j) * D + 16 * c + n);
        const Parts<T, 1> kc = exact<T>(f);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = value_at<T>(rq, (32 * kt + 8 * g + j) * D + 16 * c + n);
        const Parts<T, 1> qc = exact<T>(f);
        mma_parts<T>(aq[c], kc, xp);
        mma_parts<T>(ak[c], kc, zp);
        mma_parts<T>(ak[c], qc, yp);
      }
    }
  }
  if (own >= live) return;
#pragma unroll
  for (int c = 0; c < C::NB; ++c)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t at = (krow + own) * D + 16 * c + 4 * g + r;
      dq[at] = narrow1<T>(aq[c][r]);
      dk[at] = narrow1<T>(ak[c][r]);
    }
}

// The decays' gradient of a span: from that of its first token, <gradient of the state before
// the span, that state>, on.
__global__ void __launch_bounds__(kThreads)
decay_kernel(DeltaPlan P, const int32_t* cu, const float* S0, const float* dS0, const float* recB, const float* recD,
             const float* do_o, const float* dv_v, float* dg) {
  __shared__ double red[2][kThreads / 64];
  const int h = blockIdx.y, lane = threadIdx.x & 63, w = threadIdx.x >> 6, size = P.d * P.d;
  Span sp;
  if (!find_span<kThreads>(P, cu, blockIdx.x, &sp)) return;
  const int64_t pair = (int64_t)sp.s * P.value_heads + h;
  const size_t record = ((size_t)h * P.units + sp.slot) * size;
  const float* a = sp.idx > 0 ? recB + record : S0 ? S0 + pair * size : nullptr;
  const float* b = sp.idx > 0 ? recD + record - size : S0 ? dS0 + pair * size : nullptr;
  double sum = 0.0;
  if (a)
    for (int i = threadIdx.x * 4; i < size; i += kThreads * 4) {
      const f32x4_t x = *reinterpret_cast<const f32x4_t*>(a + i), y = *reinterpret_cast<const f32x4_t*>(b + i);
#pragma unroll
      for (int r = 0; r < 4; ++r) sum += (double)x[r] * (double)y[r];
    }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) red[1][w] = sum;
  __syncthreads();
  double at = 0.0;
  for (int i = 0; i < kThreads / 64; ++i) at += red[1][i];
  const int64_t row = gate_row(P, sp, h);
  for (int t0 = sp.begin, flip = 0; t0 < sp.end; t0 += kThreads, flip ^= 1) {
    const int t = t0 + (int)threadIdx.x;
    const double step = t < sp.end ? (double)dv_v[row + t] - (double)do_o[row + t] : 0.0;
    double c = step;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double x = __shfl_up(c, o);
      if (lane >= o) c += x;
    }
    if (lane == 63) red[flip][w] = c;
    __syncthreads();
    double before = at;
    for (int i = 0; i < kThreads / 64; ++i) {
      if (i < w) before += red[flip][i];
      at += red[flip][i];
    }
    if (t < sp.end) dg[row + t] = (float)(before + (c - step));
  }
}

}  // namespace

gbla_status launch_delta_grads(const DeltaPlan& p, const void* q, const void* k, const float* S0,
                               const int32_t* cu, const void* dout, void* ws, void* dq, void* dk,
                               void* dv, float* dlog_decay, const float* dS0, hipStream_t st) {
  if (p.tokens == 0) return GBLA_OK;
  unsigned char* base = static_cast<unsigned char*>(ws);
  auto floats = [&](size_t off) { return reinterpret_cast<const float*>(base + off); };
  return by_type(p, [&](auto t, auto dim) {
    using T = decltype(t);
    constexpr int D = decltype(dim)::value;
    hipLaunchKernelGGL((grads_kernel<T, D>), dim3(p.tiles, p.heads), dim3(kThreads), 0, st, p, tile_spans(p),
                       (const T*)q, (const T*)k, (const T*)dout, cu, reinterpret_cast<const Gates*>(base + p.off_gates),
                       floats(p.off_S), floats(p.off_N), floats(p.off_E), floats(p.off_F), (T*)dq, (T*)dk, (T*)dv);
    hipLaunchKernelGGL(decay_kernel, dim3(p.grid_units, p.value_heads), dim3(kThreads), 0, st, p, cu, S0, dS0,
                       floats(p.off_B), floats(p.off_D), floats(p.off_do_o), floats(p.off_dv_v), dlog_decay);
  });
}

}  // namespace gbla
