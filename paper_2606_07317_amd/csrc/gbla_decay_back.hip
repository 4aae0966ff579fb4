// gbla_decay_back.hip -- the decay attention's backward: gradients of the keys, the
// values, the decay and the initial state (gfx950).
//
// With D the gradient of the state after a tile of L tokens:
//   dk_s = sum_{t >= s} scale lam^(t-s) (do_t v_s) q_t + lam^(L-1-s) D v_s
//   dv_s = sum_{t >= s} scale lam^(t-s) (q_t k_s) do_t + lam^(L-1-s) D^T k_s
//   D_in = lam^L D + scale sum_t lam^(t+1) q_t do_t^T
// summed over the query heads that share the key head.  A workgroup walks its unit's
// tiles from the last to the first with D in registers; wave w owns tokens
// 16 (w & 3) .. as keys.  Scores are [queries] x [own keys], whose results are the
// second products' operands as they lie.
//
// The decay's gradient is a sum over pairs of an earlier token s and a later one t
// (the initial state counts as token -1, the final one as the last token), each
// weighed with their distance.  It is taken apart so that no term is a difference of
// large sums over the sequence:
//   both in one tile:           (t - s) score_ts (do_t v_s)
//   s before t's tile:          (t + 1) q_t dq_t, the dq of the state (walk_kernel)
//   t after s's tile:           (L - 1 - s) k_s dk_s, the dk of D
//   tiles passed in between:    L times the pairs that pass the tile; counted from
//     the pairs <S_in, D_in> that enter the tile's unit, less what q_t dq_t of the
//     unit's tiles up to this one take out, plus what k_s dk_s of its tiles before
//     this one bring in.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gbla_decay_tiles.h"

namespace gbla {
namespace {

template <typename T, int D>
__global__ void __launch_bounds__((DC<T, D>::NT), 1)
keys_kernel(DecayPlan P, const T* q, const T* k, const T* v, const float* log_decay,
            const float* S0, const int32_t* cu, const T* dout, const float* dfinal,
            const float* recS, const float* recD, T* dk, T* dv, float* dS0, double* dg) {
  using C = DC<T, D>;
  __shared__ __attribute__((aligned(16))) unsigned char ldsQ[C::kTileBytes], ldsO[C::kTileBytes],
      ldsD[C::NP * C::kPlane];
  const int h = blockIdx.y, lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4, tw = w & 3, eh = w >> 2;
  Span sp;
  double dsum = 0.0;
  const bool found = find_span<C::NT>(P, cu, blockIdx.x, &sp);
  if (found) {
    const int64_t pair = (int64_t)sp.s * P.kv_heads + h;
    const float* init;  // the gradient of the state after the span
    const float* kept;  // the states before its units, [column of S][row] as dq's walk has them
    if (P.single) {
      init = dfinal ? dfinal + pair * (D * D) : nullptr;
      kept = recS + ((size_t)h * P.units + (P.ragged ? sp.row0 / P.unit + sp.s
                                                     : (int64_t)sp.s * P.units_per_seq)) * (D * D);
    } else {
      const size_t at = ((size_t)h * P.units + sp.slot) * (D * D);
      init = dfinal || !sp.last ? recD + at : nullptr;
      kept = recS + at;
    }
    State<T, C> S, add;
    if (init) S.load(init, false, w, lane);
    else S.clear();
    bool some = init != nullptr;

    const int tiles = (sp.end - sp.begin + kTile - 1) / kTile;
    TileLoad<C> lq, lo;
    OwnRows<T, C> kf, vf;
    auto fetch = [&](int t, int gi) {
      const int64_t row = row_of(P, sp, P.heads, h * P.group + gi, t) * D;
      lq.load(q + row, sp.end - t);
      lo.load(dout + row, sp.end - t);
    };
    if (tiles > 0) fetch(sp.begin + (tiles - 1) * kTile, 0);
    const Decay lam(log_decay[h]);
    const float full = lam(kTile);
    float score[4][4], weight[2][8];
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) score[b][i] = P.scale * lam(max(0, 16 * (b - tw) + 4 * g + i - n));
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int j = 0; j < 8; ++j) weight[ks][j] = P.scale * lam(32 * ks + 8 * g + j + 1);

    for (int tile = tiles - 1; tile >= 0; --tile) {
      const int t0 = sp.begin + tile * kTile, live = min(kTile, sp.end - t0);
      const int64_t krow = row_of(P, sp, P.kv_heads, h, t0) * D;
      kf.load(k + krow, live, 16 * tw + n, g);
      vf.load(v + krow, live, 16 * tw + n, g);
      f32x4_t ak[C::OB], av[C::OB];
#pragma unroll
      for (int o = 0; o < C::OB; ++o) ak[o] = av[o] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
      float inner = 0.0f;
      add.clear();
      for (int gi = 0; gi < P.group; ++gi) {
        lq.store(ldsQ);
        lo.store(ldsO);
        if (gi == 0 && some) S.to_planes(ldsD, w, lane);
        lds_barrier();
        if (gi + 1 < P.group) fetch(t0, gi + 1);
        else if (tile > 0) fetch(t0 - kTile, 0);
        if (gi == 0 && some) {
          // D^T k by rows of the planes [column][row], D v by their columns
#pragma unroll
          for (int ks = 0; ks < C::KS; ++ks)
#pragma unroll
            for (int x = C::NP - 1; x >= 0; --x)
#pragma unroll
              for (int o = 0; o < C::OB; ++o) {
                const int blk = eh * C::OB + o;
                Num<T>::mma(av[o], row_at<T, C>(ldsD + x * C::kPlane, 16 * blk + n, ks, g), kf.v[ks]);
                Num<T>::mma(ak[o], col_at<T, C, false>(ldsD + x * C::kPlane, blk, ks, lane), vf.v[ks]);
              }
          const float out = lam(max(0, live - 1 - 16 * tw - n));
#pragma unroll
          for (int o = 0; o < C::OB; ++o)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              ak[o][r] *= out;
              av[o][r] *= out;
            }
          if (dg && 16 * tw + n < live) {
            const T* k4 = k + krow + (int64_t)(16 * tw + n) * D + 16 * eh * C::OB + 4 * g;
            float dot = 0.0f;
#pragma unroll
            for (int o = 0; o < C::OB; ++o)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const float x = sizeof(T) == 2 ? __uint_as_float((uint32_t)k4[16 * o + r] << 16)
                                               : (float)k4[16 * o + r];
                dot = fmaf(x, ak[o][r], dot);
              }
            // tokens of the unit after token s
            const int at = (t0 - sp.begin) % P.unit;
            const int size = min(P.unit, sp.end - (t0 - at));
            dsum += (double)dot * (double)(size - 1 - at - 16 * tw - n);
          }
        }
        float px[4][4], py[4][4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          f32x4_t x = {0.0f, 0.0f, 0.0f, 0.0f}, y = {0.0f, 0.0f, 0.0f, 0.0f};
          if (b >= tw) {
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks) {
              Num<T>::mma(x, row_at<T, C>(ldsQ, 16 * b + n, ks, g), kf.v[ks]);
              Num<T>::mma(y, row_at<T, C>(ldsO, 16 * b + n, ks, g), vf.v[ks]);
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bool in = b > tw || (b == tw && 4 * g + i >= n);
            px[b][i] = in ? x[i] * score[b][i] : 0.0f;
            py[b][i] = in ? y[i] * score[b][i] : 0.0f;
            if (dg && in && eh == 0)
              inner = fmaf(px[b][i] * y[i], (float)(16 * (b - tw) + 4 * g + i - n), inner);
          }
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          if (2 * ks + 1 < tw) continue;
          const float x[8] = {px[2 * ks][0],     px[2 * ks][1],     px[2 * ks][2],     px[2 * ks][3],
                              px[2 * ks + 1][0], px[2 * ks + 1][1], px[2 * ks + 1][2], px[2 * ks + 1][3]};
          const float y[8] = {py[2 * ks][0],     py[2 * ks][1],     py[2 * ks][2],     py[2 * ks][3],
                              py[2 * ks + 1][0], py[2 * ks + 1][1], py[2 * ks + 1][2], py[2 * ks + 1][3]};
          Parts<T, 2> xx, yy;
          xx.set(x);
          yy.set(y);
#pragma unroll
          for (int o = 0; o < C::OB; ++o) {
            xx.mma_right(av[o], col_at<T, C, true>(ldsO, eh * C::OB + o, ks, lane));
            yy.mma_right(ak[o], col_at<T, C, true>(ldsQ, eh * C::OB + o, ks, lane));
          }
        }
        add.add_products(ldsQ, ldsO, weight, w, lane);
        lds_barrier();
      }
      S.advance(live == kTile ? full : lam(live), add);
      some = true;
      dsum += (double)inner;
      const __amdgpu_buffer_rsrc_t rk = make_rsrc(dk + krow, (uint32_t)(live * C::kRow));
      const __amdgpu_buffer_rsrc_t rv = make_rsrc(dv + krow, (uint32_t)(live * C::kRow));
      const uint32_t at = (uint32_t)((16 * tw + n) * C::kRow + (16 * eh * C::OB + 4 * g) * C::ES);
#pragma unroll
      for (int o = 0; o < C::OB; ++o) {
        if constexpr (sizeof(T) == 2) {
          const u32x2_t a = {pack_bf16x2(ak[o][0], ak[o][1]), pack_bf16x2(ak[o][2], ak[o][3])};
          const u32x2_t b = {pack_bf16x2(av[o][0], av[o][1]), pack_bf16x2(av[o][2], av[o][3])};
          __builtin_amdgcn_raw_buffer_store_b64(a, rk, at + 16 * o * C::ES, 0, 0);
          __builtin_amdgcn_raw_buffer_store_b64(b, rv, at + 16 * o * C::ES, 0, 0);
        } else {
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, ak[o]), rk, at + 16 * o * C::ES, 0, 0);
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, av[o]), rv, at + 16 * o * C::ES, 0, 0);
        }
      }
      if (dg && (t0 - sp.begin) % P.unit == 0) {  // the unit's first tile: <S_in, D_in>
        const int unit = (t0 - sp.begin) / P.unit;
        const int size = min(P.unit, sp.end - t0);
        if (S0 || sp.idx + unit > 0) {
          add.load(kept + (int64_t)unit * (D * D), true, w, lane);
          float dot = 0.0f;
#pragma unroll
          for (int i = 0; i < C::SB; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) dot = fmaf(add.s[i][r], S.s[i][r], dot);
          dsum += (double)dot * (double)size;
        }
      }
    }
    if (dS0 && sp.begin == 0) S.store(dS0 + pair * (D * D), false, w, lane);
  }
  if (dg) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) dsum += __shfl_xor(dsum, o);
    if (lane == 0) dg[((int64_t)h * P.grid_units + blockIdx.x) * 8 + w] = dsum;
  }
}

// The sum of a key head's parts: [2][K][grid_units][8] doubles, `waves` of each 8
// in use.
__global__ void __launch_bounds__(kThreads)
decay_sum_kernel(int kv_heads, int units, int waves, const double* dg, float* out) {
  __shared__ double red[kThreads];
  const int h = blockIdx.x;
  double sum = 0.0;
  for (int half = 0; half < 2; ++half) {
    const double* p = dg + ((int64_t)half * kv_heads + h) * units * 8;
    for (int i = threadIdx.x; i < units * waves; i += kThreads) sum += p[(int64_t)(i / waves) * 8 + i % waves];
  }
  red[threadIdx.x] = sum;
  __syncthreads();
  for (int o = kThreads / 2; o > 0; o >>= 1) {
    if ((int)threadIdx.x < o) red[threadIdx.x] += red[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) out[h] = (float)red[0];
}

template <typename T, int D>
void launch_keys(const DecayPlan& p, const void* q, const void* k, const void* v, const float* log_decay,
                 const float* S0, const int32_t* cu, const void* dout, const float* dfinal,
                 unsigned char* ws, void* dk, void* dv, float* dlog_decay, float* dS0, hipStream_t st) {
  double* dg = dlog_decay ? reinterpret_cast<double*>(ws + p.off_dg) : nullptr;
  double* mine = dg ? dg + (int64_t)p.kv_heads * p.grid_units * 8 : nullptr;
  hipLaunchKernelGGL((keys_kernel<T, D>), dim3(p.grid_units, p.kv_heads), dim3(DC<T, D>::NT), 0, st, p,
                     (const T*)q, (const T*)k, (const T*)v, log_decay, S0, cu, (const T*)dout, dfinal,
                     reinterpret_cast<const float*>(ws + p.off_S),
                     reinterpret_cast<const float*>(ws + p.off_D), (T*)dk, (T*)dv, dS0, mine);
  if (dg)
    hipLaunchKernelGGL(decay_sum_kernel, dim3(p.kv_heads), dim3(kThreads), 0, st, p.kv_heads,
                       p.grid_units, DC<T, D>::NW, dg, dlog_decay);
}

}  // namespace

gbla_status launch_decay_keys(const DecayPlan& p, const void* q, const void* k, const void* v,
                              const float* log_decay, const float* S0, const int32_t* cu,
                              const void* dout, const float* dfinal, void* ws, void* dk, void* dv,
                              float* dlog_decay, float* dS0, hipStream_t st) {
  unsigned char* base = static_cast<unsigned char*>(ws);
#define GBLA_KEYS(T, D)                                                                          \
  launch_keys<T, D>(p, q, k, v, log_decay, S0, cu, dout, dfinal, base, dk, dv, dlog_decay, dS0, st)
  const bool half = p.dtype == GBLA_BF16;
  if (p.d == 32) {
    if (half) GBLA_KEYS(uint16_t, 32);
    else GBLA_KEYS(float, 32);
  } else if (p.d == 64) {
    if (half) GBLA_KEYS(uint16_t, 64);
    else GBLA_KEYS(float, 64);
  } else {
    if (half) GBLA_KEYS(uint16_t, 128);
    else GBLA_KEYS(float, 128);
  }
#undef GBLA_KEYS
  return hipGetLastError() == hipSuccess ? GBLA_OK : GBLA_ERR_HIP;
}

}  // namespace gbla
