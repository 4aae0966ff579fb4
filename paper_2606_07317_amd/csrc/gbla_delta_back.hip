// gbla_delta_back.hip -- the gated delta rule's backward, from the last tile to the first
// (gfx950): the gradients of u, and of the states.
//
// With N the gradient of the state after a tile, and P, M, c as in the forward
// (gbla_delta.hip; P the tile's scaled and decayed scores):
//   du = P^T do + e^(c_L - c) K N
//   f  = du - M^T (beta du),    dv = beta f
//   N_in = e^c_L N + scale (e^c Q)^T do - (e^c K)^T dv
// which needs nothing of the forward's states.  As there, a wave owns 16 value channels and
// all that one product hands to the next stays in its registers; units run at the same time,
// joined by the transposes of the forward's maps.
//
// Bound by dependent steps at two waves a SIMD (LDS holds keys, queries, gradients, scores and
// triangle: one workgroup a compute unit at heads of 128): the matrix unit works 0.29 of the
// cycles, LDS 0.32.  58000 packed tokens, 8 heads of 128: 333 us, records 222; 8 x 2048 tokens, 16
// heads of 64: 80 and 56.  Barriers for the order of the phases cost 7 %.
//
// All sums here form fp32 results of both signs (the gradients of the gates): everything that
// is computed in fp32 enters its products in three parts.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gbla_delta_tiles.h"

namespace gbla {
namespace {

constexpr int kParts = 3;
template <typename T, int D>
using BackSizes = DS<T, D, D / 16>;

constexpr int kBackWaves = 2;  // a SIMD, that the registers are kept to

struct BackArrays {
  const unsigned char* packs;  // M's transposes and the gates
  float* recD;                 // the gradient of the state after each unit; what it adds (Records)
  float *N, *F, *X;             // X: f's part from the state after the tile
};

// Records: what the unit's own tokens add to the gradient of the state before it, into recD.
template <typename T, int D, bool Records>
__global__ void __launch_bounds__((BackSizes<T, D>::NT), kBackWaves)
back_kernel(DeltaPlan P, const T* q, const T* k, const T* dout, const int32_t* cu, const float* dfinal,
            BackArrays a, float* dS0) {
  using C = BackSizes<T, D>;
  using M = Packed<T, kParts>;
  constexpr bool All = !Records;
  __shared__ __attribute__((aligned(512))) unsigned char ldsK[C::kTileBytes], ldsQ[C::kTileBytes],
      ldsO[C::kTileBytes];
  __shared__ __attribute__((aligned(16))) unsigned char ldsM[M::kBlock], ldsP[M::kBytes];
  const Gates& G = *reinterpret_cast<const Gates*>(ldsM + M::kBytes);
  const int h = blockIdx.y;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Span sp;
  if (!find_span<C::NT>(P, cu, blockIdx.x, &sp)) return;
  if (Records && sp.idx == 0) return;  // nothing comes before it
  const int64_t pair = (int64_t)sp.s * P.value_heads + h;
  const int e0 = 16 * w;
  const size_t record = ((size_t)h * P.units + sp.slot) * (D * D);
  Columns16<T, C> N;
  if (Records) N.fill(0.0f);
  else if (!P.single && (dfinal || !sp.last)) N.load_record(a.recD + record, e0, lane);
  else if (dfinal) N.load(dfinal + pair * (D * D), e0, lane);
  else N.fill(0.0f);

  const int64_t krow = first_row(P, sp, P.heads, h / P.group), vrow = first_row(P, sp, P.value_heads, h);
  const size_t slot0 = (size_t)h * P.tiles + tile_slot(P, sp.row0, sp.s);
  RowsLoad<T, C> lk, lq, lo;
  BlockLoad<C, M::kBlock> lm;
  auto fetch = [&](int t) {  // (none before the unit's first tile)
    const int left = t < sp.begin ? 0 : sp.end - t;
    const int64_t row = max(t, 0);
    lk.load(k + (krow + row) * D, left);
    lq.load(q + (krow + row) * D, left);
    lo.load(dout + (vrow + row) * D, left);
    lm.load(a.packs + (slot0 + row / kDeltaTile) * M::kBlock, left > 0);
  };
  const int last = sp.begin < sp.end ? sp.begin + (sp.end - 1 - sp.begin) / kDeltaTile * kDeltaTile : sp.begin - 1;
  if (sp.begin < sp.end) fetch(last);
  for (int t0 = last; t0 >= sp.begin; t0 -= kDeltaTile) {
    const size_t slot = slot0 + t0 / kDeltaTile;
    lk.store(ldsK);
    lq.store(ldsQ);
    lo.store(ldsO);
    lm.store(ldsM);
    lds_barrier();
    // Scores [later tokens][own earlier token] as operands for all waves.
    {
      constexpr int NP = C::NW < 4 ? 4 / C::NW : 1, PG = C::NW == 8 ? 1 : 2;
      const int pg0 = C::NW == 8 ? w >> 2 : 0;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int b = (w + C::NW * i) & 3, s = row_of(b, n);
        f32x4_t p[2 * PG];
#pragma unroll
        for (int j = 0; j < 2 * PG; ++j) p[j] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int ks = 0; ks < C::KS; ++ks) {
          const auto own = row_units<T, C>(ldsK, s, ks, g);
#pragma unroll
          for (int j = 0; j < 2 * PG; ++j) Num<T>::mma(p[j], row_units<T, C>(ldsQ, row_of(2 * pg0 + j, n), ks, g), own);
        }
#pragma unroll
        for (int z = 0; z < PG; ++z) {
          const int ks = pg0 + z;
          float y[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = p[2 * z + (j >> 2)][j & 3];
          decayed<false>(G, s, 32 * ks + 8 * g, P.scale, y);
          Parts<T, kParts> parts;
          split(parts, y);
          if (ks == 1 || b < 2) M::put(ldsP, upper_pair(b, ks), lane, parts);
        }
      }
    }
    // The gradient of u: from the states after the tile, from the tile's outputs; f is that
    // without the tile's later ones.
    f32x4_t x[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) x[b] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) {
      const Parts<T, kParts> s = N.template operand<kParts>(ks);
      if constexpr (All) store_columns<T, C>(a.N + slot * (D * D), ks, e0, lane, s);
      typename Num<T>::V8 kk[4];
#pragma unroll
      for (int b = 0; b < 4; ++b) kk[b] = row_units<T, C>(ldsK, row_of(b, n), ks, g);
#pragma unroll
      for (int i = Parts<T, kParts>::kN - 1; i >= 0; --i)
#pragma unroll
        for (int b = 0; b < 4; ++b) Num<T>::mma(x[b], kk[b], s.v[i]);
    }
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) x[b][r] *= G.rest[row_of(b, 4 * g + r)];
    auto put = [&](float* m) {
#pragma unroll
      for (int b = 0; b < 4; ++b)
        *reinterpret_cast<f32x4_t*>(m + (slot * D + e0 + n) * kDeltaTile + row_of(b, 4 * g)) = x[b];
    };
    if constexpr (All) put(a.X);
    lds_barrier();  // the scores
    {
      typename Num<T>::V8 o[2];
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) o[ks] = value_column<T, C>(ldsO, w, ks, lane);
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int ks = b >> 1; ks < 2; ++ks) {
          const Parts<T, kParts> y = M::get(ldsP, upper_pair(b, ks), lane);
#pragma unroll
          for (int i = Parts<T, kParts>::kN - 1; i >= 0; --i) Num<T>::mma(x[b], y.v[i], o[ks]);
        }
      Parts<T, kParts> y[2];
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        float z[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = G.beta[32 * ks + 8 * g + j] * x[2 * ks + (j >> 2)][j & 3];
        split(y[ks], z);
      }
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int ks = b >> 1; ks < 2; ++ks) mma_parts<T>(x[b], M::get(ldsM, upper_pair(b, ks), lane), y[ks]);
    }
    if constexpr (All) put(a.F);
    fetch(t0 - kDeltaTile);
    {
      Parts<T, kParts> up[2], down[2];
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        float z[8];
        Num<T>::widen(value_column<T, C>(ldsO, w, ks, lane), z);
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] *= P.scale * G.into[32 * ks + 8 * g + j];
        split(up[ks], z);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int t = 32 * ks + 8 * g + j;
          z[j] = -G.into[t] * (G.beta[t] * x[2 * ks + (j >> 2)][j & 3]);
        }
        split(down[ks], z);
      }
      const float whole = G.whole;
#pragma unroll
      for (int i = 0; i < C::NB; ++i) {
        f32x4_t z = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
          const auto kc = key_column<T, C>(ldsK, i, kt, lane), qc = key_column<T, C>(ldsQ, i, kt, lane);
#pragma unroll
          for (int j = Parts<T, kParts>::kN - 1; j >= 0; --j) {
            Num<T>::mma(z, kc, down[kt].v[j]);
            Num<T>::mma(z, qc, up[kt].v[j]);
          }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) N.s[i][r] = fmaf(whole, N.s[i][r], z[r]);
      }
    }
    lds_barrier();
  }
  if (Records) N.store_record(a.recD + record, e0, lane);
  else if (dS0 && sp.idx == 0) N.store(dS0 + pair * (D * D), e0, lane);
}

BackArrays arrays(const DeltaPlan& p, void* ws) {
  unsigned char* base = static_cast<unsigned char*>(ws);
  auto floats = [&](size_t off) { return reinterpret_cast<float*>(base + off); };
  return {base + p.off_packT, floats(p.off_D), floats(p.off_N),
          floats(p.off_F), floats(p.off_E)};
}

}  // namespace

gbla_status launch_delta_back_records(const DeltaPlan& p, const void* q, const void* k, const int32_t* cu,
                                      const void* dout, void* ws, hipStream_t st) {
  if (p.single) return GBLA_OK;
  return by_type(p, [&](auto t, auto dim) {
    using T = decltype(t);
    constexpr int D = decltype(dim)::value;
    hipLaunchKernelGGL((back_kernel<T, D, true>), dim3(p.grid_units, p.value_heads), dim3((BackSizes<T, D>::NT)), 0,
                       st, p, (const T*)q, (const T*)k, (const T*)dout, cu, (const float*)nullptr,
                       arrays(p, ws), (float*)nullptr);
  });
}

gbla_status launch_delta_back_walk(const DeltaPlan& p, const void* q, const void* k, const int32_t* cu,
                                   const void* dout, const float* dfinal, void* ws, float* dS0,
                                   hipStream_t st) {
  return by_type(p, [&](auto t, auto dim) {
    using T = decltype(t);
    constexpr int D = decltype(dim)::value;
    hipLaunchKernelGGL((back_kernel<T, D, false>), dim3(p.grid_units, p.value_heads), dim3((BackSizes<T, D>::NT)), 0,
                       st, p, (const T*)q, (const T*)k, (const T*)dout, cu, dfinal, arrays(p, ws), dS0);
  });
}

}  // namespace gbla
