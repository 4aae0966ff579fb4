// gbla_delta.hip -- the gated delta rule in chunks (gfx950): the forward.
//
//   u_t = beta_t (v_t - e^g_t S_{t-1}^T k_t),  S_t = e^g_t S_{t-1} + k_t u_t^T,  o_t = scale S_t^T q_t
// over a tile of L <= 64 tokens with the state S before it, c the sum of g from the tile's
// start, L_ts = e^(c_t - c_s) k_t k_s (s < t) and (I + L beta) M = L:
//   y_t = v_t - e^c_t S^T k_t,   e = y - M (beta y),   u = beta e
//   o_t = scale (e^c_t S^T q_t + sum_{s <= t} e^(c_t - c_s) (q_t k_s) u_s)
//   S_out = e^c_L S + sum_s e^(c_L - c_s) k_s u_s^T
// (e_t is what the token's value differs from the state's prediction.)  Every exponent is
// <= 0, so strong decays underflow to 0 and nothing overflows, and nothing is divided by
// beta.
//
// M depends on keys and gates alone: a first launch (prep_kernel) forms it for all tiles at
// once, and the walks read it as operands.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gbla_delta_tiles.h"

namespace gbla {
namespace {

// Three parts of what the state is made of, so that it keeps fp32's accuracy (with two its
// error was 3e-6 of its norm); two of what only the output takes, 2^-16 of a term, below its
// own bf16 rounding.
constexpr int kParts = 3, kOutParts = 2;

// log2 of a token's decay in 64 bits; -inf (and so low that exp is 0 many times over) stays
// finite, so that differences of sums do.
__device__ __forceinline__ double log2_decay(float g) {
  return (double)(g < -1e5f ? -1e5f : g) * 1.4426950408889634074;
}

// A tile's gates and its M.  A wave takes 16 columns of the tile; which, goes around from
// workgroup to workgroup, as the first have the most rows below them.  M is formed by blocks of
// 16 rows, from the first on: with X = (I + L_ii beta)^-1, by substitution (one wave's sixteen
// lanes a block),
//   M_ij = X (L_ij - sum_{j <= m < i} (L_im beta) M_mj)
// in fp32 products, whose results are the next one's operands as they lie.  (Powers of L
// beta would need fewer steps, but cancel: binomial coefficients, where keys are alike.)
// packsT (backward): M's transpose too.
//
// Bound by the issue of its instructions, of which the substitution and the split into parts
// are the most (vector instructions take 0.44 to 0.58 of the cycles, five workgroups a compute
// unit).  32768 tokens, 8 heads of 64: 33 us; 178000 packed tokens, 8 heads of 128: 188 us, 20 KB
// written a tile at 2.4 TB/s.  (All waves substituting for their own block, keys beside L in LDS
// and four workgroups: 42 and 290 us.)
template <typename T, int D>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 5 : 3)
prep_kernel(DeltaPlan P, TileSpans tiles, const T* k, const float* log_decay, const float* beta,
            const int32_t* cu, unsigned char* packs, unsigned char* packsT) {
  using C = DS<T, D, 4>;
  constexpr int kL = 68;  // floats of a row of L
  // the keys; once multiplied, L beta and then M in their place
  __shared__ __attribute__((aligned(512))) unsigned char ldsK[C::kTileBytes > kDeltaTile * kL * 4 ? C::kTileBytes : kDeltaTile * kL * 4];
  __shared__ __attribute__((aligned(16))) float ldsX[4][16][20];
  float (*ldsL)[kL] = reinterpret_cast<float (*)[kL]>(ldsK);
  __shared__ __attribute__((aligned(16))) Gates G;
  __shared__ int bad;
  Span sp;
  if (!find_span<C::NT>(tiles, cu, blockIdx.x, &sp)) return;
  const int h = blockIdx.y, lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(((threadIdx.x >> 6) + blockIdx.x) & 3);
  const int live = sp.end - sp.begin;
  RowsLoad<T, C> lk;
  lk.load(k + (first_row(P, sp, P.heads, h / P.group) + sp.begin) * D, live);
  const int64_t at = gate_row(P, sp, h) + sp.begin;
  float gt = 0.0f, bt = 0.0f;
  if (w == 0 && lane < live) gt = log_decay[at + lane], bt = beta[at + lane];
  if (threadIdx.x == 0) bad = live;
  __syncthreads();
  if (w == 0 && lane < live && (!(gt <= 3.0e38f) || !isfinite(bt))) atomicMin(&bad, lane);
  lk.find_bad(&bad);
  lk.store(ldsK);
  __syncthreads();
  const int good = bad;
  if (good < live) {
    clear_rows<C>(ldsK, good);
    __syncthreads();
  }
  if (w == 0) {
    double c = lane < good ? log2_decay(gt) : 0.0;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double x = __shfl_up(c, o);
      if (lane >= o) c += x;
    }
    const double end = __shfl(c, 63);
    const float hi = (float)c;
    G.hi[lane] = hi;
    G.lo[lane] = (float)(c - (double)hi);
    G.beta[lane] = lane < good ? bt : 0.0f;
    G.into[lane] = __builtin_amdgcn_exp2f(hi) * fmaf((float)(c - (double)hi), 0.69314718f, 1.0f);
    const float rest = __builtin_amdgcn_exp2f((float)(end - c));
    G.rest[lane] = rest;
    G.late[lane] = lane < good ? rest * bt : 0.0f;
    if (lane == 63) G.whole = G.into[63], G.good = good;
    if (lane < 62) G.pad[lane] = 0.0f;
  }
  f32x4_t x[4];  // L's rows 16 b + 4 g + r of the wave's column n; then M's
#pragma unroll
  for (int b = 0; b < 4; ++b) x[b] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int ks = 0; ks < C::KS; ++ks) {
    const auto own = row_units<T, C>(ldsK, 16 * w + n, ks, g);
#pragma unroll
    for (int b = 0; b < 4; ++b)
      if (b >= w) Num<T>::mma(x[b], row_units<T, C>(ldsK, 16 * b + n, ks, g), own);
  }
  __syncthreads();
  {
    const int s = 16 * w + n;
    const float hi = G.hi[s], lo = G.lo[s], strength = -G.beta[s];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      if (b < w) continue;
      const int t0 = 16 * b + 4 * g;
      const f32x4_t h4 = *reinterpret_cast<const f32x4_t*>(&G.hi[t0]), l4 = *reinterpret_cast<const f32x4_t*>(&G.lo[t0]);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float y = x[b][r] * __builtin_amdgcn_exp2f((h4[r] - hi) + (l4[r] - lo));
        x[b][r] = t0 + r > s ? y : 0.0f;
        ldsL[t0 + r][s] = strength * x[b][r];
      }
    }
  }
  __syncthreads();
  // X of the diagonal blocks: lane n of group g column n of block g, row after row.
  if (w == 3) {
    float y[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float sum = n == i ? 1.0f : 0.0f;
#pragma unroll
      for (int s4 = 0; s4 < i; s4 += 4) {
        const f32x4_t z = *reinterpret_cast<const f32x4_t*>(&ldsL[16 * g + i][16 * g + s4]);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (s4 + j < i) sum = fmaf(z[j], y[s4 + j], sum);
      }
      y[i] = sum;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) ldsX[g][i][n] = y[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i < w) continue;
#pragma unroll
    for (int j = 0; j < i; ++j) {
      if (j < w) continue;
      const f32x4_t a = *reinterpret_cast<const f32x4_t*>(&ldsL[16 * i + n][16 * j + 4 * g]);
#pragma unroll
      for (int r = 0; r < 4; ++r) x[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[r], x[j][r], x[i], 0, 0, 0);
    }
    const f32x4_t inv = *reinterpret_cast<const f32x4_t*>(&ldsX[i][n][4 * g]);
    f32x4_t m = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int r = 0; r < 4; ++r) m = __builtin_amdgcn_mfma_f32_16x16x4f32(inv[r], x[i][r], m, 0, 0, 0);
    x[i] = m;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) ldsL[16 * i + 4 * g + r][16 * w + n] = -x[i][r];
  __syncthreads();
  const size_t slot = (size_t)h * P.tiles + sp.slot;
  using Pack = Packed<T, kParts>;
  unsigned char* pack = packs + slot * Pack::kBlock;
  for (int pair = w; pair < 6; pair += 4) {
    const int b = pair < 2 ? pair : 2 + (pair >> 2), ks = pair < 2 ? 0 : pair & 1;
    const f32x4_t* p = reinterpret_cast<const f32x4_t*>(&ldsL[row_of(b, n)][32 * ks + 8 * g]);
    const f32x4_t a = p[0], c = p[1];
    const float z[8] = {a[0], a[1], a[2], a[3], c[0], c[1], c[2], c[3]};
    Parts<T, kParts> parts;
    split(parts, z);
    Pack::put(pack, pair, lane, parts);
  }
  auto put_gates = [&] {
    if (threadIdx.x < kGateBytes / 16)
      reinterpret_cast<u32x4_t*>(pack + Pack::kBytes)[threadIdx.x] = reinterpret_cast<const u32x4_t*>(&G)[threadIdx.x];
  };
  put_gates();
  if (packsT) {
    pack = packsT + slot * Pack::kBlock;
    put_gates();
    for (int pair = w; pair < 6; pair += 4) {
      const int b = pair < 4 ? pair >> 1 : pair - 2, ks = pair < 4 ? pair & 1 : 1;
      float z[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] = ldsL[32 * ks + 8 * g + j][row_of(b, n)];
      Parts<T, kParts> parts;
      split(parts, z);
      Pack::put(pack, pair, lane, parts);
    }
  }
}

// What walk_kernel makes: outputs; a unit's records, which are what the unit adds to the state
// (from zeros) and what it does to the state before it (from the identity, without values);
// or what the backward needs of the forward, the strengths' gradient, and what of the decays' ends
// at each token from the state before its tile, or begins there for the state after it
// (gbla_delta_grads.hip).  The last forms no scores.
//
// A wave holds 16 value channels of the state, so that a tile's products follow one another in
// its registers; only the scores, which all waves need, go through LDS.  The matrix unit, vector
// instructions (the splits into parts) and reads of operands from LDS take 0.4 to 0.6 of the
// cycles each, and dependent steps between barriers the rest: 0.46 and 0.48 of the matrix unit
// at 178000 packed tokens, 8 heads of 128 (outputs 695 us, records 719), 0.28 and 0.37 at 32768
// tokens, 8 heads of 64 (57 us each).  Without any loads of a later tile
// the records take 681.  Two column blocks a wave, which halve the reads of LDS, took as long (half the
// waves); scores in the place of the values, for a third workgroup at heads of 64, as well.
enum WalkMode { kOutputs, kRecords, kBack };
template <typename T, int D>
using WalkSizes = DS<T, D, D / 16>;
// Waves a SIMD that the registers are kept to.
template <typename T, int D, WalkMode Mode>
constexpr int kWalkWaves = sizeof(T) == 4 || D == 32 || Mode == kBack ? 2 : 4;
struct BackOut {
  const void* dout;
  const float* F;  // the gradient of u
  float* S;
  float* E;        // holds F's part from the state after the tile, which e takes the place of
  float *from, *on, *dbeta;
  float* M;           // the maps for the gradients' scan
  bool final_gradient;  // the final state has one
};

template <typename T, int D, WalkMode Mode>
__global__ void __launch_bounds__((WalkSizes<T, D>::NT), (kWalkWaves<T, D, Mode>))
walk_kernel(DeltaPlan P, const T* q, const T* k, const T* v, const float* S0, const int32_t* cu,
            const unsigned char* packs, float* recB, float* recM, T* out,
            float* final_state, BackOut back) {
  using C = WalkSizes<T, D>;
  // Back, what is formed from the outputs are sums of both signs in fp32.
  constexpr int kOut = Mode == kBack ? 3 : kOutParts;
  using M = Packed<T, kParts>;
  using Pk = Packed<T, kOut>;
  constexpr bool Out = Mode != kRecords, Back = Mode == kBack, Scores = Mode == kOutputs;
  __shared__ __attribute__((aligned(512))) unsigned char ldsK[C::kTileBytes], ldsV[C::kTileBytes],
      ldsQ[Out ? C::kTileBytes : 16];
  __shared__ __attribute__((aligned(16))) unsigned char ldsM[M::kBytes], ldsP[Scores ? Pk::kBytes : 16];
  __shared__ __attribute__((aligned(16))) Gates G;
  __shared__ int bad[2];  // of this tile and the next
  __shared__ float sums[Back ? 4 : 1][Back ? C::NW : 1][kDeltaTile];
  const int h = blockIdx.y;
  int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Span sp;
  if (!find_span<C::NT>(P, cu, blockIdx.x, &sp)) return;
  const int64_t pair = (int64_t)sp.s * P.value_heads + h;
  const int e0 = 16 * w;  // the wave's first column
  Columns16<T, C> S;
  const size_t record = ((size_t)h * P.units + sp.slot) * (D * D);
  const bool map = !Out && blockIdx.z == 1;
  if (!Out) {
    // The scan passes over all units but the last; its first has no map where it starts from
    // zeros.  The backward's scan, which takes the maps too, begins with the last unit.
    const bool there = !sp.last && (!map || sp.idx > 0 || S0);
    const bool back_too = map && back.dout && sp.idx > 0 && (!sp.last || back.final_gradient);
    if (!there && !back_too) return;
    if (map) S.identity(e0, lane);
    else S.fill(0.0f);
  } else {
    if (!P.single && (S0 || sp.idx > 0)) S.load_record(recB + record, e0, lane);
    else if (S0) S.load(S0 + pair * (D * D), e0, lane);
    else S.fill(0.0f);
  }

  const int64_t krow = first_row(P, sp, P.heads, h / P.group), vrow = first_row(P, sp, P.value_heads, h);
  const size_t slot0 = (size_t)h * P.tiles + tile_slot(P, sp.row0, sp.s);
  // The next tile on its way: keys, queries and gates, whose places in LDS are read to a tile's
  // end, through registers; values and the triangle, which are done with before the outputs,
  // straight into theirs (fp32, whose rows there are padded: through registers too).
  constexpr bool kDirect = sizeof(T) == 2;
  RowsLoad<T, C> lk, lq, lv;
  BlockLoad<C, M::kBytes> lm;
  BlockLoad<C, kGateBytes> lg;
  const uint32_t atV = lds_address(ldsV), atM = lds_address(ldsM);
  // Outputs at four waves a SIMD hold too much to have keys, queries and gates under way from a
  // tile's start (spilled registers: 833 us for 178000 packed tokens, 8 heads of 128; from before
  // the outputs on 779, behind them 729.  Heads of 64 the other way round: 58 and 59).
  constexpr bool kLate = Mode == kOutputs && kWalkWaves<T, D, Mode> > 2 && D == 128;
  auto fetch = [&](int t) {
    lk.load(k + (krow + t) * D, sp.end - t);
    if (Out) lq.load(q + (krow + t) * D, sp.end - t);
    lg.load(packs + (slot0 + t / kDeltaTile) * M::kBlock + M::kBytes, sp.end - t > 0);
  };
  auto fetch_direct = [&](int t) {
    const int left = sp.end - t;
    const T* vt = v + (vrow + t) * D;
    const unsigned char* mt = packs + (slot0 + t / kDeltaTile) * M::kBlock;
    if constexpr (kDirect) {
      rows_to_lds<T, C>(atV, vt, map ? 0 : left, w, fresh(lane));
      block_to_lds<C, M::kBytes>(atM, mt, left > 0, w, fresh(lane));
    } else {
      lv.load(vt, map ? 0 : left);
      lm.load(mt, left > 0);
    }
  };
  if (sp.begin < sp.end) {
    fetch(sp.begin);
    fetch_direct(sp.begin);
  }
  if (threadIdx.x == 0) bad[0] = kDeltaTile;
  __syncthreads();
  // Where four waves a SIMD share the registers, phases do not mix, and addresses in LDS, which
  // cost registers held over the loop, are worked out in each.  (Elsewhere it takes longer: backward,
  // 8 x 2048 tokens, 16 heads of 64 96 us without it, 100 with; 58000 tokens, 8 heads of 128 409, 429;
  // forward, 8 x 4096 tokens, 8 heads of 32 100.5, 102.7.)
  auto again = [&] {
    if constexpr (kWalkWaves<T, D, Mode> > 2) {
      __builtin_amdgcn_sched_barrier(0);
      lane = fresh(lane), n = lane & 15, g = lane >> 4;
    }
  };
  for (int t0 = sp.begin, flip = 0; t0 < sp.end; t0 += kDeltaTile, flip ^= 1) {
    const int live = min(kDeltaTile, sp.end - t0);
    lk.store(ldsK);
    if (Out) lq.store(ldsQ);
    lg.store(&G);
    if constexpr (kDirect) {
      wait_vm<0>();
    } else {
      lv.store(ldsV);
      lm.store(ldsM);
    }
    lds_barrier();
    if (!kLate) fetch(t0 + kDeltaTile);
    if (threadIdx.x == 0) bad[flip ^ 1] = kDeltaTile;
    if (G.good < live) {
      clear_rows<C>(ldsK, G.good);
      lds_barrier();
    }
    const size_t slot = slot0 + t0 / kDeltaTile;
    again();
    // Scores [own token][earlier tokens] as operands for all waves: a wave forms NP blocks of 16
    // own tokens with PG groups of 32 earlier ones.
    if constexpr (Scores) {
      constexpr int NP = C::NW < 4 ? 4 / C::NW : 1, PG = C::NW == 8 ? 1 : 2;
      const int pg0 = C::NW == 8 ? w >> 2 : 0;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int b = (w + C::NW * i) & 3, t = row_of(b, n);
        f32x4_t p[2 * PG];
#pragma unroll
        for (int j = 0; j < 2 * PG; ++j) p[j] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int ks = 0; ks < C::KS; ++ks) {
          const auto own = row_units<T, C>(ldsQ, t, ks, g);
#pragma unroll
          for (int j = 0; j < 2 * PG; ++j) Num<T>::mma(p[j], row_units<T, C>(ldsK, row_of(2 * pg0 + j, n), ks, g), own);
        }
#pragma unroll
        for (int z = 0; z < PG; ++z) {
          const int ks = pg0 + z;
          float x[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] = p[2 * z + (j >> 2)][j & 3];
          decayed<true>(G, t, 32 * ks + 8 * g, P.scale, x);
          Parts<T, kOut> parts;
          split(parts, x);
          if (ks == 0 || b >= 2) Pk::put(ldsP, lower_pair(b, ks), lane, parts);
        }
      }
    }
    again();
    // What the state predicts for the tile's keys; the values less that, y; and what of that
    // stays as the tile is read token by token, e.
    f32x4_t y[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) y[b] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) {
      typename Num<T>::V8 kk[4];
#pragma unroll
      for (int b = 0; b < 4; ++b) kk[b] = row_units<T, C>(ldsK, row_of(b, n), ks, g);
      const Parts<T, kParts> s = S.template operand<kParts>(ks);
      if constexpr (Back) store_columns<T, C>(back.S + slot * (D * D), ks, e0, lane, s);
#pragma unroll
      for (int i = Parts<T, kParts>::kN - 1; i >= 0; --i)
#pragma unroll
        for (int b = 0; b < 4; ++b) Num<T>::mma(y[b], kk[b], s.v[i]);
    }
    // (Back: what the walk needs of the gradient of u, at the wave's tokens 32 ks + 8 g + j)
    auto vector = [&](const float* m, int ks, float* x) {
      eight(m + (slot * D + e0 + n) * kDeltaTile + 32 * ks + 8 * g, x);
    };
    float part[2][8], f[2][8];
    auto add_up = [&](int i) {
      const float sum = token_sums(part, lane);
      sums[i][w][token_of(lane)] = sum;
    };
    {
      Parts<T, kParts> by[2];
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        float into[8], beta[8];
        eight(&G.into[32 * ks + 8 * g], into);
        eight(&G.beta[32 * ks + 8 * g], beta);
        float x[8];
        auto v8 = value_column<T, C>(ldsV, w, ks, lane);
        drop_bad<T>(v8, 32 * ks + 8 * g, &bad[flip]);
        Num<T>::widen(v8, x);
        if constexpr (Back) {  // dv times what the state before the tile predicts
          vector(back.F, ks, f[ks]);
#pragma unroll
          for (int j = 0; j < 8; ++j) part[ks][j] = beta[j] * f[ks][j] * (-into[j] * y[2 * ks + (j >> 2)][j & 3]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) y[2 * ks + (j >> 2)][j & 3] = fmaf(-into[j], y[2 * ks + (j >> 2)][j & 3], x[j]);
        weighted<T>(by[ks], beta, y[2 * ks], y[2 * ks + 1]);
      }
      triangle<T, kParts, false>(y, ldsM, by, lane);
      if constexpr (Back) add_up(0);
    }
    again();
    if constexpr (Back) {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        float x[8], beta[8];
        vector(back.E, ks, x);
#pragma unroll
        for (int b = 2 * ks; b < 2 * ks + 2; ++b)
          *reinterpret_cast<f32x4_t*>(back.E + (slot * D + e0 + n) * kDeltaTile + row_of(b, 4 * g)) = y[b];
        eight(&G.beta[32 * ks + 8 * g], beta);
#pragma unroll
        for (int j = 0; j < 8; ++j) part[ks][j] = x[j] * (beta[j] * y[2 * ks + (j >> 2)][j & 3]);
      }
      add_up(1);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int j = 0; j < 8; ++j) part[ks][j] = f[ks][j] * y[2 * ks + (j >> 2)][j & 3];
      add_up(2);
    }
    lds_barrier();  // the scores are there; nobody reads the values and the triangle any more
    const int good = min(min(bad[flip], G.good), live);
    if (t0 + kDeltaTile < sp.end) fetch_direct(t0 + kDeltaTile);
    if constexpr (Out) {
      again();
      f32x4_t o[4];
#pragma unroll
      for (int b = 0; b < 4; ++b) o[b] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int ks = 0; ks < C::KS; ++ks) {
        typename Num<T>::V8 qq[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) qq[b] = row_units<T, C>(ldsQ, row_of(b, n), ks, g);
        const Parts<T, kOut> s = S.template operand<kOut>(ks);
#pragma unroll
        for (int i = Parts<T, kOut>::kN - 1; i >= 0; --i)
#pragma unroll
          for (int b = 0; b < 4; ++b) Num<T>::mma(o[b], s.v[i], qq[b]);
      }
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const float f = P.scale * G.into[row_of(b, n)];
#pragma unroll
        for (int r = 0; r < 4; ++r) o[b][r] *= f;
      }
      if constexpr (Scores) {
        Parts<T, kOut> u[2];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          float beta[8];
          eight(&G.beta[32 * ks + 8 * g], beta);
          weighted<T>(u[ks], beta, y[2 * ks], y[2 * ks + 1]);
        }
        triangle<T, kOut, true>(o, ldsP, u, lane);
      }
      if constexpr (Back) {
        const __amdgpu_buffer_rsrc_t rd =
            make_rsrc(static_cast<const T*>(back.dout) + (vrow + t0) * D, (uint32_t)(live * C::kRow));
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          float x = 0.0f;
          const uint32_t from = (uint32_t)(row_of(b, n) * C::kRow + (e0 + 4 * g) * C::ES);
          if constexpr (sizeof(T) == 2) {
            const u32x2_t z = __builtin_amdgcn_raw_buffer_load_b64(rd, from, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) x = fmaf(o[b][r], r & 1 ? bf16_hi(z[r >> 1]) : bf16_lo(z[r >> 1]), x);
          } else {
            const u32x4_t z = __builtin_amdgcn_raw_buffer_load_b128(rd, from, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) x = fmaf(o[b][r], __uint_as_float(z[r]), x);
          }
          x += __shfl_xor(x, 16);
          x += __shfl_xor(x, 32);
          sums[3][w][row_of(b, n)] = x;
        }
      } else {
        const __amdgpu_buffer_rsrc_t ro = make_rsrc(out + (vrow + t0) * D, (uint32_t)(live * C::kRow));
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int t = row_of(b, n);
          f32x4_t z = o[b];
#pragma unroll
          for (int r = 0; r < 4; ++r) z[r] = t >= good ? __builtin_nanf("") : z[r];
          const uint32_t to = (uint32_t)(t * C::kRow + (e0 + 4 * g) * C::ES);
          if constexpr (sizeof(T) == 2) {
            __builtin_amdgcn_raw_buffer_store_b64((u32x2_t){pack_bf16x2(z[0], z[1]), pack_bf16x2(z[2], z[3])}, ro,
                                                  to, 0, 0);
          } else {
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, z), ro, to, 0, 0);
          }
        }
      }
    }
    again();
    if (kLate) fetch(t0 + kDeltaTile);
    Parts<T, kParts> u[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      float late[8];
      eight(&G.late[32 * ks + 8 * g], late);
      weighted<T>(u[ks], late, y[2 * ks], y[2 * ks + 1]);
    }
    const float whole = G.whole;
#pragma unroll
    for (int i = 0; i < C::NB; ++i) {
      f32x4_t x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const auto a = key_column<T, C>(ldsK, i, kt, lane);
#pragma unroll
        for (int z = Parts<T, kParts>::kN - 1; z >= 0; --z) Num<T>::mma(x, a, u[kt].v[z]);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) S.s[i][r] = fmaf(whole, S.s[i][r], x[r]);
    }
    if (good < live) S.fill(__builtin_nanf(""));
    lds_barrier();
    if constexpr (Back) {
      // (the next tile's are written behind one more barrier)
      if ((int)threadIdx.x < live) {
        const int64_t at = gate_row(P, sp, h) + t0 + threadIdx.x;
        float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < C::NW; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] += sums[j][i][threadIdx.x];
        back.from[at] = x[0] + x[3];
        back.on[at] = x[1];
        back.dbeta[at] = x[2];
      }
    }
  }
  if constexpr (!Out) {
    if (!map) S.store_record(recB + record, e0, lane);
    if (map) S.store_transposed(recM + record, e0, lane);
    if (map && back.M) S.store_record(back.M + record, e0, lane);
  } else if (!Back && final_state && sp.last) {
    S.store(final_state + pair * (D * D), e0, lane);
  }
}

// The records become the state before each unit, in place: S -> M S + B from unit to unit.
// A workgroup takes 16 value channels, wave w the key channels 16 w ..; the state passes from
// wave to wave through LDS, in fp32, with fp32 products.  Back: from the last unit to the
// first, with M's transpose, the gradient of the state after each unit.  A step takes the rows
// 16 w .. of the map (Back: its columns), whose records hold four of their values in 16 bytes.
//
// Bound by a step's chain: the exchange through LDS, and at heads of 128 the 32 fp32 matrix
// instructions of each of two waves a SIMD (0.8 us a step where one sequence runs).  32768 tokens, 8 heads of 64: 28 us (60 with
// records as matrices and loads after the products); 58000 packed tokens, 8 heads of 128: 108
// (222).  Four units ahead: no faster, and more loads in vain where sequences are short.
template <int D, bool Back>
__global__ void __launch_bounds__(4 * D)
scan_kernel(DeltaPlan P, const int32_t* cu, const float* S0, float* recB, const float* recM) {
  constexpr int KS = D / 16, kPitch = D + 4;
  __shared__ __attribute__((aligned(16))) float lds[2][16 * kPitch];
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // The workgroups that read the same maps are eight apart: one L2 serves them.
  const int pair = (int)(blockIdx.x / (8 * KS)) * 8 + (int)(blockIdx.x % 8), e0 = 16 * (int)(blockIdx.x / 8 % KS);
  if (pair >= P.nseq * P.value_heads) return;
  const int s = pair / P.value_heads, h = pair % P.value_heads;
  const int64_t len = P.ragged ? (int64_t)cu[s + 1] - cu[s] : P.rows;
  const int first = P.ragged ? first_slot(P, cu[s], s) : s * P.units_per_seq;
  const int units = units_of(len, P.unit);
  const size_t record = ((size_t)h * P.units + first) * (D * D);
  f32x4_t* B = reinterpret_cast<f32x4_t*>(recB + record + e0 * D) + (4 * w + g) * 16 + n;
  const f32x4_t* M = reinterpret_cast<const f32x4_t*>(recM + record + 16 * w * D) + g * 16 + n;
  f32x4_t x = {0.0f, 0.0f, 0.0f, 0.0f};
  struct Records {
    f32x4_t b, m[KS];
  };
  if (S0) {
    const float* p = S0 + ((int64_t)s * P.value_heads + h) * (D * D) + (16 * w + 4 * g) * D + e0 + n;
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] = p[r * D];
  }
  // The i-th unit of the walk.  What is read of the last, which has no record, is not used;
  // the first has no map where it starts from zeros.
  auto unit = [&](int i) { return Back ? units - 1 - i : i; };
  auto fetch = [&](int i) {
    Records rec;
    const size_t at = (size_t)unit(min(i, units - 1)) * (D * D / 4);
    rec.b = B[at];
#pragma unroll
    for (int j = 0; j < KS; ++j) rec.m[j] = M[at + 64 * j];
    return rec;
  };
  if (units == 1) {
    B[0] = x;
    return;
  }
  // The next units' records are under way while one unit's are multiplied.
  constexpr int kAhead = 2;
  Records rec[kAhead];
#pragma unroll
  for (int z = 0; z < kAhead; ++z)
    if (z < units - 1) rec[z] = fetch(z);
  if (!S0) {
#pragma unroll
    for (int j = 0; j < KS; ++j) rec[0].m[j] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
  }
  // (steps behind the last keep the state and store it again: what is loaded and stored under a
  // condition would be waited for earlier)
  for (int i0 = 0; i0 < units; i0 += kAhead) {
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int i = i0 + a;
      float* sx = lds[a & 1];
      *reinterpret_cast<f32x4_t*>(&sx[n * kPitch + 16 * w + 4 * g]) = x;
      B[(size_t)unit(min(i, units - 1)) * (D * D / 4)] = x;
      lds_barrier();
      f32x4_t y[KS], z[2] = {rec[a].b, {0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
      for (int j = 0; j < KS; ++j) y[j] = *reinterpret_cast<const f32x4_t*>(&sx[n * kPitch + 16 * j + 4 * g]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < KS; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          z[r & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(rec[a].m[j][r], y[j][r], z[r & 1], 0, 0, 0);
      rec[a] = fetch(i + kAhead);
#pragma unroll
      for (int r = 0; r < 4; ++r) x[r] = i + 1 < units ? z[0][r] + z[1][r] : x[r];
    }
  }
}

}  // namespace

namespace {

// The launches before the outputs: gates and triangles; records and the states between units.
template <typename T, int D>
void launch_prep(const DeltaPlan& p, const void* k, const float* log_decay, const float* beta, const int32_t* cu,
                 unsigned char* base, bool backward, hipStream_t st) {
  if (p.tokens > 0)
    hipLaunchKernelGGL((prep_kernel<T, D>), dim3(p.tiles, p.value_heads), dim3(kThreads), 0, st, p, tile_spans(p),
                       (const T*)k, log_decay, beta, cu, base + p.off_pack, backward ? base + p.off_packT : nullptr);
}
template <typename T, int D, WalkMode Mode>
void launch_walk(const DeltaPlan& p, const void* q, const void* k, const void* v, const float* S0, const int32_t* cu,
                 unsigned char* base, void* out, float* final_state, const BackOut& back, hipStream_t st) {
  hipLaunchKernelGGL((walk_kernel<T, D, Mode>), dim3(p.grid_units, p.value_heads, Mode == kRecords ? 2 : 1),
                     dim3((WalkSizes<T, D>::NT)), 0, st, p, (const T*)q, (const T*)k, (const T*)v, S0, cu,
                     base + p.off_pack,
                     reinterpret_cast<float*>(base + p.off_B), reinterpret_cast<float*>(base + p.off_M), (T*)out,
                     final_state, back);
}
template <int D, bool Back>
void launch_scan(const DeltaPlan& p, const int32_t* cu, const float* S0, unsigned char* base, hipStream_t st) {
  const int pairs = (p.nseq * p.value_heads + 7) / 8 * 8;
  hipLaunchKernelGGL((scan_kernel<D, Back>), dim3(pairs * (D / 16)), dim3(4 * D), 0, st, p, cu, S0,
                     reinterpret_cast<float*>(base + (Back ? p.off_D : p.off_B)),
                     reinterpret_cast<const float*>(base + (Back ? p.off_MT : p.off_M)));
}

}  // namespace

gbla_status launch_delta_forward(const DeltaPlan& p, const void* q, const void* k, const void* v,
                                 const float* log_decay, const float* beta, const float* S0,
                                 const int32_t* cu, void* ws, void* out, float* final_state,
                                 hipStream_t st) {
  unsigned char* base = static_cast<unsigned char*>(ws);
  return by_type(p, [&](auto t, auto dim) {
    using T = decltype(t);
    constexpr int D = decltype(dim)::value;
    launch_prep<T, D>(p, k, log_decay, beta, cu, base, false, st);
    if (!p.single) {
      launch_walk<T, D, kRecords>(p, q, k, v, S0, cu, base, nullptr, nullptr, {}, st);
      launch_scan<D, false>(p, cu, S0, base, st);
    }
    launch_walk<T, D, kOutputs>(p, q, k, v, S0, cu, base, out, final_state, {}, st);
  });
}

gbla_status launch_delta_backward(const DeltaPlan& p, const void* q, const void* k, const void* v,
                                  const float* log_decay, const float* beta, const float* S0,
                                  const int32_t* cu, const void* dout, const float* dfinal, void* ws,
                                  void* dq, void* dk, void* dv, float* dlog_decay, float* dbeta,
                                  float* dS0, hipStream_t st) {
  unsigned char* base = static_cast<unsigned char*>(ws);
  auto floats = [&](size_t off) { return reinterpret_cast<float*>(base + off); };
  // (the decays' gradient takes it too)
  if (!dS0 && S0) dS0 = floats(p.off_dS0);
  const BackOut back = {dout, floats(p.off_F), floats(p.off_S), floats(p.off_E), floats(p.off_from), floats(p.off_on),
                        dbeta, floats(p.off_MT), dfinal != nullptr};
  gbla_status done = by_type(p, [&](auto t, auto dim) {
    using T = decltype(t);
    constexpr int D = decltype(dim)::value;
    launch_prep<T, D>(p, k, log_decay, beta, cu, base, true, st);
    if (!p.single) {
      launch_walk<T, D, kRecords>(p, q, k, v, S0, cu, base, nullptr, nullptr, back, st);
      launch_scan<D, false>(p, cu, S0, base, st);
    }
  });
  if (done == GBLA_OK) done = launch_delta_back_records(p, q, k, cu, dout, ws, st);
  if (done != GBLA_OK) return done;
  done = by_type(p, [&](auto, auto dim) {
    constexpr int D = decltype(dim)::value;
    if (!p.single) launch_scan<D, true>(p, cu, dfinal, base, st);
  });
  if (done == GBLA_OK) done = launch_delta_back_walk(p, q, k, cu, dout, dfinal, ws, dS0, st);
  if (done != GBLA_OK) return done;
  done = by_type(p, [&](auto t, auto dim) {
    using T = decltype(t);
    constexpr int D = decltype(dim)::value;
    launch_walk<T, D, kBack>(p, q, k, v, S0, cu, base, nullptr, nullptr, back, st);
  });
  if (done != GBLA_OK) return done;
  return launch_delta_grads(p, q, k, S0, cu, dout, ws, dq, dk, dv, dlog_decay, dS0,
                            dfinal != nullptr, st);
}

}  // namespace gbla
