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

// Three parts of D and of the scores, so that the sums have fp32's accuracy before they
// are rounded once (with two parts of the scores and of the values' D, 2^-17 of a term, three
// times as many bf16 gradients differed by a last bit from the fp32 sums; the third parts
// cost 3 % of a backward).
constexpr int kKeysParts = 3;
template <typename T, int D>
using KeysSizes = DC<T, D, D, D == 128 ? 8 : 4, kKeysParts, false>;

// What the rows' second pass needs, kept in LDS meanwhile: in scalar registers it leaves the
// first pass too few (a backward of 16 packed sequences, d = 128 791 us for 756).
template <typename T>
struct Rows {
  const float* init;             // D after the span
  const T *q, *dout, *k, *v;     // the span's first rows (of the first query head)
  T *dk, *dv;
  int64_t head;                  // from one query head's row to the next head's
  int group, tokens;
  float scale;
};

// A tile's gradients pair by pair (see watch): of the lane's token `own` in the channels
// that it has stored; the tile's rows begin `at` elements after the span's.
template <typename T, int D>
__device__ __forceinline__ void keys_again(const Rows<T>& a, int64_t at, int own, int live, int g,
                                           int eh, const unsigned char* ldsD, const Decay& lam) {
  using C = KeysSizes<T, D>;
  own = fresh(own);  // (what is worked out from them stays in here)
  g = fresh(g);
  const int lane = threadIdx.x & 63;
  uint64_t bad[2] = {0, 0};  // tokens with a row of q, of dout that is not finite
#pragma unroll 1
  for (int gi = 0; gi < a.group; ++gi)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const T* row = (i ? a.dout : a.q) + at + gi * a.head + min(lane, live - 1) * D;
      bad[i] |= __ballot(row_watch<T, D>(D * C::ES / 16, [&](int u) {
        return row + u * RowPieces<T, D>::kPer;
      }) != 0.0f);
    }
  if (own >= live) return;  // not stored
  // Both gradients by the same code: dv = sum (q k) do + D^T k, dk = sum (do v) q + D v.
#pragma unroll 1
  for (int i = 0; i < 2 * C::OB; ++i) {
    const bool values = i < C::OB;
    const T* left = (values ? a.q : a.dout) + at;
    const T* right = (values ? a.dout : a.q) + at;
    const T* mine = (values ? a.k : a.v) + at + own * D;
    const int e = 16 * (eh * C::OB + (values ? i : i - C::OB)) + 4 * g;
    T* to = (values ? a.dv : a.dk) + at + own * D + e;
    if (__ballot(!finite4(to)) == 0) continue;
    // scores that are not finite, and so no channel
    if ((values ? bad[0] : bad[1]) >> own != 0 || !shared_row_finite<T, D>(mine, g)) continue;
    f32x4_t sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
    for (int c = 0; c < D; ++c) {
      const float x = widen1(mine[c]);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        sum[r] = fmaf(x, plane_at<T, C>(ldsD, values ? c : e + r, values ? e + r : c), sum[r]);
    }
    sum *= lam(live - 1 - own);
#pragma unroll 1
    for (int gi = 0; gi < a.group; ++gi)
#pragma unroll 1
      for (int t = own; t < live; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) sum[r] = fmaf(widen1(right[gi * a.head + t * D + e + r]), 0.0f, sum[r]);
    if (__ballot(wanted4(to, sum)) == 0) continue;
#pragma unroll 1
    for (int gi = 0; gi < a.group; ++gi) {
#pragma unroll 1
      for (int t = own; t < live; ++t) {
        const int64_t row = gi * a.head + t * D;
        const float x = row_dot<D>(
            g, [&](int c) { return widen1(left[row + c]); }, [&](int c) { return widen1(mine[c]); });
        const float w = a.scale * lam(t - own) * x;
#pragma unroll
        for (int r = 0; r < 4; ++r) sum[r] = fmaf(w, widen1(right[row + e + r]), sum[r]);
      }
    }
    mend4(to, sum);
  }
}

// The gradients of a head whose decay is 0: dv_t = scale (q_t k_t) do_t and dk_t = scale
// (do_t v_t) q_t, and what the final state's gradient D gives the last token.
// dS0: the pair's, where the span has to write it; it may be D.
template <typename T, int D>
__device__ __forceinline__ void keys_forgetful(const DecayPlan& P, const Span& sp, const Rows<T>& a,
                                               float* dS0) {
  using R = RowPieces<T, D>;
  const int c0 = (threadIdx.x % R::kLanes) * R::kPer, rows = blockDim.x / R::kLanes;
  const int last = sp.len - 1 - sp.begin;
  for (int t0 = 0; t0 < a.tokens; t0 += rows) {
    const int t = t0 + (int)threadIdx.x / R::kLanes;
    const int64_t at = (int64_t)min(t, a.tokens - 1) * D;
    typename R::Piece k, v, sk, sv;
    R::load(k, a.k + at + c0);
    R::load(v, a.v + at + c0);
#pragma unroll
    for (int i = 0; i < R::kPer; ++i) sk[i] = sv[i] = 0.0f;
    if (t == last && a.init) {
      for (int e = 0; e < D; ++e) {
        const float x = widen1(a.v[at + e]), y = widen1(a.k[at + e]);
#pragma unroll
        for (int i = 0; i < R::kPer; ++i) {
          sk[i] = fmaf(a.init[(c0 + i) * D + e], x, sk[i]);
          sv[i] = fmaf(a.init[e * D + c0 + i], y, sv[i]);
        }
      }
    }
    for (int gi = 0; gi < a.group; ++gi) {
      typename R::Piece q, o;
      R::load(q, a.q + at + gi * a.head + c0);
      R::load(o, a.dout + at + gi * a.head + c0);
      const float x = a.scale * R::dot(q, k), y = a.scale * R::dot(o, v);
#pragma unroll
      for (int i = 0; i < R::kPer; ++i) {
        sv[i] = fmaf(x, o[i], sv[i]);
        sk[i] = fmaf(y, q[i], sk[i]);
      }
    }
    if (t < a.tokens) {
      R::store(a.dk + at + c0, sk);
      R::store(a.dv + at + c0, sv);
    }
  }
  __syncthreads();  // D has been read
  if (dS0)
    for (int i = threadIdx.x; i < D * D; i += blockDim.x) dS0[i] = sp.len == 0 && a.init ? a.init[i] : 0.0f;
}

// Shared: several query heads to a key head.
// Measured: bf16, B = 8, n = 2048, H = 16, d = 64 68 us (201 MB, 3.0 TB/s); 16 packed
// sequences, T = 57,511, H = 8, d = 128 398 us, one workgroup a CU by its LDS, matrix
// instructions under way in 27 % of a SIMD's cycles and LDS reads in 47 % (half of that
// conflicts, which the walk's swizzle would spare for registers that there are none of).
// The work between two barriers is a chain of products, decays and splits that two waves a
// SIMD do not cover.
template <typename T, int D, bool Shared>
__global__ void __launch_bounds__((KeysSizes<T, D>::NT), 2)
keys_kernel(DecayPlan P, const T* q, const T* k, const T* v, const float* log_decay,
            const float* S0, const int32_t* cu, const T* dout, const float* dfinal,
            const float* recS, const float* recD, T* dk, T* dv, float* dS0, double* dg) {
  using C = KeysSizes<T, D>;
  __shared__ __attribute__((aligned(512))) unsigned char ldsQ[kTile * C::Wide::kPitch],
      ldsO[kTile * C::Wide::kPitch], ldsD[C::NP * C::kPlane];
  __shared__ __attribute__((aligned(16))) Powers pw;
  __shared__ Rows<T> rows;
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
      kept = recS + ((size_t)h * P.units + sp.slot) * (D * D);
    } else {
      const size_t at = ((size_t)h * P.units + sp.slot) * (D * D);
      init = dfinal || !sp.last ? recD + at : nullptr;
      kept = recS + at;
    }
    const int64_t krow0 = first_row(P, sp, P.kv_heads, h), qrow0 = first_row(P, sp, P.heads, h * P.group);
    {
      const int64_t ka = (krow0 + sp.begin) * D, qa = (qrow0 + sp.begin) * D;
      const Rows<T> a = {init, q + qa, dout + qa, k + ka, v + ka, dk + ka, dv + ka,
                         (int64_t)P.rows * D, P.group, sp.end - sp.begin, P.scale};
      if (Decay(log_decay[h]).forgets()) {
        keys_forgetful<T, D>(P, sp, a, dS0 && sp.begin == 0 ? dS0 + pair * (D * D) : nullptr);
        if (dg && lane == 0) dg[((int64_t)h * P.grid_units + blockIdx.x) * C::NW + w] = 0.0;
        return;
      }
      if (threadIdx.x == 0) rows = a;
    }
    State<T, C> S;
    if (init) S.load(init, false, 0, w, lane);
    else S.clear();

    const int tiles = (sp.end - sp.begin + kTile - 1) / kTile;
    TileLoad<T, C, D> lq, lo;
    OwnRows<T, C> kf, vf;
    OwnPieces<T, C> kp;
    auto fetch = [&](int t, int gi) {
      const int64_t row = (qrow0 + (int64_t)gi * P.rows + t) * D;
      const int live = t < sp.begin ? 0 : sp.end - t;
      lq.load(q + row, live);
      lo.load(dout + row, live);
    };
    auto fetch_own = [&](int t) {  // none before the unit
      const int64_t row = (krow0 + t) * D;
      const int live = t < sp.begin ? 0 : sp.end - t;
      kf.load(k + row, live, 16 * tw + n, g);
      vf.load(v + row, live, 16 * tw + n, g);
      kp.load(k + row, dg ? live : 0, 16 * tw + n, 16 * eh * C::OB, g);
    };
    if (tiles > 0) {
      fetch(sp.begin + (tiles - 1) * kTile, 0);
      fetch_own(sp.begin + (tiles - 1) * kTile);
    }
    const Decay lam(log_decay[h]);
    const float full = lam(kTile);
    Scores<false> scores;
    scores.fill(lam, P.scale, n, g);
    pw.fill(lam, P.scale);

    // The lane that LDS addresses are made from, anew for each phase of a step: they free
    // registers, and a backward (B = 8, n = 2048, H = 16, d = 64) takes 141 us for 145.  At
    // d = 128, where the walk waits for its own products anyway, it changes little (756 us for
    // 764 of 16 packed sequences).
    auto place = [&] { return D < 128 ? fresh(lane) : lane; };

    for (int tile = tiles - 1; tile >= 0; --tile) {
      const int t0 = sp.begin + tile * kTile, live = min(kTile, sp.end - t0);
      const int64_t krow = (krow0 + t0) * D;
      f32x4_t ak[C::OB], av[C::OB];
#pragma unroll
      for (int o = 0; o < C::OB; ++o) ak[o] = av[o] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
      float inner = 0.0f;
      for (int gi = 0; gi < (Shared ? P.group : 1); ++gi) {
        lq.store(ldsQ);
        lo.store(ldsO);
        if (gi == 0) S.to_planes(ldsD, w, place());
        lds_barrier();
        const bool wrap = !Shared || gi + 1 == P.group;
        fetch(wrap ? t0 - kTile : t0, wrap ? 0 : gi + 1);
        // The values' gradient, then the keys': scores of the tile's tokens (16 a block),
        // the part of D, whose products run while the scores are decayed, the products of
        // the scores.  One after the other, since both at once do not fit the registers.
        // With several query heads the part of D is the first head's, and the branch around
        // it may not lie between a product and its use (the compiler does not count the wait
        // states of a jump reliably): it comes first then, and its results are scaled inside.
        // (Written out twice: from lambdas the single head's kernel took more registers, a
        // backward of 16 packed sequences, T = 57,511, H = 8, d = 128 787 us for 770.)
        const float out = lam(max(0, live - 1 - 16 * tw - n));
        if (Shared && gi == 0) {  // D^T k by rows of the planes [column][row], D v by their columns
          const int at_lane = place();
#pragma unroll
          for (int ks = 0; ks < C::KS; ++ks)
#pragma unroll
            for (int p = C::NP - 1; p >= 0; --p)
#pragma unroll
              for (int o = 0; o < C::OB; ++o)
                Num<T>::mma(av[o], row_at<T, typename C::Wide>(ldsD + p * C::kPlane, eh * C::OB + o, at_lane & 15, ks, at_lane >> 4), kf.v[ks]);
#pragma unroll
          for (int o = 0; o < C::OB; ++o)
#pragma unroll
            for (int r = 0; r < 4; ++r) av[o][r] *= out;
#pragma unroll
          for (int ks = 0; ks < C::KS; ++ks)
#pragma unroll
            for (int p = C::NP - 1; p >= 0; --p)
#pragma unroll
              for (int o = 0; o < C::OB; ++o)
                Num<T>::mma(ak[o], col_at<T, typename C::Wide, false>(ldsD + p * C::kPlane, eh * C::OB + o, ks, at_lane), vf.v[ks]);
#pragma unroll
          for (int o = 0; o < C::OB; ++o)
#pragma unroll
            for (int r = 0; r < 4; ++r) ak[o][r] *= out;
          // tokens of the unit after token s
          const int at = (t0 - sp.begin) & (P.unit - 1), size = min(P.unit, sp.end - (t0 - at));
          dsum += (double)kp.dot(ak) * (double)(size - 1 - at - 16 * tw - n);
        }
        f32x4_t x[4], y[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) x[b] = y[b] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
        int at_lane = place();
#pragma unroll
        for (int ks = 0; ks < C::KS; ++ks)
#pragma unroll
          for (int b = 0; b < 4; ++b)
            Num<T>::mma(x[b], row_at<T, typename C::Wide>(ldsQ, b, at_lane & 15, ks, at_lane >> 4), kf.v[ks]);
        if (!Shared) {  // D^T k by rows of the planes [column][row]
#pragma unroll
          for (int ks = 0; ks < C::KS; ++ks)
#pragma unroll
            for (int p = C::NP - 1; p >= 0; --p)
#pragma unroll
              for (int o = 0; o < C::OB; ++o)
                Num<T>::mma(av[o], row_at<T, typename C::Wide>(ldsD + p * C::kPlane, eh * C::OB + o, at_lane & 15, ks, at_lane >> 4), kf.v[ks]);
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) scores.apply(x[b], b - tw, n, g);
        if (!Shared) {
#pragma unroll
          for (int o = 0; o < C::OB; ++o)
#pragma unroll
            for (int r = 0; r < 4; ++r) av[o][r] *= out;
        }
#pragma unroll
        for (int p = 0; p < 2; ++p)
          add_scored<T, C, typename C::Wide, kKeysParts>(av, x[2 * p], x[2 * p + 1], ldsO, p, eh * C::OB, at_lane);
        if (!Shared) pipeline<T, 4 * C::KS, C::KS * C::NP * C::OB>();
        __builtin_amdgcn_sched_barrier(0);
        at_lane = place();
#pragma unroll
        for (int ks = 0; ks < C::KS; ++ks)
#pragma unroll
          for (int b = 0; b < 4; ++b)
            Num<T>::mma(y[b], row_at<T, typename C::Wide>(ldsO, b, at_lane & 15, ks, at_lane >> 4), vf.v[ks]);
        if (!Shared) {  // D v by their columns
#pragma unroll
          for (int ks = 0; ks < C::KS; ++ks)
#pragma unroll
            for (int p = C::NP - 1; p >= 0; --p)
#pragma unroll
              for (int o = 0; o < C::OB; ++o)
                Num<T>::mma(ak[o], col_at<T, typename C::Wide, false>(ldsD + p * C::kPlane, eh * C::OB + o, ks, at_lane), vf.v[ks]);
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
#pragma unroll
          for (int i = 0; i < 4; ++i)  // x is 0 where the order is wrong
            inner = fmaf(x[b][i] * y[b][i], (float)(16 * (b - tw) + 4 * g + i - n), inner);
          scores.apply(y[b], b - tw, n, g);
        }
        if (!Shared) {
#pragma unroll
          for (int o = 0; o < C::OB; ++o)
#pragma unroll
            for (int r = 0; r < 4; ++r) ak[o][r] *= out;
          // tokens of the unit after token s
          const int at = (t0 - sp.begin) & (P.unit - 1), size = min(P.unit, sp.end - (t0 - at));
          dsum += (double)kp.dot(ak) * (double)(size - 1 - at - 16 * tw - n);
        }
#pragma unroll
        for (int p = 0; p < 2; ++p)
          add_scored<T, C, typename C::Wide, kKeysParts>(ak, y[2 * p], y[2 * p + 1], ldsQ, p, eh * C::OB, at_lane);
        if (!Shared) pipeline<T, 4 * C::KS, C::KS * C::NP * C::OB, 4>();
        __builtin_amdgcn_sched_barrier(0);
        if (wrap) fetch_own(t0 - kTile);
        S.advance(gi > 0 ? 1.0f : live == kTile ? full : lam(live), ldsQ, ldsO, pw.up, w, place());
        lds_barrier();
      }
      if (eh == 0) dsum += (double)inner;
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
      if (dg && ((t0 - sp.begin) & (P.unit - 1)) == 0) {  // the unit's first tile: <S_in, D_in>
        const int unit = (t0 - sp.begin) / P.unit;
        const int size = min(P.unit, sp.end - t0);
        if (S0 || sp.idx + unit > 0) {
          State<T, C> in;
          in.load(kept + (int64_t)unit * (D * D), true, 0, w, lane);
          float dot = 0.0f;
#pragma unroll
          for (int i = 0; i < C::SR; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) dot = fmaf(in.s[i][r], S.s[i][r], dot);
          dsum += (double)dot * (double)size;
        }
      }
    }
    // The rows again where a value may have reached too far.  That takes a row of q or dout
    // that is not finite, whose own token's pair (at distance 0) makes the sum for the decay
    // NaN, or such a D, whose products with k do.
    const bool mine = __ballot(!isfinite(dsum)) != 0;
    if (lane == 0) reinterpret_cast<int*>(ldsQ)[w] = mine;
    lds_barrier();
    bool again = false;
#pragma unroll
    for (int i = 0; i < C::NW; ++i) again |= reinterpret_cast<int*>(ldsQ)[i] != 0;
    if (__builtin_expect(__ballot(again) != 0, 0)) {
      const Rows<T> a = rows;
      if (a.init) S.load(a.init, false, 0, w, lane);
      else S.clear();
#pragma unroll 1
      for (int t0 = (a.tokens - 1) / kTile * kTile; t0 >= 0; t0 -= kTile) {
        const int live = min(kTile, a.tokens - t0);
        const int64_t at = (int64_t)t0 * D;
#pragma unroll 1
        for (int gi = 0; gi < a.group; ++gi) {
          lds_barrier();
          lq.load(a.q + at + gi * a.head, live);
          lo.load(a.dout + at + gi * a.head, live);
          lq.store(ldsQ);
          lo.store(ldsO);
          if (gi == 0) S.to_planes(ldsD, w, lane);
          lds_barrier();
          if (gi == 0) keys_again<T, D>(a, at, 16 * tw + n, live, g, eh, ldsD, lam);
          S.advance(gi > 0 ? 1.0f : live == kTile ? full : lam(live), ldsQ, ldsO, pw.up, w, lane);
        }
      }
    }
    if (dS0 && sp.begin == 0) S.store(dS0 + pair * (D * D), 0, w, lane);
  }
  if (dg) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) dsum += __shfl_xor(dsum, o);
    if (lane == 0) dg[((int64_t)h * P.grid_units + blockIdx.x) * C::NW + w] = dsum;
  }
}

// The sum of a key head's parts: [2][K][count] doubles (of walk_kernel and keys_kernel, a
// wave's each).
__global__ void __launch_bounds__(kThreads)
decay_sum_kernel(int kv_heads, int64_t count, const double* dg, float* out) {
  __shared__ double red[kThreads / 64];
  const int h = blockIdx.x;
  const double* a = dg + h * count;
  const double* b = a + kv_heads * count;
  double sum = 0.0;
  for (int64_t i = threadIdx.x; i < count; i += kThreads) sum += a[i] + b[i];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < kThreads / 64; ++i) sum += red[i];
    out[h] = (float)sum;
  }
}

template <typename T, int D>
void launch_keys(const DecayPlan& p, const void* q, const void* k, const void* v, const float* log_decay,
                 const float* S0, const int32_t* cu, const void* dout, const float* dfinal,
                 unsigned char* ws, void* dk, void* dv, float* dlog_decay, float* dS0, hipStream_t st) {
  double* dg = dlog_decay ? reinterpret_cast<double*>(ws + p.off_dg) : nullptr;
  const int64_t count = (int64_t)p.grid_units * KeysSizes<T, D>::NW;
  double* mine = dg ? dg + p.kv_heads * count : nullptr;
  const auto keys = p.group > 1 ? keys_kernel<T, D, true> : keys_kernel<T, D, false>;
  hipLaunchKernelGGL(keys, dim3(p.grid_units, p.kv_heads), dim3((KeysSizes<T, D>::NT)), 0, st, p,
                     (const T*)q, (const T*)k, (const T*)v, log_decay, S0, cu, (const T*)dout, dfinal,
                     reinterpret_cast<const float*>(ws + p.off_S),
                     reinterpret_cast<const float*>(ws + p.off_D), (T*)dk, (T*)dv, dS0, mine);
  if (dg)
    hipLaunchKernelGGL(decay_sum_kernel, dim3(p.kv_heads), dim3(kThreads), 0, st, p.kv_heads, count, dg, dlog_decay);
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
