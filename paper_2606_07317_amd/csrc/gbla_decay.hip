// gbla_decay.hip -- causal linear attention with a decay per key head, in chunks
// (gfx950): the forward, and the backward's gradient of the queries, which is the
// same pass with other operands.
//
//   S_t = lam S_{t-1} + k_t v_t^T,  o_t = scale S_t^T q_t,  lam = exp(g)
// over a tile of L <= 64 tokens with the state S before it:
//   o_t   = scale (sum_{s <= t} lam^(t-s) (q_t k_s) v_s + lam^(t+1) S^T q_t)
//   S_out = lam^L S + sum_s lam^(L-1-s) k_s v_s^T
// Every power has an exponent >= 0, so strong decays underflow to 0 and nothing
// overflows.
//
// A workgroup of four waves walks the tiles of a unit with the state in registers.  Wave
// w owns tokens 16 w .. of a tile for the scores and outputs, and a 16-column block of
// the state.  Units of one sequence run at the same time: a first launch sums every
// unit's own k v^T (record_kernel), a second carries the records from unit to unit
// (scan_kernel), the third walks (walk_kernel).  Sequences of one unit, and batches
// that fill the chip by themselves, take the third alone.
//
// The gradient of the queries, dq_t = scale (sum lam^(t-s) (do_t v_s) k_s +
// lam^(t+1) S do_t), is walk_kernel of (do, v, k) with the transposed state.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gbla_decay_tiles.h"

namespace gbla {
namespace {

// The sizes that each kernel takes.
template <typename T, int D>
using RecordSizes = DC<T, D, D, D == 128 ? 8 : 4, 1, false>;
// At d = 128 a walk is two workgroups, each with half of the value channels: two run on
// a CU, so that one's matrix products meet the other's vector work.  (One of eight waves,
// which the barriers keep in step: its time was the sum of the matrix, the vector and the
// LDS work.)  In the forward two parts of the state and of the scores leave 2^-17 of a
// term, below the bf16 rounding of the output that they form; a third costs 10 % of one
// prompt (n = 32768, d = 64) and 21 % of the packed prompts (d = 128, shared heads).  Back,
// the sums are gradients' and have fp32's accuracy, by three parts of both: the state's
// products also form the decay's gradient, an fp32 sum of both signs (its error is 0.1e-6 ..
// 0.5e-6 where two parts left 1e-6 .. 3e-6).
template <bool Back>
constexpr int kWalkParts = Back ? 3 : 2;
template <typename T, int D, bool Back>
using WalkSizes = DC<T, D, D == 128 ? 64 : D, 4, kWalkParts<Back>, true>;

// Records: the sum of a unit's own products, A^T (weights B).
//   Reverse = false: weights lam^(tokens of the unit after t), for the state after it;
//   Reverse = true: scale lam^(tokens of the unit up to t), for the gradient of the
//   state before it, summed over the `group` heads of A and B.
// The last unit's (first unit's) record is not needed and left out.
template <typename T, int D, bool Reverse>
__device__ __forceinline__ void record_unit(const DecayPlan& P, const Span& sp, int h, const T* A,
                                            const T* B, int heads, int group, float g, float* rec,
                                            unsigned char* ldsA, unsigned char* ldsB, Powers& pw) {
  using C = RecordSizes<T, D>;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Decay lam(g);
  const float full = lam(kTile);
  const int n = sp.end - sp.begin, tiles = (n + kTile - 1) / kTile, steps = tiles * group;
  State<T, C> S;
  S.clear();
  TileLoad<T, C, D> la, lb;
  const int64_t row0 = first_row(P, sp, heads, h * group);
  auto fetch = [&](int step) {
    const int i = step / group;
    const int t = sp.begin + (Reverse ? tiles - 1 - i : i) * kTile;
    const int64_t row = (row0 + (int64_t)(step % group) * P.rows + t) * D;
    la.load(A + row, sp.end - t);
    lb.load(B + row, sp.end - t);
  };
  if (steps > 0) fetch(0);
  pw.fill(lam, P.scale);
  for (int step = 0; step < steps; ++step) {
    const int i = step / group, gi = step % group;
    const int live = min(kTile, sp.end - (sp.begin + (Reverse ? tiles - 1 - i : i) * kTile));
    la.store(ldsA);
    lb.store(ldsB);
    lds_barrier();
    if (step + 1 < steps) fetch(step + 1);
    const float f = gi > 0 ? 1.0f : live == kTile ? full : lam(live);
    S.advance(f, ldsA, ldsB, Reverse ? pw.up : pw.down, w, lane);
    lds_barrier();
  }
  S.store(rec, 0, w, lane);
}

// Both sides of a backward (B = 8, n = 2048, H = 16, d = 64) 32 us, 134 MB, 4.2 TB/s: bound
// by memory.  At d = 128 (16 sequences, T = 57,511, H = 8) 118 us, 4.0 TB/s, with matrix
// instructions under way in 37 % of a SIMD's cycles.
// blockIdx.z = 0: records of the state (k or v by v or k), 1 (backward): of its
// gradient.
template <typename T, int D>
__global__ void __launch_bounds__((RecordSizes<T, D>::NT), 2)
record_kernel(DecayPlan P, const T* A, const T* B, const T* q, const T* dout,
              const float* log_decay, const int32_t* cu, float* recS, float* recD) {
  using C = RecordSizes<T, D>;
  __shared__ __attribute__((aligned(512))) unsigned char ldsA[kTile * C::Wide::kPitch],
      ldsB[kTile * C::Wide::kPitch];
  __shared__ __attribute__((aligned(16))) Powers pw;
  Span sp;
  if (!find_span<C::NT>(P, cu, blockIdx.x, &sp)) return;
  const int h = blockIdx.y;
  const size_t at = ((size_t)h * P.units + sp.slot) * (D * D);
  if (blockIdx.z == 0) {
    if (sp.last) return;
    record_unit<T, D, false>(P, sp, h, A, B, P.kv_heads, 1, log_decay[h], recS + at, ldsA, ldsB,
                              pw);
  } else {
    if (sp.idx == 0) return;
    record_unit<T, D, true>(P, sp, h, q, dout, P.heads, P.group, log_decay[h], recD + at, ldsA, ldsB,
                              pw);
  }
}

// The records become the state before each unit (the first parts) or the
// gradient of the state after each unit (the others), in place.  A workgroup takes 256
// elements; its waves take consecutive quarters of up to 4 * kScanUnits units, whose
// records they hold in registers: each sums its own, the sums go from wave to wave
// through LDS, and each carries what enters its quarter over its records.  Bound by
// memory: both sides of 16 packed sequences (57,511 tokens, d = 128, H = 8, 126 MB of
// records) 65 us, 3.9 TB/s.
constexpr int kScanUnits = 8;
template <int D>
__global__ void __launch_bounds__(kThreads)
scan_kernel(DecayPlan P, const float* log_decay, const int32_t* cu, const float* S0, bool transposed,
            float* recS, const float* dfinal, float* recD) {
  constexpr int W = kThreads / 64, R = kScanUnits, slices = D * D / 256;
  __shared__ f32x4_t sums[2][W][64];
  // Neighbouring workgroups take neighbouring slices, so that those in flight read
  // whole records: slices of one offset in many records lie on few memory channels (with
  // the slice as the slowest grid index the same took 126 us).
  const int parts = recD ? 2 * slices : slices, s = blockIdx.x / parts, part = blockIdx.x % parts;
  const int h = blockIdx.y, lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool back = part >= slices;
  const int len = P.ragged ? cu[s + 1] - cu[s] : P.rows;
  const int first = P.ragged ? first_slot(P, cu[s], s) : s * P.units_per_seq;
  const int units = units_of(len, P.unit);
  const int el = ((part - (back ? slices : 0)) * 64 + lane) * 4;
  const Decay lam(log_decay[h]);
  const float full = lam(P.unit);
  // Unit i of the walk (backwards from the last): its record, and its decay.  Only
  // the sequence's last unit may be short; forwards nothing is carried over it.
  float* rec = (back ? recD : recS) + ((size_t)h * P.units + first) * (D * D) + el;
  auto at = [&](int i) {
    return reinterpret_cast<f32x4_t*>(rec + (int64_t)(back ? units - 1 - i : i) * (D * D));
  };
  const float f0 = back ? lam(len - (units - 1) * P.unit) : full;
  auto carry = [](f32x4_t& x, float f, const f32x4_t& r) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = fmaf(f, x[e], r[e]);
  };
  const float* init = back ? dfinal : S0;
  f32x4_t x = {0.0f, 0.0f, 0.0f, 0.0f};
  if (init) {
    const float* m = init + ((int64_t)s * P.kv_heads + h) * (D * D);
    if (transposed && !back) {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = m[(el % D + e) * D + el / D];
    } else {
      x = *reinterpret_cast<const f32x4_t*>(m + el);
    }
  }
  for (int base = 0, flip = 0; base < units; base += W * R, flip ^= 1) {
    const int here = min(W * R, units - base), each = (here + W - 1) / W;
    const int i0 = base + w * each, n = max(0, min(each, base + here - i0));
    f32x4_t r[R], sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < R; ++j) {
      r[j] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
      if (j < n && i0 + j < units - 1) r[j] = *at(i0 + j);
    }
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (j < n) carry(sum, i0 + j == 0 ? f0 : full, r[j]);
    sums[flip][w][lane] = sum;
    __syncthreads();
    // what enters the wave's quarter, and the next round
    f32x4_t enter = x;
#pragma unroll
    for (int v = 0; v < W; ++v) {
      if (v == w) enter = x;
      const int begin = base + v * each, m = max(0, min(each, base + here - begin));
      if (m > 0) carry(x, begin == 0 ? f0 * lam((m - 1) * P.unit) : lam(m * P.unit), sums[flip][v][lane]);
    }
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (j < n) {
        *at(i0 + j) = enter;
        carry(enter, i0 + j == 0 ? f0 : full, r[j]);
      }
  }
}

// A step's outputs pair by pair (see watch): of the lane's token `own` (a row of the
// tile's queries at `q`) in the channels that it has stored at `out`.
template <typename T, int D, bool Back>
__device__ __forceinline__ void walk_again(T* out, const T* q, int own, int live, int g,
                                           const unsigned char* ldsK, const unsigned char* ldsV,
                                           const unsigned char* ldsS, const Decay& lam, float scale) {
  using C = WalkSizes<T, D, Back>;
  own = fresh(own);  // (what is worked out from them stays in here)
  g = fresh(g);
  q += own * D;
  out += own * D;
  const int lane = threadIdx.x & 63;
  const uint64_t bad = __ballot(row_watch<T, D>(C::kRow / 16, [&](int u) {
    return reinterpret_cast<const T*>(ldsK + C::Wide::unit_at(lane, u));
  }) != 0.0f);
  // rows that are not stored; those whose scores are not finite, and so none of their channels
  if (own >= live || (bad & ((2ull << own) - 1)) != 0 || !shared_row_finite<T, D>(q, g)) return;
#pragma unroll 1
  for (int o = 0; o < C::OB; ++o) {
    const int e = 16 * o + 4 * g;
    if (__ballot(!finite4(out + e)) == 0) continue;
    f32x4_t sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
    for (int c = 0; c < D; ++c) {
      const float x = widen1(q[c]);
#pragma unroll
      for (int r = 0; r < 4; ++r) sum[r] = fmaf(x, plane_at<T, C>(ldsS, c, e + r), sum[r]);
    }
    sum *= scale * lam(own + 1);
#pragma unroll 1
    for (int s = 0; s <= own; ++s)
#pragma unroll
      for (int r = 0; r < 4; ++r) sum[r] = fmaf(tile_at<T, typename C::Slim>(ldsV, s, e + r), 0.0f, sum[r]);
    if (__ballot(wanted4(out + e, sum)) == 0) continue;
#pragma unroll 1
    for (int s = 0; s <= own; ++s) {
      const float x = row_dot<D>(
          g, [&](int c) { return widen1(q[c]); },
          [&](int c) { return tile_at<T, typename C::Wide>(ldsK, s, c); });
      const float w = scale * lam(own - s) * x;
#pragma unroll
      for (int r = 0; r < 4; ++r) sum[r] = fmaf(w, tile_at<T, typename C::Slim>(ldsV, s, e + r), sum[r]);
    }
    mend4(out + e, sum);
  }
}

// The walk of a head whose decay is 0: o_t = scale (q_t k_t) v_t, and the last token's k v^T as
// the final state.  By itself, so that 0 times a state's infinities never arises.
// final_state: the pair's, where the span has to write it.
template <typename T, int D, int VD>
__device__ __forceinline__ void walk_forgetful(const DecayPlan& P, const Span& sp, const T* q,
                                               const T* k, const T* v, int e0, const float* init,
                                               T* out, float* final_state) {
  using R = RowPieces<T, D>;
  constexpr int U = 2;  // tokens of a lane at once
  const int c0 = (threadIdx.x % R::kLanes) * R::kPer, rows = blockDim.x / R::kLanes;
  const bool mine = c0 >= e0 && c0 < e0 + VD;
  // (the bound by the workgroup's first token: the lanes of a row add up their products)
  for (int t0 = sp.begin; t0 < sp.end; t0 += U * rows) {
    typename R::Piece kk[U], vv[U];
    int64_t at[U];
    bool live[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u * rows + (int)threadIdx.x / R::kLanes;
      live[u] = t < sp.end;
      at[u] = (int64_t)min(t, sp.end - 1) * D + c0;
      R::load(kk[u], k + at[u]);
      R::load(vv[u], v + at[u]);
    }
    for (int gi = 0; gi < P.group; ++gi) {
      const int64_t head = (int64_t)gi * P.rows * D;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        typename R::Piece x;
        R::load(x, q + head + at[u]);
        const float p = P.scale * R::dot(x, kk[u]);
#pragma unroll
        for (int i = 0; i < R::kPer; ++i) x[i] = p * vv[u][i];
        if (live[u] && mine) R::store(out + head + at[u], x);
      }
    }
  }
  if (!final_state) return;
  for (int i = threadIdx.x; i < D * VD; i += blockDim.x) {
    const int c = i / VD, e = e0 + i % VD;
    const int64_t last = (int64_t)(sp.len - 1) * D;
    final_state[c * D + e] = sp.len > 0 ? widen1(k[last + c]) * widen1(v[last + e])
                             : init     ? init[c * D + e]
                                        : 0.0f;
  }
}

// The walk.  q, out: `heads` heads, k, v: `kv_heads`.  The state before the unit
// comes from rec (split) or S0 (single; transposed [e][c] for the gradient of q).
// final_state: written by the sequence's last unit.  Back (the gradient of q): the
// states before the units of a single walk are kept in rec, and `dg` takes the parts
// of the decay's gradient of the pairs whose earlier token lies before the tile,
// with q the forward's queries in `other`.
// Shared: several query heads to a key head.
// Measured: bf16, B = 1, n = 32768, H = 8, d = 64 32 us (134 MB, 4.2 TB/s); 64 packed
// sequences, T = 177,929, H = 8, K = 2, d = 128 379 us, where matrix instructions are
// under way in 35 % of a SIMD's cycles and LDS reads in 34 %: two waves a SIMD (the
// registers allow no more) leave the two, the vector work and the barriers mostly one
// after the other.  Half of the LDS reads (the state's blocks as operands from the
// registers, scores through LDS) took the same time, at more registers.
template <typename T, int D, bool Back, bool Shared>
__global__ void __launch_bounds__((WalkSizes<T, D, Back>::NT), (sizeof(T) == 2 && D == 32 ? 4 : 2))
walk_kernel(DecayPlan P, const T* q, const T* k, const T* v, const float* log_decay, const float* S0,
            const int32_t* cu, float* rec, T* out, float* final_state, const T* other, double* dg) {
  using C = WalkSizes<T, D, Back>;
  __shared__ __attribute__((aligned(512))) unsigned char ldsK[kTile * C::Wide::kPitch],
      ldsV[kTile * C::Slim::kPitch], ldsS[C::NP * C::kPlane];
  __shared__ __attribute__((aligned(16))) Powers pw;
  const int h = blockIdx.y, lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4, tw = w;
  // Halves of one unit eight workgroups apart: on one XCD, whose L2 has what they share.
  constexpr int halves = D / C::VD;
  const int unit = halves == 1 ? blockIdx.x : (blockIdx.x >> 4) * 8 + (blockIdx.x & 7);
  const int e0 = halves == 1 ? 0 : ((blockIdx.x >> 3) & 1) * C::VD;
  if (halves > 1 && unit >= P.grid_units) return;
  Span sp;
  double dsum = 0.0;
  const bool found = find_span<C::NT>(P, cu, unit, &sp);
  if (found) {
    const int64_t pair = (int64_t)sp.s * P.kv_heads + h;
    const float* init = S0 ? S0 + pair * (D * D) : nullptr;
    bool transposed = Back;
    float* keep = nullptr;  // records of a single walk
    if (P.single) {
      if (Back && rec)
        keep = rec + ((size_t)h * P.units + sp.slot) * (D * D);
    } else {
      init = rec + ((size_t)h * P.units + sp.slot) * (D * D);
      transposed = false;
      if (!S0 && sp.idx == 0) init = nullptr;
    }
    State<T, C> S;
    if (init) S.load(init, transposed, e0, w, lane);
    else S.clear();

    TileLoad<T, C, D> lk;
    TileLoad<T, C, C::VD> lv;
    OwnRows<T, C> qq;
    OwnPieces<T, C> qo;  // of the forward's queries, for the decay's gradient
    const int64_t krow0 = first_row(P, sp, P.kv_heads, h), qrow0 = first_row(P, sp, P.heads, h * P.group);
    auto fetch_kv = [&](int t) {
      const int64_t row = (krow0 + t) * D;
      lk.load(k + row, sp.end - t);
      lv.load(v + row + e0, sp.end - t);
    };
    auto fetch_q = [&](int t, int gi) {
      const int64_t row = (qrow0 + (int64_t)gi * P.rows + t) * D;
      qq.load(q + row, sp.end - t, 16 * tw + n, g);
      if (Back) qo.load(other + row, dg ? sp.end - t : 0, 16 * tw + n, e0, g);
    };
    if (sp.begin < sp.end) {
      fetch_kv(sp.begin);
      fetch_q(sp.begin, 0);
    }
    const Decay lam(log_decay[h]);
    if (lam.forgets()) {
      walk_forgetful<T, D, C::VD>(P, sp, q + qrow0 * D, k + krow0 * D, v + krow0 * D, e0, init, out + qrow0 * D,
                                  final_state && sp.last ? final_state + pair * (D * D) : nullptr);
      if (Back && dg && lane == 0) dg[(((int64_t)h * P.grid_units + unit) * halves + e0 / C::VD) * C::NW + w] = 0.0;
      return;
    }
    const float full = lam(kTile);
    const float into = P.scale * lam(16 * tw + n + 1);
    Scores<true> scores;
    scores.fill(lam, P.scale, n, g);
    pw.fill(lam, P.scale);

    // A step: one query head's tokens of a tile.  Its rows are read before the step and
    // the next step's as soon as the products with them are under way, under no
    // condition (past the end they load nothing): the compiler waits for as many loads
    // as the path with the fewest has in flight, so that a branch around a prefetch
    // makes every step wait for it.
    for (int t0 = sp.begin, gi = 0; t0 < sp.end;) {
      const int live = min(kTile, sp.end - t0);
      const bool final = t0 + kTile >= sp.end;
      if (!Shared || gi == 0) {
        if (Back && keep && ((t0 - sp.begin) & (P.unit - 1)) == 0)
          S.store(keep + (int64_t)((t0 - sp.begin) / P.unit) * (D * D), e0, w, lane);
        lk.store(ldsK);
        lv.store(ldsV);
        S.to_planes(ldsS, w, lane);
        lds_barrier();
        if (!Shared) fetch_kv(t0 + kTile);
      }
      const int64_t row = (qrow0 + (int64_t)gi * P.rows + t0) * D;
      const bool wrap = !Shared || gi + 1 == P.group;
      const int next_t = wrap ? t0 + kTile : t0, next_gi = wrap ? 0 : gi + 1;
      {
        // Scores of the tile's tokens (16 a block), then the state's part of the output,
        // whose products run while the scores are decayed.
        f32x4_t p[4], acc[C::OB];
#pragma unroll
        for (int b = 0; b < 4; ++b) p[b] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int ks = 0; ks < C::KS; ++ks)
#pragma unroll
          for (int b = 0; b < 4; ++b)
            Num<T>::mma(p[b], row_at<T, typename C::Wide>(ldsK, b, n, ks, g), qq.v[ks]);
#pragma unroll
        for (int o = 0; o < C::OB; ++o) acc[o] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int ks = 0; ks < C::KS; ++ks)
#pragma unroll
          for (int x = C::NP - 1; x >= 0; --x)
#pragma unroll
            for (int o = 0; o < C::OB; ++o)
              Num<T>::mma(acc[o], row_at<T, typename C::Wide>(ldsS + x * C::kPlane, o, n, ks, g), qq.v[ks]);
        const OwnPieces<T, C> qo_now = qo;
        fetch_q(next_t, next_gi);
#pragma unroll
        for (int b = 0; b < 4; ++b) scores.apply(p[b], tw - b, n, g);
#pragma unroll
        for (int o = 0; o < C::OB; ++o)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[o][r] *= into;
        if (Back) {
          // sum_t ((t + 1) - (tokens of the unit from the tile on)) q_t dq_t
          const int at = ((t0 - sp.begin) & (P.unit - 1));
          const int rest = min(P.unit, sp.end - (t0 - at)) - at;
          dsum += (double)qo_now.dot(acc) * (double)(16 * tw + n + 1 - rest);
        }
#pragma unroll
        for (int x = 0; x < 2; ++x)
          add_scored<T, C, typename C::Slim, kWalkParts<Back>>(acc, p[2 * x], p[2 * x + 1], ldsV, x, 0, lane);
        pipeline<T, 4 * C::KS, C::KS * C::NP * C::OB>();
        if (Shared && gi == 0) fetch_kv(t0 + kTile);
        float bad = 0.0f;
        watch<C::OB>(bad, acc);
        const __amdgpu_buffer_rsrc_t ro = make_rsrc(out + row, (uint32_t)(live * C::kRow));
        const uint32_t at = (uint32_t)((16 * tw + n) * C::kRow + (e0 + 4 * g) * C::ES);
#pragma unroll
        for (int o = 0; o < C::OB; ++o) {
          if constexpr (sizeof(T) == 2) {
            const u32x2_t y = {pack_bf16x2(acc[o][0], acc[o][1]), pack_bf16x2(acc[o][2], acc[o][3])};
            __builtin_amdgcn_raw_buffer_store_b64(y, ro, at + 16 * o * C::ES, 0, 0);
          } else {
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, acc[o]), ro,
                                                   at + 16 * o * C::ES, 0, 0);
          }
        }
        if (__builtin_expect(seen(bad), 0))
          walk_again<T, D, Back>(out + row + e0, q + row, 16 * tw + n, live, g, ldsK, ldsV, ldsS, lam, P.scale);
      }
      if (Shared && ++gi < P.group) continue;
      gi = 0;
      if (!final || (final_state && sp.last)) {
        S.advance(live == kTile ? full : lam(live), ldsK, ldsV, pw.down + kTile - live, w, lane);
      }
      lds_barrier();
      t0 += kTile;
    }
    if (final_state && sp.last) S.store(final_state + pair * (D * D), e0, w, lane);
  }
  if (Back && dg) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) dsum += __shfl_xor(dsum, o);
    if (lane == 0) dg[(((int64_t)h * P.grid_units + unit) * halves + e0 / C::VD) * C::NW + w] = dsum;
  }
}

template <typename T, int D>
dim3 walk_grid(const DecayPlan& p) {
  const bool whole = WalkSizes<T, D, false>::VD == D;
  return dim3(whole ? p.grid_units : (p.grid_units + 7) / 8 * 16, p.kv_heads);
}

template <typename F>
gbla_status by_type(const DecayPlan& p, F f) {
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

gbla_status launch_decay_forward(const DecayPlan& p, const void* q, const void* k, const void* v,
                                 const float* log_decay, const float* S0, const int32_t* cu,
                                 void* ws, void* out, float* final_state, hipStream_t st) {
  float* rec = reinterpret_cast<float*>(static_cast<unsigned char*>(ws) + p.off_S);
  return by_type(p, [&](auto t, auto dim) {
    using T = decltype(t);
    constexpr int D = decltype(dim)::value;
    const dim3 grid(p.grid_units, p.kv_heads);
    if (!p.single) {
      hipLaunchKernelGGL((record_kernel<T, D>), grid, dim3(RecordSizes<T, D>::NT), 0, st, p, (const T*)k, (const T*)v,
                         (const T*)nullptr, (const T*)nullptr, log_decay, cu, rec, (float*)nullptr);
      hipLaunchKernelGGL((scan_kernel<D>), dim3(p.nseq * (D * D / 256), p.kv_heads), dim3(kThreads), 0,
                         st, p, log_decay, cu, S0, false, rec, (const float*)nullptr, (float*)nullptr);
    }
    const auto walk = p.group > 1 ? walk_kernel<T, D, false, true> : walk_kernel<T, D, false, false>;
    hipLaunchKernelGGL(walk, (walk_grid<T, D>(p)), dim3((WalkSizes<T, D, false>::NT)), 0, st, p, (const T*)q, (const T*)k, (const T*)v, log_decay,
                       S0, cu, rec, (T*)out, final_state, (const T*)nullptr, (double*)nullptr);
  });
}

gbla_status launch_decay_backward(const DecayPlan& p, const void* q, const void* k, const void* v,
                                  const float* log_decay, const float* S0, const int32_t* cu,
                                  const void* dout, const float* dfinal, void* ws, void* dq,
                                  void* dk, void* dv, float* dlog_decay, float* dS0,
                                  hipStream_t st) {
  unsigned char* base = static_cast<unsigned char*>(ws);
  float* recS = reinterpret_cast<float*>(base + p.off_S);
  float* recD = reinterpret_cast<float*>(base + p.off_D);
  double* dg = dlog_decay ? reinterpret_cast<double*>(base + p.off_dg) : nullptr;
  const gbla_status done = by_type(p, [&](auto t, auto dim) {
    using T = decltype(t);
    constexpr int D = decltype(dim)::value;
    const dim3 grid(p.grid_units, p.kv_heads);
    if (!p.single) {
      hipLaunchKernelGGL((record_kernel<T, D>), dim3(p.grid_units, p.kv_heads, 2), dim3(RecordSizes<T, D>::NT), 0, st, p,
                         (const T*)v, (const T*)k, (const T*)q, (const T*)dout, log_decay, cu, recS,
                         recD);
      hipLaunchKernelGGL((scan_kernel<D>), dim3(p.nseq * (2 * D * D / 256), p.kv_heads),
                         dim3(kThreads), 0, st, p, log_decay, cu, S0, true, recS, dfinal, recD);
    }
    const auto walk = p.group > 1 ? walk_kernel<T, D, true, true> : walk_kernel<T, D, true, false>;
    hipLaunchKernelGGL(walk, (walk_grid<T, D>(p)), dim3((WalkSizes<T, D, false>::NT)), 0, st, p, (const T*)dout, (const T*)v, (const T*)k,
                       log_decay, S0, cu, p.single && !dg ? (float*)nullptr : recS, (T*)dq, (float*)nullptr, (const T*)q, dg);
  });
  if (done != GBLA_OK) return done;
  return launch_decay_keys(p, q, k, v, log_decay, S0, cu, dout, dfinal, ws, dk, dv, dlog_decay, dS0,
                           st);
}

}  // namespace gbla
