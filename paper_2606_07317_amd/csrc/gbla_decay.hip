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
// A workgroup walks the tiles of a unit with the state in registers (four waves; at
// d = 128 eight, each with half of the output's channels).  Wave w owns tokens
// 16 (w & 3) .. of a tile for the scores and outputs, and a 16-column block of the
// state.  Units of one sequence run at the same time: a first launch sums every
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

// Records: the sum of a unit's own products, A^T (weights B).
//   Reverse = false: weights lam^(tokens of the unit after t), for the state after it;
//   Reverse = true: scale lam^(tokens of the unit up to t), for the gradient of the
//   state before it, summed over the `group` heads of A and B.
// The last unit's (first unit's) record is not needed and left out.
template <typename T, int D, bool Reverse>
__device__ __forceinline__ void record_unit(const DecayPlan& P, const Span& sp, int h, const T* A,
                                            const T* B, int heads, int group, float g, float* rec,
                                            unsigned char* ldsA, unsigned char* ldsB) {
  using C = DC<T, D>;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), gg = lane >> 4;
  const Decay lam(g);
  const float full = lam(kTile);
  const int n = sp.end - sp.begin, tiles = (n + kTile - 1) / kTile, steps = tiles * group;
  float weight[2][8];
  State<T, C> S, add;
  S.clear();
  TileLoad<C> la, lb;
  auto fetch = [&](int step) {
    const int i = step / group, head = h * group + step % group;
    const int t = sp.begin + (Reverse ? tiles - 1 - i : i) * kTile;
    const int64_t row = row_of(P, sp, heads, head, t) * D;
    la.load(A + row, sp.end - t);
    lb.load(B + row, sp.end - t);
  };
  if (steps > 0) fetch(0);
#pragma unroll
  for (int ks = 0; ks < 2; ++ks)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int t = 32 * ks + 8 * gg + j;
      weight[ks][j] = Reverse ? P.scale * lam(t + 1) : lam(kTile - 1 - t);
    }
  for (int step = 0; step < steps; ++step) {
    const int i = step / group, gi = step % group;
    const int live = min(kTile, sp.end - (sp.begin + (Reverse ? tiles - 1 - i : i) * kTile));
    la.store(ldsA);
    lb.store(ldsB);
    lds_barrier();
    if (step + 1 < steps) fetch(step + 1);
    if (gi == 0) add.clear();
    add.add_products(ldsA, ldsB, weight, w, lane);
    if (gi == group - 1) S.advance(live == kTile ? full : lam(live), add);
    lds_barrier();
  }
  S.store(rec, false, w, lane);
}

// blockIdx.z = 0: records of the state (k or v by v or k), 1 (backward): of its
// gradient.
template <typename T, int D>
__global__ void __launch_bounds__((DC<T, D>::NT), 1)
record_kernel(DecayPlan P, const T* A, const T* B, const T* q, const T* dout,
              const float* log_decay, const int32_t* cu, float* recS, float* recD) {
  using C = DC<T, D>;
  __shared__ __attribute__((aligned(16))) unsigned char ldsA[C::kTileBytes], ldsB[C::kTileBytes];
  Span sp;
  if (!find_span<C::NT>(P, cu, blockIdx.x, &sp)) return;
  const int h = blockIdx.y;
  const size_t at = ((size_t)h * P.units + sp.slot) * (D * D);
  if (blockIdx.z == 0) {
    if (sp.last) return;
    record_unit<T, D, false>(P, sp, h, A, B, P.kv_heads, 1, log_decay[h], recS + at, ldsA, ldsB);
  } else {
    if (sp.idx == 0) return;
    record_unit<T, D, true>(P, sp, h, q, dout, P.heads, P.group, log_decay[h], recD + at, ldsA, ldsB);
  }
}

// The records become the state before each unit (z even) or the gradient of the
// state after each unit (z odd), in place: four elements a thread, unit after unit.
template <int D>
__global__ void __launch_bounds__(kThreads)
scan_kernel(DecayPlan P, const float* log_decay, const int32_t* cu, const float* S0, bool transposed,
            float* recS, const float* dfinal, float* recD) {
  const int s = blockIdx.x, h = blockIdx.y;
  const bool back = blockIdx.z >= gridDim.z / (recD ? 2 : 1);
  const int part = back ? blockIdx.z - gridDim.z / 2 : blockIdx.z;
  int first, len;
  if (P.ragged) {
    first = units_before(cu, s, P.unit);
    len = cu[s + 1] - cu[s];
  } else {
    first = s * P.units_per_seq;
    len = P.rows;
  }
  const int units = units_of(len, P.unit);
  const int el = (part * kThreads + threadIdx.x) * 4;
  if (el >= D * D) return;
  const Decay lam(log_decay[h]);
  const float full = lam(P.unit);
  float* rec = (back ? recD : recS) + ((size_t)h * P.units + first) * (D * D) + el;
  const float* init = back ? dfinal : S0;
  f32x4_t x = {0.0f, 0.0f, 0.0f, 0.0f};
  if (init) {
    const float* m = init + ((int64_t)s * P.kv_heads + h) * (D * D);
    if (transposed && !back) {
#pragma unroll
      for (int r = 0; r < 4; ++r) x[r] = m[(el % D + r) * D + el / D];
    } else {
      x = *reinterpret_cast<const f32x4_t*>(m + el);
    }
  }
  // Unit u of the walk: stored in place of its record, then carried over it.  The
  // first record of a group is loaded while the last group's are carried.
  constexpr int G = 8;
  auto at = [&](int i) { return rec + (int64_t)(back ? units - 1 - i : i) * (D * D); };
  for (int i = 0; i < units; i += G) {
    f32x4_t r[G];
#pragma unroll
    for (int j = 0; j < G; ++j)
      if (i + j < units - 1) r[j] = *reinterpret_cast<const f32x4_t*>(at(i + j));
#pragma unroll
    for (int j = 0; j < G; ++j) {
      if (i + j < units) *reinterpret_cast<f32x4_t*>(at(i + j)) = x;
      if (i + j < units - 1) {
        // only the sequence's last unit may be short; backwards it comes first
        const float f = back && i + j == 0 ? lam(len - (units - 1) * P.unit) : full;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = fmaf(f, x[e], r[j][e]);
      }
    }
  }
}

// The walk.  q, out: `heads` heads, k, v: `kv_heads`.  The state before the unit
// comes from rec (split) or S0 (single; transposed [e][c] for the gradient of q).
// final_state: written by the sequence's last unit.  Back (the gradient of q): the
// states before the units of a single walk are kept in rec, and `dg` takes the parts
// of the decay's gradient of the pairs whose earlier token lies before the tile,
// with q the forward's queries in `other`.
template <typename T, int D, bool Back>
__global__ void __launch_bounds__((DC<T, D>::NT), 1)
walk_kernel(DecayPlan P, const T* q, const T* k, const T* v, const float* log_decay, const float* S0,
            const int32_t* cu, float* rec, T* out, float* final_state, const T* other, double* dg) {
  using C = DC<T, D>;
  __shared__ __attribute__((aligned(16))) unsigned char ldsK[C::kTileBytes], ldsV[C::kTileBytes],
      ldsS[C::NP * C::kPlane];
  const int h = blockIdx.y, lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4, tw = w & 3, eh = w >> 2;
  Span sp;
  double dsum = 0.0;
  const bool found = find_span<C::NT>(P, cu, blockIdx.x, &sp);
  if (found) {
    const int64_t pair = (int64_t)sp.s * P.kv_heads + h;
    const float* init = S0 ? S0 + pair * (D * D) : nullptr;
    bool transposed = Back;
    float* keep = nullptr;  // records of a single walk
    if (P.single) {
      if (Back && rec)
        keep = rec + ((size_t)h * P.units + (P.ragged ? sp.row0 / P.unit + sp.s
                                                       : (int64_t)sp.s * P.units_per_seq)) * (D * D);
    } else {
      init = rec + ((size_t)h * P.units + sp.slot) * (D * D);
      transposed = false;
      if (!S0 && sp.idx == 0) init = nullptr;
    }
    State<T, C> S, add;
    if (init) S.load(init, transposed, w, lane);
    else S.clear();
    bool some = init != nullptr;  // the state is not all zeros

    const int steps = (sp.end - sp.begin + kTile - 1) / kTile * P.group;
    TileLoad<C> lk, lv;
    OwnRows<T, C> own;
    auto fetch_kv = [&](int t) {
      const int64_t row = row_of(P, sp, P.kv_heads, h, t) * D;
      lk.load(k + row, sp.end - t);
      lv.load(v + row, sp.end - t);
    };
    auto fetch_q = [&](int t, int gi) {
      own.load(q + row_of(P, sp, P.heads, h * P.group + gi, t) * D, sp.end - t, 16 * tw + n, g);
    };
    if (steps > 0) {
      fetch_kv(sp.begin);
      fetch_q(sp.begin, 0);
    }
    const Decay lam(log_decay[h]);
    const float full = lam(kTile);
    // decays of the wave's scores: [earlier token 16 b + 4 g + i][own token 16 tw + n]
    float score[4][4], weight[2][8];
    const float into = P.scale * lam(16 * tw + n + 1);
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) score[b][i] = P.scale * lam(max(0, 16 * (tw - b) + n - 4 * g - i));
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int j = 0; j < 8; ++j) weight[ks][j] = lam(kTile - 1 - (32 * ks + 8 * g + j));

    for (int step = 0; step < steps; step += P.group) {
      const int t0 = sp.begin + step / P.group * kTile;
      const int live = min(kTile, sp.end - t0);
      const bool final = t0 + kTile >= sp.end;
      if (Back && keep && (t0 - sp.begin) % P.unit == 0)
        S.store(keep + (int64_t)((t0 - sp.begin) / P.unit) * (D * D), false, w, lane);
      lk.store(ldsK);
      lv.store(ldsV);
      if (some) S.to_planes(ldsS, w, lane);
      lds_barrier();
      if (!final) fetch_kv(t0 + kTile);
      for (int gi = 0; gi < P.group; ++gi) {
        const OwnRows<T, C> qq = own;
        if (gi + 1 < P.group) fetch_q(t0, gi + 1);
        else if (!final) fetch_q(t0 + kTile, 0);
        const int64_t row = row_of(P, sp, P.heads, h * P.group + gi, t0) * D;
        f32x4_t acc[C::OB];
#pragma unroll
        for (int o = 0; o < C::OB; ++o) acc[o] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
        if (some) {
#pragma unroll
          for (int ks = 0; ks < C::KS; ++ks)
#pragma unroll
            for (int x = C::NP - 1; x >= 0; --x)
#pragma unroll
              for (int o = 0; o < C::OB; ++o)
                Num<T>::mma(acc[o], row_at<T, C>(ldsS + x * C::kPlane, 16 * (eh * C::OB + o) + n, ks, g),
                            qq.v[ks]);
#pragma unroll
          for (int o = 0; o < C::OB; ++o)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[o][r] *= into;
          if (Back && dg && 16 * tw + n < live) {
            // sum_t ((t + 1) - (tokens of the unit from the tile on)) q_t dq_t
            const T* o4 = other + row + (int64_t)(16 * tw + n) * D + 16 * eh * C::OB + 4 * g;
            float dot = 0.0f;
#pragma unroll
            for (int o = 0; o < C::OB; ++o)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const float x = sizeof(T) == 2 ? __uint_as_float((uint32_t)o4[16 * o + r] << 16)
                                               : (float)o4[16 * o + r];
                dot = fmaf(x, acc[o][r], dot);
              }
            const int at = (t0 - sp.begin) % P.unit;
            const int rest = min(P.unit, sp.end - (t0 - at)) - at;
            dsum += (double)dot * (double)(16 * tw + n + 1 - rest);
          }
        }
        // scores of the earlier tokens' blocks b <= tw, decayed, as operands
        float p[4][4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          f32x4_t x = {0.0f, 0.0f, 0.0f, 0.0f};
          if (b <= tw) {
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks)
              Num<T>::mma(x, row_at<T, C>(ldsK, 16 * b + n, ks, g), qq.v[ks]);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)
            p[b][i] = b < tw || (b == tw && 4 * g + i <= n) ? x[i] * score[b][i] : 0.0f;
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          if (2 * ks > tw) continue;
          const float x[8] = {p[2 * ks][0],     p[2 * ks][1],     p[2 * ks][2],     p[2 * ks][3],
                              p[2 * ks + 1][0], p[2 * ks + 1][1], p[2 * ks + 1][2], p[2 * ks + 1][3]};
          Parts<T, 2> pp;
          pp.set(x);
#pragma unroll
          for (int o = 0; o < C::OB; ++o)
            pp.mma_right(acc[o], col_at<T, C, true>(ldsV, eh * C::OB + o, ks, lane));
        }
        const __amdgpu_buffer_rsrc_t ro = make_rsrc(out + row, (uint32_t)(live * C::kRow));
        const uint32_t at = (uint32_t)((16 * tw + n) * C::kRow + (16 * eh * C::OB + 4 * g) * C::ES);
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
      }
      if (!final || (final_state && sp.last)) {
        if (live < kTile)
#pragma unroll
          for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int j = 0; j < 8; ++j) weight[ks][j] = lam(max(0, live - 1 - (32 * ks + 8 * g + j)));
        add.clear();
        add.add_products(ldsK, ldsV, weight, w, lane);
        S.advance(live == kTile ? full : lam(live), add);
        some = true;
      }
      lds_barrier();
    }
    if (final_state && sp.last) S.store(final_state + pair * (D * D), false, w, lane);
  }
  if (Back && dg) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) dsum += __shfl_xor(dsum, o);
    if (lane == 0) dg[((int64_t)h * P.grid_units + blockIdx.x) * 8 + w] = dsum;
  }
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
    const dim3 grid(p.grid_units, p.kv_heads), block(DC<T, D>::NT);
    if (!p.single) {
      hipLaunchKernelGGL((record_kernel<T, D>), grid, block, 0, st, p, (const T*)k, (const T*)v,
                         (const T*)nullptr, (const T*)nullptr, log_decay, cu, rec, (float*)nullptr);
      hipLaunchKernelGGL((scan_kernel<D>), dim3(p.nseq, p.kv_heads, D * D / 1024), dim3(kThreads), 0,
                         st, p, log_decay, cu, S0, false, rec, (const float*)nullptr, (float*)nullptr);
    }
    hipLaunchKernelGGL((walk_kernel<T, D, false>), grid, block, 0, st, p, (const T*)q, (const T*)k,
                       (const T*)v, log_decay, S0, cu, rec, (T*)out, final_state, (const T*)nullptr,
                       (double*)nullptr);
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
    const dim3 grid(p.grid_units, p.kv_heads), block(DC<T, D>::NT);
    if (!p.single) {
      hipLaunchKernelGGL((record_kernel<T, D>), dim3(p.grid_units, p.kv_heads, 2), block, 0, st, p,
                         (const T*)v, (const T*)k, (const T*)q, (const T*)dout, log_decay, cu, recS,
                         recD);
      hipLaunchKernelGGL((scan_kernel<D>), dim3(p.nseq, p.kv_heads, 2 * (D * D / 1024)),
                         dim3(kThreads), 0, st, p, log_decay, cu, S0, true, recS, dfinal, recD);
    }
    hipLaunchKernelGGL((walk_kernel<T, D, true>), grid, block, 0, st, p, (const T*)dout,
                       (const T*)v, (const T*)k, log_decay, S0, cu,
                       p.single && !dg ? (float*)nullptr : recS, (T*)dq, (float*)nullptr, (const T*)q, dg);
  });
  if (done != GBLA_OK) return done;
  return launch_decay_keys(p, q, k, v, log_decay, S0, cu, dout, dfinal, ws, dk, dv, dlog_decay, dS0,
                           st);
}

}  // namespace gbla
