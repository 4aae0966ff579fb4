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

// Wave w takes the tokens row_of(w, ..) of a tile as its own.  All that is computed in fp32
// enters (bf16) as two parts: the states come so from the walks; the vectors u and dv are
// weighted and split once for all waves, into LDS as [value channel][token], where both the own
// tokens' operands and the others' are transposed reads.
//
// LDS holds them first; after the pairs' products the same place holds keys and queries below,
// and above the first 32 key channels of both states, [value channel][key channel]; the others
// follow by turns below and above, each loaded while the one before is multiplied.
//
// Bound by dependent steps at two waves a SIMD (registers): the matrix unit works 0.2 of the
// cycles, LDS 0.25, and 192 KB a tile of heads of 128 come at 3.2 TB/s.  8 x 2048 tokens, 16
// heads of 64: 106 us; 58000 packed tokens, 8 heads of 128: 445.  (Every wave gathering and
// splitting the states and vectors by itself: 491 and 2175.)
template <typename T, int D>
struct GradSizes {
  using C = DS<T, D, 4>;           // rows of the operands
  using V = DS<T, kDeltaTile, 4>;  // rows of the vectors
  using B = DS<T, 32, 4>;          // rows of 32 key channels of a state
  static constexpr int kN = Parts<T, kParts>::kN;
  static constexpr int kPlane = D * V::kPitch, kState = (sizeof(T) == 2 ? 2 : 1) * D * B::kPitch;
  static constexpr int kUpper = 2 * C::kTileBytes > 2 * kState ? 2 * C::kTileBytes : 2 * kState;
  static constexpr int kBytes = kUpper + 2 * kState > 2 * kN * kPlane ? kUpper + 2 * kState : 2 * kN * kPlane;
};
template <typename T, int D>
__global__ void __launch_bounds__(kThreads, D * sizeof(T) > 256 ? 1 : 2)
grads_kernel(DeltaPlan P, TileSpans tiles, const T* q, const T* k, const T* dout, const int32_t* cu,
             const unsigned char* packs, const float* S, const float* N, const float* E, const float* F, T* dq,
             T* dk, T* dv) {
  using Z = GradSizes<T, D>;
  using C = typename Z::C;
  using V = typename Z::V;
  using B = typename Z::B;
  constexpr bool kDirect = sizeof(T) == 2;
  __shared__ __attribute__((aligned(512))) unsigned char lds[Z::kBytes];
  __shared__ __attribute__((aligned(16))) Gates G;
  unsigned char *ldsK = lds, *ldsQ = lds + C::kTileBytes;
  Span sp;
  if (!find_span<kThreads>(tiles, cu, blockIdx.x, &sp)) return;
  const int hk = blockIdx.y, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = w >> 1;
  int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, own = row_of(w, n);
  // (addresses are worked out phase by phase: held over the kernel they cost registers)
  auto again = [&] { lane = fresh(lane), n = lane & 15, g = lane >> 4, own = row_of(w, n); };
  const int live = sp.end - sp.begin;
  if (live <= 0) return;
  const int64_t krow = first_row(P, sp, P.heads, hk) + sp.begin;
  const uint32_t bytes = (uint32_t)(live * C::kRow), at_lds = lds_address(lds);
  f32x4_t aq[C::NB], ak[C::NB];  // channels row_of(c, 4 g + r) of the own token
#pragma unroll
  for (int c = 0; c < C::NB; ++c) aq[c] = ak[c] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
  for (int gi = 0; gi < P.group; ++gi) {
    const int h = hk * P.group + gi;
    const size_t slot = (size_t)h * P.tiles + sp.slot;
    const int64_t vrow = first_row(P, sp, P.value_heads, h) + sp.begin;
    const __amdgpu_buffer_rsrc_t ro = make_rsrc(dout + vrow * D, bytes);
    if (gi > 0) lds_barrier();
    if (threadIdx.x < kGateBytes / 16)
      reinterpret_cast<u32x4_t*>(&G)[threadIdx.x] =
          reinterpret_cast<const u32x4_t*>(packs + slot * Packed<T, 3>::kBlock + Packed<T, 3>::kBytes)[threadIdx.x];
    auto gradient = [&](int t, int ks) {  // of the outputs
      Parts<T, 1> o;
      const uint32_t at = (uint32_t)(t * C::kRow + (32 * ks + 8 * g) * C::ES);
      if constexpr (sizeof(T) == 2) {
        o.v[0] = __builtin_amdgcn_raw_buffer_load_b128(ro, at, 0, 0);
      } else {
        o.v[0].a = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(ro, at, 0, 0));
        o.v[0].b = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(ro, at + 16, 0, 0));
      }
      return o;
    };
    {
      const int id = fresh((int)threadIdx.x), unit = id & 7;
      f32x4_t x[2][C::KS][2];
#pragma unroll
      for (int z = 0; z < 2; ++z)
#pragma unroll
        for (int i = 0; i < C::KS; ++i) {
          const f32x4_t* from = reinterpret_cast<const f32x4_t*>((z ? F : E) + slot * (D * kDeltaTile)) +
                                2 * (i * kThreads + id);
          x[z][i][0] = from[0];
          x[z][i][1] = from[1];
        }
      lds_barrier();
      float beta[8];
      eight(&G.beta[8 * unit], beta);
#pragma unroll
      for (int z = 0; z < 2; ++z)
#pragma unroll
        for (int i = 0; i < C::KS; ++i) {
          Parts<T, kParts> p;
          weighted<T>(p, beta, x[z][i][0], x[z][i][1]);
          const int row = (i * kThreads + id) / 8;
          if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int j = 0; j < Z::kN; ++j)
              *reinterpret_cast<u32x4_t*>(lds + (Z::kN * z + j) * Z::kPlane + V::unit_at(row, unit)) = p.v[j];
          } else {
            f32x4_t* to = reinterpret_cast<f32x4_t*>(lds + z * Z::kPlane + V::unit_at(row, 2 * unit));
            to[0] = p.v[0].a;
            to[1] = p.v[0].b;
          }
        }
    }
    lds_barrier();
    auto vectors = [&](int z, int b, int ks) {  // u (z = 0) or dv of the tokens row_of(b, ..)
      Parts<T, kParts> p;
#pragma unroll
      for (int j = 0; j < Z::kN; ++j) p.v[j] = key_column<T, V>(lds + (Z::kN * z + j) * Z::kPlane, b, ks, lane);
      return p;
    };
    // Pairs of an own token and others of the tile, [others][own]; the products of one order
    // are left out where the others' half has only the other.
    again();
    Parts<T, kParts> xp[2], yp[2], zp[2];
    auto pairs = [&](auto kt_, auto before_, auto after_) {
      constexpr int kt = decltype(kt_)::value;
      constexpr bool Before = decltype(before_)::value, After = decltype(after_)::value;
      float x[8], y[8], z[8], hi[8], lo[8];
      eight(&G.hi[32 * kt + 8 * g], hi);
      eight(&G.lo[32 * kt + 8 * g], lo);
      const float own_hi = G.hi[own], own_lo = G.lo[own];
      f32x4_t ou[2], uo[2], vu[2], uv[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) ou[i] = uo[i] = vu[i] = uv[i] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
      // (the next step's rows from memory are under way while this one's are multiplied)
      Parts<T, 1> o, others[2], next, next_others[2];
      auto ahead = [&](int ks) {
        if constexpr (Before) next = gradient(own, ks);
        if constexpr (After) next_others[0] = gradient(row_of(2 * kt, n), ks), next_others[1] = gradient(row_of(2 * kt + 1, n), ks);
      };
      ahead(0);
#pragma unroll
      for (int ks = 0; ks < C::KS; ++ks) {
        o = next, others[0] = next_others[0], others[1] = next_others[1];
        if (ks + 1 < C::KS) ahead(ks + 1);
        Parts<T, kParts> u, v;
        if constexpr (Before) v = vectors(1, w, ks);
        if constexpr (After) u = vectors(0, w, ks);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int b = 2 * kt + i;
          if constexpr (Before) {
            const Parts<T, kParts> a = vectors(0, b, ks);
            mma_parts<T>(uo[i], a, o);
            mma_parts<T>(uv[i], a, v);
          }
          if constexpr (After) {
            mma_parts<T>(vu[i], vectors(1, b, ks), u);
            mma_parts<T>(ou[i], others[i], u);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int j = 4 * i + r, t = 32 * kt + 8 * g + j;
          const float away = (own_hi - hi[j]) + (own_lo - lo[j]);
          const bool before = After ? Before && t <= own : true, after = Before ? After && t >= own : true;
          const float f = __builtin_amdgcn_exp2f(before ? away : -away), sf = P.scale * f;
          if constexpr (Before) x[j] = before ? sf * uo[i][r] : 0.0f;
          if constexpr (After) y[j] = after ? sf * ou[i][r] : 0.0f;
          if constexpr (Before && After) z[j] = t == own ? 0.0f : -f * (before ? uv[i][r] : vu[i][r]);
          else z[j] = -f * (Before ? uv[i][r] : vu[i][r]);
        }
      if constexpr (Before) split(xp[kt], x);
      if constexpr (After) split(yp[kt], y);
      split(zp[kt], z);
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    if (half) {
      pairs(I0{}, std::true_type{}, std::false_type{});
      pairs(I1{}, std::true_type{}, std::true_type{});
    } else {
      pairs(I0{}, std::true_type{}, std::true_type{});
      pairs(I1{}, std::false_type{}, std::true_type{});
    }
    again();
    Parts<T, kParts> u[C::KS], v[C::KS];
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) {
      u[ks] = vectors(0, w, ks);
      v[ks] = vectors(1, w, ks);
    }
    if (own < live) {
#pragma unroll
      for (int ks = 0; ks < C::KS; ++ks) {
        T* to = dv + (vrow + own) * D + 32 * ks + 8 * g;
        if constexpr (sizeof(T) == 2) {
          u32x4_t y;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            y[j] = pack_bf16x2(bf16_lo(v[ks].v[0][j]) + bf16_lo(v[ks].v[1][j]),
                               bf16_hi(v[ks].v[0][j]) + bf16_hi(v[ks].v[1][j]));
          *reinterpret_cast<u32x4_t*>(to) = y;
        } else {
          reinterpret_cast<f32x4_t*>(to)[0] = v[ks].v[0].a;
          reinterpret_cast<f32x4_t*>(to)[1] = v[ks].v[0].b;
        }
      }
    }
    lds_barrier();
    again();
    // Key channels 32 cc .. of both states, straight into LDS (fp32, whose rows there are
    // padded: through registers), S's before N's.
    constexpr int kPieces = D * 16 / kThreads;
    u32x4_t piece[kDirect ? 1 : kPieces];
    auto states = [&](int cc, int at) {
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const float* m = (z ? N : S) + slot * (D * D);
        if constexpr (kDirect) {
          rows_to_lds<T, B, 2 * D>(at_lds + at + z * Z::kState, reinterpret_cast<const T*>(m) + cc * (2 * D * 32),
                                   2 * D, w, lane);
        } else {
#pragma unroll
          for (int i = 0; i < kPieces / 2; ++i) {
            const int p = i * kThreads + (int)threadIdx.x;
            piece[z * (kPieces / 2) + i] = *reinterpret_cast<const u32x4_t*>(m + (p / 8) * D + 32 * cc + 4 * (p % 8));
          }
        }
      }
    };
    auto arrive = [&](int at) {
      if constexpr (kDirect) {
        wait_vm<0>();
      } else {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          const int p = i % (kPieces / 2) * kThreads + (int)threadIdx.x;
          *reinterpret_cast<u32x4_t*>(lds + at + i / (kPieces / 2) * Z::kState + B::unit_at(p / 8, p % 8)) = piece[i];
        }
      }
    };
    if constexpr (kDirect) {
      rows_to_lds<T, C>(at_lds, k + krow * D, live, w, lane);
      rows_to_lds<T, C>(at_lds + C::kTileBytes, q + krow * D, live, w, lane);
    }
    states(0, Z::kUpper);
    if constexpr (!kDirect) {
      RowsLoad<T, C> rows;
      rows.load(k + krow * D, live);
      rows.store(ldsK);
      rows.load(q + krow * D, live);
      rows.store(ldsQ);
    }
    arrive(Z::kUpper);
    lds_barrier();
    auto apply = [&](auto kt_, auto before_, auto after_) {
      constexpr int kt = decltype(kt_)::value;
#pragma unroll
      for (int c = 0; c < C::NB; ++c) {
        Parts<T, 1> kc, qc;
        kc.v[0] = key_column<T, C>(ldsK, c, kt, lane);
        mma_parts<T>(ak[c], kc, zp[kt]);
        if constexpr (decltype(before_)::value) mma_parts<T>(aq[c], kc, xp[kt]);
        if constexpr (decltype(after_)::value) {
          qc.v[0] = key_column<T, C>(ldsQ, c, kt, lane);
          mma_parts<T>(ak[c], qc, yp[kt]);
        }
        if (c & 1) __builtin_amdgcn_sched_barrier(0);
      }
    };
    if (half) {
      apply(I0{}, std::true_type{}, std::false_type{});
      apply(I1{}, std::true_type{}, std::true_type{});
    } else {
      apply(I0{}, std::true_type{}, std::true_type{});
      apply(I1{}, std::false_type{}, std::true_type{});
    }
    again();
    Parts<T, 1> o[C::KS];
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) o[ks] = gradient(own, ks);
    const float into = G.into[own], rest = G.rest[own], scaled = P.scale * into;
#pragma unroll
    for (int cc = 0; cc < C::KS; ++cc) {
      const int here = cc & 1 ? 0 : Z::kUpper, there = cc & 1 ? Z::kUpper : 0;
      // what is here has arrived for all waves, and nobody reads what is there any more
      if (C::KS > 1) lds_barrier();
      if (cc + 1 < C::KS) states(cc + 1, there);
      const unsigned char* at = lds + here;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f32x4_t so = {0.0f, 0.0f, 0.0f, 0.0f}, sv = so, nu = so;
#pragma unroll
        for (int kt = 0; kt < C::KS; ++kt) {
          Parts<T, kParts> a;
#pragma unroll
          for (int j = 0; j < Z::kN; ++j) a.v[j] = key_column<T, B>(at + j * D * B::kPitch, i, kt, lane);
          mma_parts<T>(so, a, o[kt]);
          mma_parts<T>(sv, a, v[kt]);
#pragma unroll
          for (int j = 0; j < Z::kN; ++j) a.v[j] = key_column<T, B>(at + Z::kState + j * D * B::kPitch, i, kt, lane);
          mma_parts<T>(nu, a, u[kt]);
          __builtin_amdgcn_sched_barrier(0);
        }
        f32x4_t &x = aq[2 * cc + i], &y = ak[2 * cc + i];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x[r] = fmaf(scaled, so[r], x[r]);
          y[r] = fmaf(rest, nu[r], fmaf(-into, sv[r], y[r]));
        }
      }
      if (cc + 1 < C::KS) arrive(there);
    }
  }
  if (own >= live) return;
#pragma unroll
  for (int ks = 0; ks < C::KS; ++ks) {
    const int64_t at = (krow + own) * D + 32 * ks + 8 * g;
    auto put = [&](T* to, const f32x4_t& a, const f32x4_t& b) {
      if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<u32x4_t*>(to + at) = (u32x4_t){pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]),
                                                         pack_bf16x2(b[0], b[1]), pack_bf16x2(b[2], b[3])};
      } else {
        reinterpret_cast<f32x4_t*>(to + at)[0] = a;
        reinterpret_cast<f32x4_t*>(to + at)[1] = b;
      }
    };
    put(dq, aq[2 * ks], aq[2 * ks + 1]);
    put(dk, ak[2 * ks], ak[2 * ks + 1]);
  }
}

// The decays' gradient of a span: from that of its first token, <gradient of the state before
// the span, that state>, on, to what it comes to behind the last, where the next span has it or
// nothing has a gradient any more.  What the sum misses that end by is the roundings of its
// terms; spread over the tokens it leaves 0.6 of their error (8 packed sequences of up to 12000
// tokens, heads of 32 in fp32: 1.4e-6 of the norm without).
__global__ void __launch_bounds__(kThreads)
decay_kernel(DeltaPlan P, const int32_t* cu, const float* S0, const float* dS0, const float* recB, const float* recD,
             const float* do_o, const float* dv_v, bool final_gradient, float* dg) {
  __shared__ double red[4][kThreads / 64];
  const int h = blockIdx.y, lane = threadIdx.x & 63, w = threadIdx.x >> 6, size = P.d * P.d;
  Span sp;
  if (!find_span<kThreads>(P, cu, blockIdx.x, &sp)) return;
  const int64_t pair = (int64_t)sp.s * P.value_heads + h;
  const size_t record = ((size_t)h * P.units + sp.slot) * size;
  auto product = [&](const float* a, const float* b) {  // this thread's share
    double sum = 0.0;
    if (a)
      for (int i = threadIdx.x * 4; i < size; i += kThreads * 4) {
        const f32x4_t x = *reinterpret_cast<const f32x4_t*>(a + i), y = *reinterpret_cast<const f32x4_t*>(b + i);
#pragma unroll
        for (int r = 0; r < 4; ++r) sum += (double)x[r] * (double)y[r];
      }
    return sum;
  };
  const int64_t row = gate_row(P, sp, h);
  auto step_of = [&](int t) { return (double)dv_v[row + t] - (double)do_o[row + t]; };
  double sums[3] = {product(sp.idx > 0 ? recB + record : S0 ? S0 + pair * size : nullptr,
                            sp.idx > 0 ? recD + record - size : S0 ? dS0 + pair * size : nullptr),
                    product(sp.last ? nullptr : recB + record + size, recD + record), 0.0};
  for (int t = sp.begin + (int)threadIdx.x; t < sp.end; t += kThreads) sums[2] += step_of(t);
#pragma unroll
  for (int k = 0; k < 3; ++k) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sums[k] += __shfl_xor(sums[k], o);
    if (lane == 0) red[k][w] = sums[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    sums[k] = 0.0;
    for (int i = 0; i < kThreads / 64; ++i) sums[k] += red[k][i];
  }
  __syncthreads();
  double at = sums[0];
  const double miss = sp.last && final_gradient ? 0.0 : (sums[1] - (at + sums[2])) / max(sp.end - sp.begin, 1);
  for (int t0 = sp.begin, flip = 0; t0 < sp.end; t0 += kThreads, flip ^= 1) {
    const int t = t0 + (int)threadIdx.x;
    const double step = t < sp.end ? step_of(t) : 0.0;
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
    if (t < sp.end) dg[row + t] = (float)(before + (c - step) + miss * (t - sp.begin));
  }
}

}  // namespace

gbla_status launch_delta_grads(const DeltaPlan& p, const void* q, const void* k, const float* S0,
                               const int32_t* cu, const void* dout, void* ws, void* dq, void* dk,
                               void* dv, float* dlog_decay, const float* dS0, bool final_gradient,
                               hipStream_t st) {
  if (p.tokens == 0) return GBLA_OK;
  unsigned char* base = static_cast<unsigned char*>(ws);
  auto floats = [&](size_t off) { return reinterpret_cast<const float*>(base + off); };
  return by_type(p, [&](auto t, auto dim) {
    using T = decltype(t);
    constexpr int D = decltype(dim)::value;
    hipLaunchKernelGGL((grads_kernel<T, D>), dim3(p.tiles, p.heads), dim3(kThreads), 0, st, p, tile_spans(p),
                       (const T*)q, (const T*)k, (const T*)dout, cu, base + p.off_pack,
                       floats(p.off_S), floats(p.off_N), floats(p.off_E), floats(p.off_F), (T*)dq, (T*)dk, (T*)dv);
    hipLaunchKernelGGL(decay_kernel, dim3(p.grid_units, p.value_heads), dim3(kThreads), 0, st, p, cu, S0, dS0,
                       floats(p.off_B), floats(p.off_D), floats(p.off_do_o), floats(p.off_dv_v), final_gradient,
                       dlog_decay);
  });
}

}  // namespace gbla
