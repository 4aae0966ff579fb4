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
// and of log_decay, by tiles (pairs_kernel) and joined over them (decay_kernel).
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
// heads of 64: 103 us; 58000 packed tokens, 8 heads of 128: 450.  (Every wave gathering and
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

// The decays' gradient, dg_t = <dZ_t, Z_t>, as the sum of the terms that pass token t's decay and
// of no others, so that it is as accurate where the decay is strong as where it is not:
//   sum_{s < t <= r} A_rs + sum_{r >= t} B_r + sum_{s < t} C_s + W
//   A_rs = D_rs (scale (q_r k_s) (do_r u_s) - (k_r k_s) (dv_r u_s))          within the tile
//   B_r  = e^c_r (scale do_r S^T q_r - dv_r S^T k_r)     from the state before it (the walk's)
//   C_s  = e^(c_L - c_s) k_s^T N u_s                      to the state after it (the walk's)
//   W    = e^c_L <S, N>                                   over all of it
// (The difference of neighbours, dv_t v_t - do_t o_t, holds the token's own pair, which no decay
// makes smaller: summed over the tokens its roundings were 3e-4 of the gradient at decays of
// e^-8, and all of it at e^-30.)
//
// W comes of <S, N> at the ends of a span of tiles (decay_kernel), off by 2^-24 of the gradients
// about it.  That is little beside what a token of the tile has of its neighbours, which is of the
// size of its own decay, unless that is below 2^-8: then the tile's W is the product of the states
// as the walks left them (bf16: in two parts, 2^-17 of it each).  Without such a token a W below
// 2^-64 is taken as nothing.  (The states of every tile would be 128 KB more to read at heads of
// 128: 60000 packed tokens, 8 heads, 2395 us a backward; 2505 with a forgetting token among 50.)
//
// Bound by HBM and the wait for it: 56 KB a tile at heads of 64, 8 x 2048 tokens, 16 heads: 62 us
// (3.7 TB/s); 112 KB at heads of 128, 58000 packed tokens, 8 heads: 186 us (4.4).  E and F both in
// LDS: 78 and 282; neither, with branches between the blocks: 88 and 281; as a phase of the
// gradients' kernel, which has both: 72 and 370 more.
constexpr float kDirectStep = -8.0f;  // log2
constexpr float kNothing = 0x1p-64f;

// Thread's share of <S, N> of two states as store_columns leaves them.
template <typename T, int D>
__device__ __forceinline__ float states_product(const float* S, const float* N) {
  const u32x4_t *s = reinterpret_cast<const u32x4_t*>(S), *n = reinterpret_cast<const u32x4_t*>(N);
  float sum = 0.0f;
  if constexpr (sizeof(T) == 2) {
    for (int i = threadIdx.x; i < D * D / 8; i += kThreads) {
      const int at = i / (4 * D) * (8 * D) + i % (4 * D);  // of the first parts; 4 D on, the second
      const u32x4_t a = s[at], b = s[at + 4 * D], c = n[at], d = n[at + 4 * D];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        sum = fmaf(bf16_lo(a[j]) + bf16_lo(b[j]), bf16_lo(c[j]) + bf16_lo(d[j]), sum);
        sum = fmaf(bf16_hi(a[j]) + bf16_hi(b[j]), bf16_hi(c[j]) + bf16_hi(d[j]), sum);
      }
    }
  } else {
    for (int i = threadIdx.x; i < D * D / 4; i += kThreads) {
      const u32x4_t a = s[i], c = n[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) sum = fmaf(__uint_as_float(a[j]), __uint_as_float(c[j]), sum);
    }
  }
  return sum;
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// A tile of a value head: what its tokens have but W.  Wave w has the later tokens 16 w .. (which
// wave that is goes around, as in prep_kernel) and sums over the earlier ones in its registers.  E,
// which all waves need, goes straight into LDS in fp32, [value channel][token] (16-byte units of a
// row at u ^ (row / 8 % 4 * 4): the four rows that a wave reads at once lie in different banks);
// E and F enter the products in three parts (bf16).
template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 3)
pairs_kernel(DeltaPlan P, TileSpans tiles, const T* q, const T* k, const T* dout, const int32_t* cu,
             const unsigned char* packs, const float* S, const float* N, const float* E, const float* F,
             const float* from, const float* on, DeltaTileSums* sums, float* dg) {
  using C = DS<T, D, 4>;
  __shared__ __attribute__((aligned(512))) float lds[D][kDeltaTile];
  __shared__ __attribute__((aligned(16))) float gates[3][kDeltaTile];
  __shared__ float passing[4][kDeltaTile];
  __shared__ double product[4];
  Span sp;
  if (!find_span<kThreads>(tiles, cu, blockIdx.x, &sp)) return;
  const int live = sp.end - sp.begin;
  if (live <= 0) return;
  const int h = blockIdx.y, lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(((threadIdx.x >> 6) + blockIdx.x) & 3);
  const size_t slot = (size_t)h * P.tiles + sp.slot;
  const Gates& G = *reinterpret_cast<const Gates*>(packs + slot * Packed<T, 3>::kBlock + Packed<T, 3>::kBytes);
  // (loaded without a condition, under which they would be waited for)
  const int64_t at = gate_row(P, sp, h) + sp.begin + min(lane, live - 1);
  const float hi = G.hi[lane], lo = G.lo[lane], beta = G.beta[lane], whole = G.whole;
  const float ends = from[at], begins = on[at];
  {
    const uint32_t at_lds = lds_address(lds);
    const u32x4_t r = rsrc_sgprs(E + slot * (D * kDeltaTile), D * kDeltaTile * 4);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      const int piece = 4 * i + w, row = 4 * piece + g;
      dma16(r, at_lds + 1024 * piece, (uint32_t)(row * 256 + ((n ^ ((row >> 3 & 3) << 2)) * 16)));
    }
  }
  const int64_t krow = first_row(P, sp, P.heads, h / P.group) + sp.begin,
                vrow = first_row(P, sp, P.value_heads, h) + sp.begin;
  const uint32_t bytes = (uint32_t)(live * C::kRow);
  const __amdgpu_buffer_rsrc_t rq = make_rsrc(q + krow * D, bytes), rk = make_rsrc(k + krow * D, bytes),
                               ro = make_rsrc(dout + vrow * D, bytes);
  auto row = [&](const __amdgpu_buffer_rsrc_t& r, int t, int ks) {
    Parts<T, 1> o;
    const uint32_t at = (uint32_t)(t * C::kRow + (32 * ks + 8 * g) * C::ES);
    if constexpr (sizeof(T) == 2) {
      o.v[0] = __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0);
    } else {
      o.v[0].a = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0));
      o.v[0].b = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, at + 16, 0, 0));
    }
    return o;
  };
  const int own = 16 * w + n;
  f32x4_t qk[4], kk[4], ou[4], vu[4];  // products with the earlier tokens 16 b + 4 g + r
#pragma unroll
  for (int b = 0; b < 4; ++b) qk[b] = kk[b] = ou[b] = vu[b] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
  Parts<T, 1> own_o[C::KS];
  float own_f[C::KS][8];
#pragma unroll
  for (int ks = 0; ks < C::KS; ++ks) {
    own_o[ks] = row(ro, own, ks);
    const float* p = F + slot * (D * kDeltaTile) + (32 * ks + 8 * g) * kDeltaTile + own;
#pragma unroll
    for (int j = 0; j < 8; ++j) own_f[ks][j] = p[j * kDeltaTile];
  }
  // (Each wave's row blocks without branches between them: their loads are under way at once.  The
  // last product's result is waited for here: the compiler left one wait state too few behind the
  // branches.)
  auto by_wave = [&](auto products) {
    auto f = [&](auto blocks) {
      products(blocks);
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_nop 10");
      __builtin_amdgcn_sched_barrier(0);
    };
    if (w == 0) f(std::integral_constant<int, 1>{});
    else if (w == 1) f(std::integral_constant<int, 2>{});
    else if (w == 2) f(std::integral_constant<int, 3>{});
    else f(std::integral_constant<int, 4>{});
  };
  by_wave([&](auto blocks) {
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) {
      const Parts<T, 1> own_q = row(rq, own, ks), own_k = row(rk, own, ks);
#pragma unroll
      for (int b = 0; b < decltype(blocks)::value; ++b) {
        const Parts<T, 1> keys = row(rk, 16 * b + n, ks);
        mma_parts<T>(qk[b], keys, own_q);
        mma_parts<T>(kk[b], keys, own_k);
      }
    }
  });
  if (threadIdx.x < kDeltaTile) gates[0][lane] = hi, gates[1][lane] = lo, gates[2][lane] = beta;
  wait_vm<0>();
  lds_barrier();
  by_wave([&](auto blocks) {
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) {
      Parts<T, 3> f, e;
      split(f, own_f[ks]);
#pragma unroll
      for (int b = 0; b < decltype(blocks)::value; ++b) {
        const float* p = &lds[32 * ks + 8 * g][(16 * b + n) ^ (16 * g)];
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = p[j * kDeltaTile];
        split(e, x);
        mma_parts<T>(ou[b], e, own_o[ks]);
        mma_parts<T>(vu[b], e, f);
      }
    }
  });
  const float own_hi = gates[0][own], own_lo = gates[1][own], own_beta = gates[2][own];
  // Of the own token r: sums of A_rs up to s, which are what token s + 1 has from r > s on.
  float x[16], before = 0.0f;
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const int s = 16 * b + 4 * g;
    const f32x4_t h4 = *reinterpret_cast<const f32x4_t*>(&gates[0][s]), l4 = *reinterpret_cast<const f32x4_t*>(&gates[1][s]),
                  b4 = *reinterpret_cast<const f32x4_t*>(&gates[2][s]);
    float part[4], sum = 0.0f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float f = __builtin_amdgcn_exp2f((own_hi - h4[r]) + (own_lo - l4[r])) * b4[r];
      const float a = f * (P.scale * qk[b][r] * ou[b][r] - own_beta * kk[b][r] * vu[b][r]);
      sum += s + r < own ? a : 0.0f;
      part[r] = sum;
    }
    // over the groups of lanes, which have the tokens in order
    float up = __shfl_up(sum, 16);
    sum += g >= 1 ? up : 0.0f;
    up = __shfl_up(sum, 32);
    sum += g >= 2 ? up : 0.0f;
    up = __shfl_up(sum, 16);
    const float first = before + (g >= 1 ? up : 0.0f);
#pragma unroll
    for (int r = 0; r < 4; ++r) x[4 * b + r] = s + r < own ? first + part[r] : 0.0f;
    before += __shfl(sum, 48 + n);
  }
  halve<8, 8>(x, lane);
  halve<4, 4>(x, lane);
  halve<2, 2>(x, lane);
  halve<1, 1>(x, lane);
  passing[w][16 * (n >> 2) + 4 * g + (n & 3)] = x[0];
  const float last_hi = __shfl_up(hi, 1), last_lo = __shfl_up(lo, 1);
  const float step = lane > 0 ? (hi - last_hi) + (lo - last_lo) : hi;
  const bool multiply = __ballot(step < kDirectStep) != 0 && whole > 0.0f;
  if (multiply) {
    const double share = wave_sum(states_product<T, D>(S + slot * (D * D), N + slot * (D * D)));
    if (lane == 0) product[w] = share;
  }
  __syncthreads();
  if (threadIdx.x >= kDeltaTile) return;
  double b = lane < live ? ends : 0.0f, c = lane < live ? begins : 0.0f;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double y = __shfl_down(b, o), z = __shfl_up(c, o);
    b += lane + o < 64 ? y : 0.0;
    c += lane >= o ? z : 0.0;
  }
  const double all_b = __shfl(b, 0), all_c = __shfl(c, 63), up = __shfl_up(c, 1);
  double sum = b + (lane > 0 ? up : 0.0);
  if (lane > 0)
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += passing[i][lane - 1];
  if (lane < live) dg[at] = (float)sum;
  if (lane == 0) {
    double over = 0.0;
    if (multiply) over = (double)whole * ((product[0] + product[1]) + (product[2] + product[3]));
    sums[slot] = {all_b, all_c, over, 0.0f, multiply || whole < kNothing};
  }
}

// W of a span's tiles, into their tokens' gradients.  With a_j = <S, N> at a tile's start, W_j =
// a_j - sum B and a_{j+1} = W_j + sum C: from the span's start on, where both states are at hand,
// and from every tile on whose W is known; and back from the span's end, where the next one
// has both (or nothing has a gradient any more).  Where both ways reach, either's error grows with
// its steps, and they are joined in that measure.
__global__ void __launch_bounds__(kThreads)
decay_kernel(DeltaPlan P, const int32_t* cu, const float* S0, const float* dS0, const float* recB, const float* recD,
             bool final_gradient, DeltaTileSums* sums, float* dg) {
  __shared__ double red[2][kThreads / 64];
  const int h = blockIdx.y, lane = threadIdx.x & 63, w = threadIdx.x >> 6, size = P.d * P.d;
  Span sp;
  if (!find_span<kThreads>(P, cu, blockIdx.x, &sp)) return;
  if (sp.begin >= sp.end) return;
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
    return wave_sum(sum);
  };
  const double shares[2] = {product(sp.idx > 0 ? recB + record : S0 ? S0 + pair * size : nullptr,
                                    sp.idx > 0 ? recD + record - size : S0 ? dS0 + pair * size : nullptr),
                            product(sp.last ? nullptr : recB + record + size, recD + record)};
  if (lane == 0) red[0][w] = shares[0], red[1][w] = shares[1];
  __syncthreads();
  const int count = (sp.end - sp.begin + kDeltaTile - 1) / kDeltaTile;
  DeltaTileSums* mine =
      sums + (size_t)h * P.tiles + tile_slot(P, sp.row0, sp.s) + sp.begin / kDeltaTile;
  if (w == 0) {
    // Sums that start anew at direct tiles, 64 tiles at a time, a lane a tile.
    double carry = (red[0][0] + red[0][1]) + (red[0][2] + red[0][3]);
    float steps = 0.0f;
    for (int j0 = 0; j0 < count; j0 += 64) {
      const bool in = j0 + lane < count;
      DeltaTileSums t = {};
      if (in) t = mine[j0 + lane];
      bool anew = in && t.direct;
      double v = anew ? t.over + t.on : t.on - t.from;
      float m = in && !anew ? 1.0f : 0.0f;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const double y = __shfl_up(v, o);
        const float z = __shfl_up(m, o);
        const bool other = __shfl_up((int)anew, o);
        if (lane >= o && !anew) v += y, m += z, anew = other;
      }
      if (!anew) v += carry, m += steps;
      double start = __shfl_up(v, 1);
      float from = __shfl_up(m, 1);
      if (lane == 0) start = carry, from = steps;
      if (!t.direct) t.over = start - t.from;
      t.steps = from;
      if (in) mine[j0 + lane] = t;
      carry = __shfl(v, 63), steps = __shfl(m, 63);
    }
    bool known = !(sp.last && final_gradient);
    carry = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
    steps = 0.0f;
    for (int j0 = (count - 1) / 64 * 64; j0 >= 0; j0 -= 64) {
      const bool in = j0 + lane < count;
      DeltaTileSums t = {};
      if (in) t = mine[j0 + lane];
      bool anew = in && t.direct;
      double v = anew ? t.over + t.from : t.from - t.on;
      float m = in && !anew ? 1.0f : 0.0f;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const double y = __shfl_down(v, o);
        const float z = __shfl_down(m, o);
        const bool other = __shfl_down((int)anew, o);
        if (lane + o < 64 && !anew) v += y, m += z, anew = other;
      }
      if (!anew) v += carry, m += steps;
      const bool there = anew || known;
      double end = __shfl_down(v, 1);
      float to = __shfl_down(m, 1);
      bool reached = __shfl_down((int)there, 1);
      if (lane == 63) end = carry, to = steps, reached = known;
      if (in && !t.direct && reached) {
        const double a = t.steps + 0.5f, b = to + 0.5f;
        mine[j0 + lane].over = (t.over * b + (end - t.on) * a) / (a + b);
      }
      carry = __shfl(v, 0), steps = __shfl(m, 0), known = __shfl((int)there, 0);
    }
  }
  __syncthreads();
  const int64_t row = gate_row(P, sp, h);
  for (int t = sp.begin + (int)threadIdx.x; t < sp.end; t += kThreads)
    dg[row + t] = (float)(dg[row + t] + mine[(t - sp.begin) / kDeltaTile].over);
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
    DeltaTileSums* sums = reinterpret_cast<DeltaTileSums*>(base + p.off_sums);
    hipLaunchKernelGGL((pairs_kernel<T, D>), dim3(p.tiles, p.value_heads), dim3(kThreads), 0, st, p, tile_spans(p),
                       (const T*)q, (const T*)k, (const T*)dout, cu, base + p.off_pack, floats(p.off_S),
                       floats(p.off_N), floats(p.off_E), floats(p.off_F), floats(p.off_from), floats(p.off_on), sums,
                       dlog_decay);
    hipLaunchKernelGGL(decay_kernel, dim3(p.grid_units, p.value_heads), dim3(kThreads), 0, st, p, cu, S0, dS0,
                       floats(p.off_B), floats(p.off_D), final_gradient, sums, dlog_decay);
  });
}

}  // namespace gbla
