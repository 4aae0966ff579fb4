// gbla_decay_tiles.h -- device helpers of the decay attention's kernels: tiles of
// 64 tokens, their operands and products on the matrix instructions.
//
// All products of a tile are 16 x 16 blocks over K steps of 32.  A lane (n, g) =
// (lane & 15, lane >> 4) holds eight values of an operand's row or column n:
//   natural order  k = 32 ks + 8 g + j           (rows read as they lie)
//   split order    k = 32 ks + 4 g + j and 32 ks + 16 + 4 g + j, j < 4
// The result of a product has rows 4 g + i of column n, so two results one above
// the other are, in the same registers, an operand in split order: the scores of a
// tile go from the first product to the second without LDS.  That needs the scores
// as [earlier tokens] x [a wave's own 16 tokens], so results are formed transposed,
// [channels] x [tokens].
//
// bf16 operands are exact; operands that the kernels compute in fp32 enter as the
// sum of one to three bf16 parts (8 significant bits each).  fp32 operands use
// v_mfma_f32_16x16x4_f32, eight to a K step.
//
// Tiles in LDS: [token][D], rows D elements and 16 bytes apart, so that sixteen rows
// of a 16-byte column start on sixteen different groups of four banks.
#pragma once

#include <math.h>

#include "gbla_decay.h"
#include "gbla_device.h"
#include "gbla_split.h"

namespace gbla {

struct F8 {
  f32x4_t a, b;
};

template <typename T>
struct Num;

template <>
struct Num<uint16_t> {
  using V8 = u32x4_t;
  static __device__ __forceinline__ V8 zero() { return (u32x4_t){0, 0, 0, 0}; }
  static __device__ __forceinline__ void mma(f32x4_t& c, const V8& a, const V8& b) { c = mfma_bf16(a, b, c); }
  static __device__ __forceinline__ void widen(const V8& v, float* x) {
#pragma unroll
    for (int p = 0; p < 4; ++p) x[2 * p] = bf16_lo(v[p]), x[2 * p + 1] = bf16_hi(v[p]);
  }
};

template <>
struct Num<float> {
  using V8 = F8;
  static __device__ __forceinline__ V8 zero() { return {{0, 0, 0, 0}, {0, 0, 0, 0}}; }
  static __device__ __forceinline__ void mma(f32x4_t& c, const V8& a, const V8& b) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.a[j], b.a[j], c, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.b[j], b.b[j], c, 0, 0, 0);
  }
  static __device__ __forceinline__ void widen(const V8& v, float* x) {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = v.a[j], x[4 + j] = v.b[j];
  }
};

// Eight fp32 values as an operand of N parts (fp32: one, exact).
template <typename T, int N>
struct Parts {
  static constexpr int kN = sizeof(T) == 2 ? N : 1;
  typename Num<T>::V8 v[kN];
  __device__ __forceinline__ void set(const float* x) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[0].a[j] = x[j], v[0].b[j] = x[4 + j];
    } else {
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        float a = x[2 * p], b = x[2 * p + 1];
#pragma unroll
        for (int i = 0; i < kN; ++i) {
          const uint32_t h = pack_bf16x2(a, b);
          v[i][p] = h;
          a -= bf16_lo(h);
          b -= bf16_hi(h);
        }
      }
    }
  }
  // c += A this, the smaller parts first
  __device__ __forceinline__ void mma_right(f32x4_t& c, const typename Num<T>::V8& a) const {
#pragma unroll
    for (int i = kN - 1; i >= 0; --i) Num<T>::mma(c, a, v[i]);
  }
};

template <typename T, int DIM>
struct DC {
  static constexpr int D = DIM;
  static constexpr int EH = D == 128 ? 2 : 1;  // groups of four waves, by the output's channels
  static constexpr int NW = 4 * EH;
  static constexpr int NT = 64 * NW;
  static constexpr int ES = (int)sizeof(T);
  static constexpr int kRow = D * ES;          // bytes of a row in memory
  static constexpr int kPitch = kRow + 16;     // and in LDS
  static constexpr int kTileBytes = kTile * kPitch;
  static constexpr int KS = D / 32;            // K steps over channels
  static constexpr int NB = D / 16;            // 16-channel blocks
  static constexpr int OB = NB / EH;           // of a wave's output
  static constexpr int SB = NB * NB / NW;      // state blocks of a wave: one column block,
                                               // SB row blocks
  static constexpr int CH = kTile * kRow / 16 / NT;  // 16-byte pieces of a thread per tile
  // Planes of the state in LDS, [column][row]: two parts leave 2^-18 of a value,
  // far below the bf16 rounding of the results that they form.
  static constexpr int NP = ES == 2 ? 2 : 1;
  static constexpr int kPlane = D * kPitch;
  // A wave's state blocks: columns 16 cb .., rows 16 (rb + i) .., i < SB.
  static __device__ __forceinline__ int col_block(int w) { return D == 32 ? (w & 1) : w; }
  static __device__ __forceinline__ int row_block(int w) { return D == 32 ? (w >> 1) : 0; }
};

// exp(n g) for whole n >= 0: the product n g log2(e) in two parts, so that its
// error does not grow with it.
struct Decay {
  float hi, lo;
  __device__ __forceinline__ explicit Decay(float g) {
    g = g < -1e4f ? -1e4f : g;  // -inf: exp(0 g) is 1, all other powers 0; NaN stays
    const float l2 = 1.44269502162933349609f, l2lo = 1.92596299112661746887e-8f;
    hi = g * l2;
    lo = fmaf(g, l2, -hi) + g * l2lo;
  }
  __device__ __forceinline__ float operator()(int n) const {
    const float f = (float)n, x = f * hi;
    const float r = fmaf(f, hi, -x) + f * lo;
    return __builtin_amdgcn_exp2f(x) * fmaf(r, 0.69314718055994530942f, 1.0f);
  }
};

// s_waitcnt lgkmcnt(0); s_barrier: LDS is settled on both sides, and loads from
// memory that are still in flight stay in flight (a workgroup fence would wait for
// the next tile's).
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// A tile of a thread's 16-byte pieces on its way from memory to LDS; rows from
// `live` on are zeros.
template <typename C>
struct TileLoad {
  u32x4_t x[C::CH];
  __device__ __forceinline__ void load(const void* row0, int live) {
    const int rows = live < 0 ? 0 : live > kTile ? kTile : live;
    const __amdgpu_buffer_rsrc_t r = make_rsrc(row0, (uint32_t)(rows * C::kRow));
#pragma unroll
    for (int i = 0; i < C::CH; ++i)
      x[i] = __builtin_amdgcn_raw_buffer_load_b128(r, (uint32_t)(i * C::NT + threadIdx.x) * 16u, 0, 0);
  }
  __device__ __forceinline__ void store(unsigned char* lds) const {
    constexpr int per = C::kRow / 16;
#pragma unroll
    for (int i = 0; i < C::CH; ++i) {
      const int at = i * C::NT + threadIdx.x;
      *reinterpret_cast<u32x4_t*>(lds + (at / per) * C::kPitch + (at % per) * 16) = x[i];
    }
  }
};

// A wave's own sixteen rows as operands over channels (natural order): lane n's row.
template <typename T, typename C>
struct OwnRows {
  typename Num<T>::V8 v[C::KS];
  __device__ __forceinline__ void load(const void* row0, int live, int row, int g) {
    const int rows = live < 0 ? 0 : live > kTile ? kTile : live;
    const __amdgpu_buffer_rsrc_t r = make_rsrc(row0, (uint32_t)(rows * C::kRow));
    const uint32_t at = (uint32_t)(row * C::kRow + 8 * g * C::ES);
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) {
      const uint32_t o = at + (uint32_t)(32 * ks * C::ES);
      if constexpr (sizeof(T) == 2) {
        v[ks] = __builtin_amdgcn_raw_buffer_load_b128(r, o, 0, 0);
      } else {
        v[ks].a = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, o, 0, 0));
        v[ks].b = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, o + 16, 0, 0));
      }
    }
  }
};

// Row `row` of a tile in LDS, channels 32 ks + 8 g + j.
template <typename T, typename C>
__device__ __forceinline__ typename Num<T>::V8 row_at(const unsigned char* lds, int row, int ks, int g) {
  const unsigned char* p = lds + row * C::kPitch + (32 * ks + 8 * g) * C::ES;
  if constexpr (sizeof(T) == 2) return *reinterpret_cast<const u32x4_t*>(p);
  else return {*reinterpret_cast<const f32x4_t*>(p), *reinterpret_cast<const f32x4_t*>(p + 16)};
}

// Column 16 cb + n of a tile in LDS, rows 32 ks + .. in split or natural order.
template <typename T, typename C, bool Split>
__device__ __forceinline__ typename Num<T>::V8 col_at(const unsigned char* lds, int cb, int ks, int lane) {
  const int n = lane & 15, g = lane >> 4;
  const int r0 = 32 * ks + (Split ? 4 : 8) * g, r1 = r0 + (Split ? 16 : 4);
  if constexpr (sizeof(T) == 2) {
    const unsigned char* p = lds + (r0 + (n >> 2)) * C::kPitch + (16 * cb + 4 * (n & 3)) * 2;
    const u32x2_t u = tr_read16(p), w = tr_read16(p + (r1 - r0) * C::kPitch);
    return (u32x4_t){u[0], u[1], w[0], w[1]};
  } else {
    const float* p = reinterpret_cast<const float*>(lds + r0 * C::kPitch) + 16 * cb + n;
    const float* q = reinterpret_cast<const float*>(lds + r1 * C::kPitch) + 16 * cb + n;
    constexpr int P = C::kPitch / 4;
    return {{p[0], p[P], p[2 * P], p[3 * P]}, {q[0], q[P], q[2 * P], q[3 * P]}};
  }
}

// A wave's blocks of a state X[row][column] in fp32.
template <typename T, typename C>
struct State {
  f32x4_t s[C::SB];  // block i: rows 16 (rb + i) + 4 g + r, column 16 cb + n

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < C::SB; ++i) s[i] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
  }
  // from / to memory [row][column] (or [column][row])
  __device__ __forceinline__ void load(const float* m, bool transposed, int w, int lane) {
    const int col = 16 * C::col_block(w) + (lane & 15), row = 16 * C::row_block(w) + 4 * (lane >> 4);
    if (transposed) {
#pragma unroll
      for (int i = 0; i < C::SB; ++i)
        s[i] = *reinterpret_cast<const f32x4_t*>(m + (int64_t)col * C::D + row + 16 * i);
    } else {
#pragma unroll
      for (int i = 0; i < C::SB; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[i][r] = m[(row + 16 * i + r) * C::D + col];
    }
  }
  __device__ __forceinline__ void store(float* m, bool transposed, int w, int lane) const {
    const int col = 16 * C::col_block(w) + (lane & 15), row = 16 * C::row_block(w) + 4 * (lane >> 4);
    if (transposed) {
#pragma unroll
      for (int i = 0; i < C::SB; ++i)
        *reinterpret_cast<f32x4_t*>(m + (int64_t)col * C::D + row + 16 * i) = s[i];
    } else {
#pragma unroll
      for (int i = 0; i < C::SB; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) m[(row + 16 * i + r) * C::D + col] = s[i][r];
    }
  }
  // into the planes [column][row]
  __device__ __forceinline__ void to_planes(unsigned char* planes, int w, int lane) const {
    const int col = 16 * C::col_block(w) + (lane & 15), row = 16 * C::row_block(w) + 4 * (lane >> 4);
    unsigned char* p = planes + col * C::kPitch + row * C::ES;
#pragma unroll
    for (int i = 0; i < C::SB; ++i) {
      if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<f32x4_t*>(p + 16 * i * C::ES) = s[i];
      } else {
        const uint32_t h0 = pack_bf16x2(s[i][0], s[i][1]), h1 = pack_bf16x2(s[i][2], s[i][3]);
        *reinterpret_cast<u32x2_t*>(p + 16 * i * C::ES) = (u32x2_t){h0, h1};
        *reinterpret_cast<u32x2_t*>(p + 16 * i * C::ES + C::kPlane) =
            (u32x2_t){pack_bf16x2(s[i][0] - bf16_lo(h0), s[i][1] - bf16_hi(h0)),
                      pack_bf16x2(s[i][2] - bf16_lo(h1), s[i][3] - bf16_hi(h1))};
      }
    }
  }
  // s = f s + x
  __device__ __forceinline__ void advance(float f, const State& x) {
#pragma unroll
    for (int i = 0; i < C::SB; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) s[i][r] = fmaf(f, s[i][r], x.s[i][r]);
  }
  // += A^T (weights B) over a tile's tokens: rows are A's channels, columns B's.
  // weight[ks][j] belongs to token 32 ks + 8 g + j.  The weighted operand enters in
  // three parts, so the state has fp32's accuracy.
  __device__ __forceinline__ void add_products(const unsigned char* A, const unsigned char* B,
                                               const float (*weight)[8], int w, int lane) {
#pragma unroll
    for (int ks = 0; ks < kTile / 32; ++ks) {
      float x[8];
      Num<T>::widen(col_at<T, C, false>(B, C::col_block(w), ks, lane), x);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] *= weight[ks][j];
      Parts<T, 3> b;
      b.set(x);
#pragma unroll
      for (int i = 0; i < C::SB; ++i)
        b.mma_right(s[i], col_at<T, C, false>(A, C::row_block(w) + i, ks, lane));
    }
  }
};

// The unit (split) or sequence (single) of a workgroup: tokens [begin, end) of
// sequence s, whose first row is `row0` of a head's rows.
struct Span {
  int s, idx;           // sequence, unit in it
  int len, begin, end;  // tokens
  int64_t row0;         // packed row (ragged) or 0
  bool last;            // the sequence's last unit
  int slot;             // record slot of the workgroup's (first) unit
};

// Every thread of the workgroup must call it; false for the whole workgroup where
// there is none.
template <int NT>
__device__ __forceinline__ bool find_span(const DecayPlan& P, const int32_t* cu, int u, Span* o) {
  if (P.single) {
    o->s = u;
    o->idx = 0;
  } else if (P.ragged) {
    if (!locate_unit<NT>(cu, P.nseq, P.unit, u, &o->s, &o->idx)) return false;
  } else {
    o->s = u / P.units_per_seq;
    o->idx = u - o->s * P.units_per_seq;
  }
  if (P.ragged) {
    o->row0 = cu[o->s];
    o->len = cu[o->s + 1] - cu[o->s];
  } else {
    o->row0 = 0;
    o->len = P.rows;
  }
  o->begin = P.single ? 0 : o->idx * P.unit;
  o->end = P.single ? o->len : min(o->len, o->begin + P.unit);
  o->last = o->end >= o->len;
  o->slot = u;
  return true;
}

// Row of token t of span s in head h (of `heads`), in elements of a [.., D] tensor.
__device__ __forceinline__ int64_t row_of(const DecayPlan& P, const Span& s, int heads, int h, int t) {
  return (P.ragged ? (int64_t)h * P.rows + s.row0 : ((int64_t)s.s * heads + h) * P.rows) + t;
}

}  // namespace gbla
