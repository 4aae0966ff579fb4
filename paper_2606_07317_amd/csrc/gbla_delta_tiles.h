// gbla_delta_tiles.h -- device helpers of the gated delta rule's kernels: tiles of 64
// tokens, their operands and products on the matrix instructions.
//
// A wave owns 16 value channels (a column block) or a few such blocks, all 64 tokens of
// a tile and all key channels of the state.  Everything that one product hands to the
// next then stays in the wave's registers: with operands held as (n, g) = (lane & 15,
// lane >> 4), eight values k = 32 ks + 8 g + j of row or column n, and results as rows
// 4 g + r of column n, two results of 16 rows, whose rows are taken in the order
//   row_of(b, n) = 32 (b / 2) + 8 (n / 4) + 4 (b % 2) + n % 4,  b = 2 ks, 2 ks + 1,
// are in the same registers the operand of K step ks.  So rows of 16-row blocks are
// always taken in that order, tokens and key channels alike.
//
// Operands that the kernels compute in fp32 enter as sums of bf16 parts (8 significant
// bits each); fp32 inputs use v_mfma_f32_16x16x4_f32, eight to a K step.
#pragma once

#include "gbla_decay_tiles.h"
#include "gbla_delta.h"

namespace gbla {

__device__ __forceinline__ int row_of(int b, int n) {
  return 32 * (b >> 1) + 8 * (n >> 2) + 4 * (b & 1) + (n & 3);
}

// Sizes of a kernel of NWAVES waves that each own COLS column blocks.
template <typename T, int DIM, int NWAVES, int COLS>
struct DS {
  static constexpr int D = DIM;
  static constexpr int NW = NWAVES, CB = COLS;
  static constexpr int NT = 64 * NW;
  static constexpr int ES = (int)sizeof(T);
  static constexpr int kRow = D * ES;     // bytes of a row in memory
  static constexpr int KS = D / 32;       // K steps over channels
  static constexpr int NB = D / 16;       // row blocks of the state
  // A tile's rows in LDS.  Three kinds of reads meet there: 16 rows row_of(b, ..) of one
  // 16-byte unit; for 16 key channels row_of(i, ..) the transposed reads of four rows and
  // half of four units; for 16 value channels those of four rows and two units.  bf16 rows
  // store unit u at u ^ swizzle(r), which gives all sixteen accesses of the first two
  // different units of the 256 bytes that a cycle serves; fp32 rows are 16 bytes apart.
  static constexpr int kPitch = kRow + (ES == 2 ? 0 : 16);
  static constexpr int kTileBytes = kDeltaTile * kPitch;
  static __device__ __forceinline__ int swizzle(int r) {
    if constexpr (ES == 4) return 0;
    const int high = (r >> 3) & 3;
    if constexpr (D == 128) return ((r & 3) << 2) ^ high;
    else if constexpr (D == 64) return ((r << 1) & 4) ^ high;
    else return high;
  }
  static __device__ __forceinline__ int unit_at(int r, int u) { return r * kPitch + ((u ^ swizzle(r)) << 4); }
};

// What the tiles' kernels need of a tile's gates; tokens past the tile's end, or past one
// whose key or gates are not finite, have decay 1 and strength 0.
struct Gates {
  float hi[kDeltaTile], lo[kDeltaTile];  // log2 of the decay from the tile's start, in two parts
  float beta[kDeltaTile];
  float into[kDeltaTile];  // decay from the tile's start through the token
  float rest[kDeltaTile];  // decay from the token to the tile's end
  float whole;             // decay over the tile
  int good;                // tokens before the first whose key or gates are not finite
  float pad[62];
};
static_assert(sizeof(Gates) == kGateBytes, "size of Gates");

// decay from token s (of log2 hi, lo) to token t >= s
__device__ __forceinline__ float decay_between(const Gates& G, int t, float hi, float lo) {
  return __builtin_amdgcn_exp2f((G.hi[t] - hi) + (G.lo[t] - lo));
}

// c += a b of two operands in parts, the smaller products first; of products with a
// negligible part none.
template <typename T, int NA, int NB>
__device__ __forceinline__ void mma_parts(f32x4_t& c, const Parts<T, NA>& a, const Parts<T, NB>& b) {
  constexpr int A = Parts<T, NA>::kN, B = Parts<T, NB>::kN, most = (A > B ? A : B) - 1;
#pragma unroll
  for (int sum = most; sum >= 0; --sum)
#pragma unroll
    for (int i = 0; i < A; ++i)
      if (sum - i >= 0 && sum - i < B) Num<T>::mma(c, a.v[i], b.v[sum - i]);
}

// Row r of a tile in LDS, channels 32 ks + 8 g + j.
template <typename T, typename C>
__device__ __forceinline__ typename Num<T>::V8 row_units(const unsigned char* lds, int r, int ks, int g) {
  if constexpr (sizeof(T) == 2) {
    return *reinterpret_cast<const u32x4_t*>(lds + C::unit_at(r, 4 * ks + g));
  } else {
    const f32x4_t* p = reinterpret_cast<const f32x4_t*>(lds + C::unit_at(r, 8 * ks + 2 * g));
    return {p[0], p[1]};
  }
}

// Column `row_of(i, n)` of a tile in LDS, tokens 32 kt + 8 g + j.
template <typename T, typename C>
__device__ __forceinline__ typename Num<T>::V8 key_column(const unsigned char* lds, int i, int kt, int lane) {
  const int n = lane & 15, g = lane >> 4;
  if constexpr (sizeof(T) == 2) {
    const int r = 32 * kt + 8 * g + (n >> 2), u = 4 * (i >> 1) + (n & 3), half = 8 * (i & 1);
    const u32x2_t x = tr_read16(lds + C::unit_at(r, u) + half);
    const u32x2_t y = tr_read16(lds + C::unit_at(r + 4, u) + half);
    return (u32x4_t){x[0], x[1], y[0], y[1]};
  } else {
    constexpr int P = C::kPitch / 4;
    const float* p = reinterpret_cast<const float*>(lds) + (32 * kt + 8 * g) * P + row_of(i, n);
    return {{p[0], p[P], p[2 * P], p[3 * P]}, {p[4 * P], p[5 * P], p[6 * P], p[7 * P]}};
  }
}

// Column 16 cb + n of a tile in LDS, tokens 32 kt + 8 g + j.
template <typename T, typename C>
__device__ __forceinline__ typename Num<T>::V8 value_column(const unsigned char* lds, int cb, int kt, int lane) {
  const int n = lane & 15, g = lane >> 4;
  if constexpr (sizeof(T) == 2) {
    const int r = 32 * kt + 8 * g + (n >> 2), u = 2 * cb + ((n >> 1) & 1), half = 8 * (n & 1);
    const u32x2_t x = tr_read16(lds + C::unit_at(r, u) + half);
    const u32x2_t y = tr_read16(lds + C::unit_at(r + 4, u) + half);
    return (u32x4_t){x[0], x[1], y[0], y[1]};
  } else {
    constexpr int P = C::kPitch / 4;
    const float* p = reinterpret_cast<const float*>(lds) + (32 * kt + 8 * g) * P + 16 * cb + n;
    return {{p[0], p[P], p[2 * P], p[3 * P]}, {p[4 * P], p[5 * P], p[6 * P], p[7 * P]}};
  }
}

// A tile's rows on their way from memory to LDS, 16 bytes a piece; rows from `live` on are
// zeros.
template <typename T, typename C>
struct RowsLoad {
  static constexpr int per = C::kRow / 16, N = kDeltaTile * per / C::NT;
  u32x4_t x[N];
  __device__ __forceinline__ void load(const T* first, int live) {
    const int rows = live < 0 ? 0 : live > kDeltaTile ? kDeltaTile : live;
    const __amdgpu_buffer_rsrc_t r = make_rsrc(first, (uint32_t)(rows * C::kRow));
#pragma unroll
    for (int i = 0; i < N; ++i)
      x[i] = __builtin_amdgcn_raw_buffer_load_b128(r, (uint32_t)((i * C::NT + threadIdx.x) * 16), 0, 0);
  }
  __device__ __forceinline__ void store(unsigned char* lds) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = i * C::NT + threadIdx.x;
      *reinterpret_cast<u32x4_t*>(lds + C::unit_at(at / per, at % per)) = x[i];
    }
  }
  // Lowers *first to the row of this thread's first piece with an infinite or NaN value.
  __device__ __forceinline__ void find_bad(int* first) const {
    bool any = false;
    bool bad[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      bad[i] = false;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t w = x[i][j];
        if constexpr (sizeof(T) == 2) bad[i] |= (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
        else bad[i] |= (w & 0x7f800000u) == 0x7f800000u;
      }
      any |= bad[i];
    }
    if (__builtin_expect(__ballot(any) != 0, 0)) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (bad[i]) atomicMin(first, (i * C::NT + (int)threadIdx.x) / per);
    }
  }
};

// Rows from `from` on of a tile in LDS become zeros.
template <typename C>
__device__ __forceinline__ void clear_rows(unsigned char* lds, int from) {
  for (int at = from * C::kPitch + (int)threadIdx.x * 16; at < C::kTileBytes; at += C::NT * 16)
    *reinterpret_cast<u32x4_t*>(lds + at) = (u32x4_t){0, 0, 0, 0};
}

// A 64 x 64 lower (upper) triangle as operands: the six (row block b, K step ks) that are
// not all zero, each [pieces of 16 bytes][lane]: N bf16 parts, or eight fp32 values.
__device__ __forceinline__ int lower_pair(int b, int ks) { return b < 2 ? b : 2 * b - 2 + ks; }
__device__ __forceinline__ int upper_pair(int b, int ks) { return b < 2 ? 2 * b + ks : b + 2; }
template <typename T, int N>
struct Packed {
  static constexpr int kPieces = sizeof(T) == 2 ? N : 2;
  static constexpr int kBytes = 6 * kPieces * 64 * 16;
  static __device__ __forceinline__ Parts<T, N> get(const unsigned char* pack, int pair, int lane) {
    const u32x4_t* p = reinterpret_cast<const u32x4_t*>(pack) + pair * (64 * kPieces) + lane;
    Parts<T, N> x;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < N; ++i) x.v[i] = p[64 * i];
    } else {
      x.v[0] = {__builtin_bit_cast(f32x4_t, p[0]), __builtin_bit_cast(f32x4_t, p[64])};
    }
    return x;
  }
  static __device__ __forceinline__ void put(unsigned char* pack, int pair, int lane, const Parts<T, N>& x) {
    u32x4_t* p = reinterpret_cast<u32x4_t*>(pack) + pair * (64 * kPieces) + lane;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < N; ++i) p[64 * i] = x.v[i];
    } else {
      p[0] = __builtin_bit_cast(u32x4_t, x.v[0].a);
      p[64] = __builtin_bit_cast(u32x4_t, x.v[0].b);
    }
  }
};

// Copies of a tile's packed triangle and gates on their way to LDS.
template <typename C, int Bytes>
struct BlockLoad {
  static constexpr int N = (Bytes / 16 + C::NT - 1) / C::NT;
  u32x4_t x[N];
  __device__ __forceinline__ void load(const void* from, bool any) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc(from, any ? (uint32_t)Bytes : 0u);
#pragma unroll
    for (int i = 0; i < N; ++i)
      x[i] = __builtin_amdgcn_raw_buffer_load_b128(r, (uint32_t)((i * C::NT + threadIdx.x) * 16), 0, 0);
  }
  __device__ __forceinline__ void store(void* lds) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = i * C::NT + threadIdx.x;
      if (Bytes % (16 * C::NT) == 0 || at < Bytes / 16) reinterpret_cast<u32x4_t*>(lds)[at] = x[i];
    }
  }
};

// A wave's blocks of a state X[key channel][value channel] in fp32: s[c][i][r] is row
// row_of(i, 4 g + r), column 16 (cb0 + c) + n.
template <typename T, typename C>
struct Columns16 {
  f32x4_t s[C::CB][C::NB];
  __device__ __forceinline__ void fill(float x) {
#pragma unroll
    for (int c = 0; c < C::CB; ++c)
#pragma unroll
      for (int i = 0; i < C::NB; ++i) s[c][i] = (f32x4_t){x, x, x, x};
  }
  __device__ __forceinline__ void identity(int col0, int lane) {
#pragma unroll
    for (int c = 0; c < C::CB; ++c)
#pragma unroll
      for (int i = 0; i < C::NB; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          s[c][i][r] = row_of(i, 4 * (lane >> 4) + r) == col0 + 16 * c + (lane & 15) ? 1.0f : 0.0f;
  }
  // m: [row][column]
  __device__ __forceinline__ void load(const float* m, int col0, int lane) {
#pragma unroll
    for (int c = 0; c < C::CB; ++c)
#pragma unroll
      for (int i = 0; i < C::NB; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          s[c][i][r] = m[row_of(i, 4 * (lane >> 4) + r) * C::D + col0 + 16 * c + (lane & 15)];
  }
  __device__ __forceinline__ void store(float* m, int col0, int lane) const {
#pragma unroll
    for (int c = 0; c < C::CB; ++c)
#pragma unroll
      for (int i = 0; i < C::NB; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          m[row_of(i, 4 * (lane >> 4) + r) * C::D + col0 + 16 * c + (lane & 15)] = s[c][i][r];
  }
  // m: [column][row]
  __device__ __forceinline__ void store_columns(float* m, int col0, int lane) const {
#pragma unroll
    for (int c = 0; c < C::CB; ++c) {
      float* to = m + (col0 + 16 * c + (lane & 15)) * C::D + 8 * (lane >> 4);
#pragma unroll
      for (int i = 0; i < C::NB; ++i)
        *reinterpret_cast<f32x4_t*>(to + 32 * (i >> 1) + 4 * (i & 1)) = s[c][i];
    }
  }
  // K step ks of column block c as an operand.
  template <int N>
  __device__ __forceinline__ Parts<T, N> operand(int c, int ks) const {
    const f32x4_t &a = s[c][2 * ks], &b = s[c][2 * ks + 1];
    const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    Parts<T, N> p;
    p.set(x);
    return p;
  }
};

// Sums over a wave's 16 value channels (lanes n) of a lane's values of its 16 tokens, x[ks][j]
// of token 32 ks + 8 g + j: halving exchanges, after which lane n has token
// 32 (n / 8) + 8 g + n % 8's.
template <int W, int O>
__device__ __forceinline__ void halve(float* v, int lane) {
  const bool high = lane & O;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    const float keep = high ? v[i + W] : v[i], give = high ? v[i] : v[i + W];
    v[i] = keep + __shfl_xor(give, O);
  }
}
__device__ __forceinline__ float token_sums(float (&x)[2][8], int lane) {
  float* v = &x[0][0];
  halve<8, 8>(v, lane);
  halve<4, 4>(v, lane);
  halve<2, 2>(v, lane);
  halve<1, 1>(v, lane);
  return v[0];
}
__device__ __forceinline__ int token_of(int lane) { return 32 * ((lane >> 3) & 1) + 8 * (lane >> 4) + (lane & 7); }

// The tiles of a plan as spans of their own.
struct TileSpans {
  int32_t nseq, rows, ragged, single, unit, units_per_seq;
};
inline TileSpans tile_spans(const DeltaPlan& p) { return {p.nseq, p.rows, p.ragged, 0, kDeltaTile, p.tiles_per_seq}; }
// The slot of tile 0 of sequence s (packed: that starts at row c).
__device__ __forceinline__ int tile_slot(const DeltaPlan& P, int64_t c, int s) {
  return P.ragged ? (int)(c / kDeltaTile) + s : s * P.tiles_per_seq;
}
// A tile's gates [rows][tile] start: row of its first token in a [B,V,n] or [V,T] array.
__device__ __forceinline__ int64_t gate_row(const DeltaPlan& P, const Span& s, int h) {
  return P.ragged ? (int64_t)h * P.rows + s.row0 : ((int64_t)s.s * P.value_heads + h) * P.rows;
}

template <typename F>
inline gbla_status by_type(const DeltaPlan& p, F f) {
  auto dims = [&](auto t) {
    if (p.d == 32) f(t, std::integral_constant<int, 32>{});
    else if (p.d == 64) f(t, std::integral_constant<int, 64>{});
    else f(t, std::integral_constant<int, 128>{});
  };
  if (p.dtype == GBLA_BF16) dims(uint16_t{});
  else dims(float{});
  return hipGetLastError() == hipSuccess ? GBLA_OK : GBLA_ERR_HIP;
}

}  // namespace gbla
