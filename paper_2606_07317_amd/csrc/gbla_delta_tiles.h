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

// Sizes of a kernel of NWAVES waves.
template <typename T, int DIM, int NWAVES>
struct DS {
  static constexpr int D = DIM;
  static constexpr int NW = NWAVES;
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
  float late[kDeltaTile];  // that times beta
  float whole;             // decay over the tile
  int good;                // tokens before the first whose key or gates are not finite
  float pad[62];
};
static_assert(sizeof(Gates) == kGateBytes, "size of Gates");

// Eight consecutive values of an array in LDS.
__device__ __forceinline__ void eight(const float* p, float* x) {
  const f32x4_t a = *reinterpret_cast<const f32x4_t*>(p), b = *reinterpret_cast<const f32x4_t*>(p + 4);
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = a[j], x[4 + j] = b[j];
}
// x[j], a product of the tokens `own` and other + j, times `scale` and the decay between the two;
// zero where the other is not at or before (Before) / at or after it.  By selects: what is loaded
// under a condition is waited for one by one.
template <bool Before>
__device__ __forceinline__ void decayed(const Gates& G, int own, int other, float scale, float* x) {
  const float oh = G.hi[own], ol = G.lo[own];
  float hi[8], lo[8];
  eight(&G.hi[other], hi);
  eight(&G.lo[other], lo);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float away = (oh - hi[j]) + (ol - lo[j]);
    const float f = __builtin_amdgcn_exp2f(Before ? away : -away);
    const bool in = Before ? other + j <= own : other + j >= own;
    const float y = x[j] * (scale * f);
    x[j] = in ? y : 0.0f;
  }
}

// x - (the bf16 in the low / high half of h), exactly, for an h that rounds x: one instruction
// where unpacking and subtracting are two.  The factors (-1, 0) are kept in scalar registers:
// as an inline constant -1.0 stands for its fp32 bits, whose high half is the factor.
__device__ __forceinline__ float rest_lo(uint32_t h, float x) {
  uint32_t f = 0x0000bf80u;
  asm("" : "+s"(f));
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, h), __builtin_bit_cast(bf16x2_t, f), x, false);
}
__device__ __forceinline__ float rest_hi(uint32_t h, float x) {
  uint32_t f = 0xbf800000u;
  asm("" : "+s"(f));
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, h), __builtin_bit_cast(bf16x2_t, f), x, false);
}
// Eight fp32 values as an operand in N parts.
template <typename T, int N>
__device__ __forceinline__ void split(Parts<T, N>& p, const float* x) {
  if constexpr (sizeof(T) == 4) {
    p.set(x);
  } else {
    // (part by part: a dot product's result is used several instructions later)
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = x[j];
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) p.v[i][j] = pack_bf16x2(y[2 * j], y[2 * j + 1]);
      if (i + 1 < N) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          y[2 * j] = rest_lo(p.v[i][j], y[2 * j]);
          y[2 * j + 1] = rest_hi(p.v[i][j], y[2 * j + 1]);
        }
      }
    }
  }
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
    // one added to exponents that are all ones carries out of them
    constexpr uint32_t kExponents = sizeof(T) == 2 ? 0x7f807f80u : 0x7f800000u;
    constexpr uint32_t kOnes = sizeof(T) == 2 ? 0x00800080u : 0x00800000u;
    constexpr uint32_t kCarries = sizeof(T) == 2 ? 0x80008000u : 0x80000000u;
    uint32_t bad[N], any = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      bad[i] = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) bad[i] |= (x[i][j] & kExponents) + kOnes;
      any |= bad[i];
    }
    if (__builtin_expect(__ballot((any & kCarries) != 0) != 0, 0)) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (bad[i] & kCarries) atomicMin(first, (i * C::NT + (int)threadIdx.x) / per);
    }
  }
};

// A tile's rows, and `bytes` of a block, straight from memory to LDS (bf16: its tiles' rows lie
// next to each other there): a kilobyte an instruction, the waves in turn.  What they load has
// arrived once its waves have waited for all of their loads and met at a barrier.
template <typename T, typename C, int Rows = kDeltaTile>
__device__ __forceinline__ void rows_to_lds(uint32_t lds, const T* first, int live, int w, int lane) {
  constexpr int per = C::kRow / 16, step = 64 / per;  // units of a row, rows of an instruction
  const int rows = live < 0 ? 0 : live > Rows ? Rows : live;
  const u32x4_t r = rsrc_sgprs(first, (uint32_t)(rows * C::kRow));
#pragma unroll
  for (int i = 0; i < Rows / step / C::NW; ++i) {
    const int at = i * C::NW + w, row = at * step + lane / per;
    dma16(r, lds + 1024 * at, (uint32_t)(row * C::kRow + ((lane % per) ^ C::swizzle(row)) * 16));
  }
}
template <typename C, int Bytes>
__device__ __forceinline__ void block_to_lds(uint32_t lds, const void* from, bool any, int w, int lane) {
  static_assert(Bytes % 1024 == 0, "whole instructions");
  const u32x4_t r = rsrc_sgprs(from, any ? (uint32_t)Bytes : 0u);
#pragma unroll
  for (int i = 0; i < (Bytes / 1024 + C::NW - 1) / C::NW; ++i) {
    const int at = i * C::NW + w;
    if (at < Bytes / 1024) dma16(r, lds + 1024 * at, (uint32_t)(1024 * at + 16 * lane));
  }
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p);
}

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
  static constexpr int kBlock = kBytes + kGateBytes;  // with the tile's gates behind it
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

// Eight values of a column, tokens t .. t + 7: from the first that is not finite on they become
// zeros, and *first is lowered to its token.
template <typename T>
__device__ __forceinline__ void drop_bad(typename Num<T>::V8& v, int t, int* first) {
  float x[8];
  Num<T>::widen(v, x);
  float z = 0.0f;  // stays 0 while all are finite
#pragma unroll
  for (int j = 0; j < 8; ++j) z = fmaf(x[j], 0.0f, z);
  if (__builtin_expect(__ballot(z != 0.0f) != 0, 0)) {
    int bad = 8;
#pragma unroll
    for (int j = 7; j >= 0; --j) bad = isfinite(x[j]) ? bad : j;
    if (bad < 8) atomicMin(first, t + bad);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < bad ? x[j] : 0.0f;
    Parts<T, 1> p;
    p.set(x);
    v = p.v[0];
  }
}

// x[b] += the packed lower triangle's rows of block b times `by` (Swapped: by's transpose times
// theirs).  One operand ahead: more cost registers, none the wait for LDS.
template <typename T, int N, bool Swapped>
__device__ __forceinline__ void triangle(f32x4_t (&x)[4], const unsigned char* pack, const Parts<T, N> (&by)[2],
                                         int lane) {
  Parts<T, N> next = Packed<T, N>::get(pack, 0, lane);
#pragma unroll
  for (int pair = 0; pair < 6; ++pair) {
    const int b = pair < 2 ? pair : 2 + (pair >> 2), ks = pair < 2 ? 0 : pair & 1;
    const Parts<T, N> m = next;
    if (pair < 5) next = Packed<T, N>::get(pack, pair + 1, lane);
    if constexpr (Swapped) mma_parts<T>(x[b], by[ks], m);
    else mma_parts<T>(x[b], m, by[ks]);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// A tile's packed triangle and gates on their way to LDS.
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

// A wave's column block of a state X[key channel][value channel] in fp32: s[i][r] is row
// row_of(i, 4 g + r), column col0 + n.
template <typename T, typename C>
struct Columns16 {
  f32x4_t s[C::NB];
  __device__ __forceinline__ void fill(float x) {
#pragma unroll
    for (int i = 0; i < C::NB; ++i) s[i] = (f32x4_t){x, x, x, x};
  }
  __device__ __forceinline__ void identity(int col0, int lane) {
#pragma unroll
    for (int i = 0; i < C::NB; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) s[i][r] = row_of(i, 4 * (lane >> 4) + r) == col0 + (lane & 15) ? 1.0f : 0.0f;
  }
  // m: [row][column]
  __device__ __forceinline__ void load(const float* m, int col0, int lane) {
#pragma unroll
    for (int i = 0; i < C::NB; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) s[i][r] = m[row_of(i, 4 * (lane >> 4) + r) * C::D + col0 + (lane & 15)];
  }
  __device__ __forceinline__ void store(float* m, int col0, int lane) const {
#pragma unroll
    for (int i = 0; i < C::NB; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) m[row_of(i, 4 * (lane >> 4) + r) * C::D + col0 + (lane & 15)] = s[i][r];
  }
  // Records between launches hold four rows of a column in 16 bytes, as the waves that load
  // them have them: [block of 16 columns][row / 4][column][row % 4].
  __device__ __forceinline__ void load_record(const float* m, int col0, int lane) {
    const f32x4_t* p = reinterpret_cast<const f32x4_t*>(m + col0 * C::D) + (lane & 15);
#pragma unroll
    for (int i = 0; i < C::NB; ++i) s[i] = p[4 * row_of(i, 4 * (lane >> 4))];
  }
  __device__ __forceinline__ void store_record(float* m, int col0, int lane) const {
    f32x4_t* p = reinterpret_cast<f32x4_t*>(m + col0 * C::D) + (lane & 15);
#pragma unroll
    for (int i = 0; i < C::NB; ++i) p[4 * row_of(i, 4 * (lane >> 4))] = s[i];
  }
  // The transpose's record.
  __device__ __forceinline__ void store_transposed(float* m, int col0, int lane) const {
    const int col = col0 + (lane & 15);
#pragma unroll
    for (int i = 0; i < C::NB; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = row_of(i, 4 * (lane >> 4) + r);
        m[(row & ~15) * C::D + ((col >> 2) * 16 + (row & 15)) * 4 + (col & 3)] = s[i][r];
      }
  }
  // K step ks as an operand.
  template <int N>
  __device__ __forceinline__ Parts<T, N> operand(int ks) const {
    const f32x4_t &a = s[2 * ks], &b = s[2 * ks + 1];
    const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    Parts<T, N> p;
    split(p, x);
    return p;
  }
};

// K step ks of a state's column block for the gradients' kernel, into m of D * D words.  bf16: the
// first two parts, [ks][part][column][32 rows], so that a wave writes a kilobyte on end and 32
// rows are read as one block; fp32: [column][row].
template <typename T, typename C, int N>
__device__ __forceinline__ void store_columns(float* m, int ks, int col0, int lane, const Parts<T, N>& p) {
  const int col = col0 + (lane & 15), g = lane >> 4;
  if constexpr (sizeof(T) == 2) {
    u32x4_t* to = reinterpret_cast<u32x4_t*>(m) + (2 * ks * C::D + col) * 4 + g;
    to[0] = p.v[0];
    to[4 * C::D] = p.v[1];
  } else {
    f32x4_t* to = reinterpret_cast<f32x4_t*>(m + col * C::D + 32 * ks + 8 * g);
    to[0] = p.v[0].a;
    to[1] = p.v[0].b;
  }
}

// by[ks] = f times y's values of the tokens 32 ks + 8 g + j, in N parts.
template <typename T, int N>
__device__ __forceinline__ void weighted(Parts<T, N>& by, const float* f, const f32x4_t& a, const f32x4_t& b) {
  float x[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = f[j] * a[j], x[4 + j] = f[4 + j] * b[j];
  split(by, x);
}

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
