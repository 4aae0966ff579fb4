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
// Tiles in LDS: [token][D].  Two kinds of reads meet there: 16 rows of one 16-byte unit
// (row_at) and columns (col_at; bf16 by transposed reads of four rows and two units a
// group of 16 lanes).  The walk's bf16 rows store unit u at u ^ swizzle(r), so that the
// rows that either reads at once fall on different banks (64 packed sequences, T = 177,929,
// d = 128, shared heads: 407 us a forward, 419 with rows 16 bytes apart).  The other
// kernels' rows are 16 bytes apart, since the swizzle's addresses cost registers that
// they do not have (16 packed sequences, T = 57,511, d = 128: 764 us a backward, 903 with
// swizzled keys, 782 with swizzled records), and fp32 rows, whose reads of single values
// that suits.
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
};

// A tile or plane in LDS: rows of W elements, swizzled or 16 bytes apart.
template <typename T, int W, bool Swizzled>
struct Lay {
  static constexpr int ES = (int)sizeof(T);
  static constexpr int kRow = W * ES;
  static constexpr bool kSwizzled = Swizzled && ES == 2;
  static constexpr int kPitch = kRow + (kSwizzled ? 0 : 16);
  // Rows 0-3 and 4-7, 8-11 and 12-15, 0-3 and 8-11, 4-7 and 12-15 (what a transposed
  // read takes at once, in either order) get different pairs of units, all sixteen rows
  // different units; as far as a row has them (W / 8 units).
  static constexpr int kShift = W == 128 ? 0 : W == 64 ? 1 : 2;
  static __device__ __forceinline__ int swizzle(int r) {
    if constexpr (!kSwizzled) return 0;
    return ((((r ^ ((r >> 1) & 4)) & 7) >> kShift) << 1) | ((r >> 3) & 1);
  }
  // Byte offset of the 16-byte unit u of row r.
  static __device__ __forceinline__ int unit_at(int r, int u) { return r * kPitch + ((u ^ swizzle(r)) << 4); }
};

// Sizes of a kernel of D channels: a workgroup of NWAVES waves with VD of the value
// channels, the state in PARTS bf16 parts for its products.
template <typename T, int DIM, int VDIM, int NWAVES, int PARTS, bool SWIZZLED>
struct DC {
  static constexpr int D = DIM;
  static constexpr int VD = VDIM;
  static constexpr int NW = NWAVES;
  static constexpr int EH = NW / 4;            // groups of four waves, by the output's channels
  static constexpr int NT = 64 * NW;
  static constexpr int ES = (int)sizeof(T);
  static constexpr int kRow = D * ES;          // bytes of a row in memory
  static constexpr int KS = D / 32;            // K steps over channels
  static constexpr int OB = VD / 16 / EH;      // 16-channel blocks of a wave's output
  // A wave's state blocks: one column block, SR row blocks.
  static constexpr int NBK = D / 16, NBV = VD / 16;
  static constexpr int SR = NBK * NBV / NW;
  using Wide = Lay<T, D, SWIZZLED>;                      // tiles of all channels, planes [column][row]
  using Slim = Lay<T, VD, SWIZZLED>;                     // tiles of the value channels
  static constexpr int NP = ES == 2 ? PARTS : 1;
  static constexpr int kPlane = VD * Wide::kPitch;
  static __device__ __forceinline__ int col_block(int w) { return w % NBV; }
  static __device__ __forceinline__ int row_block(int w) { return w / NBV * SR; }
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
  // exp(g) is 0: no state goes on, whatever it holds (wave-uniform).
  __device__ __forceinline__ bool forgets() const {
    return __builtin_amdgcn_readfirstlane(__float_as_int((*this)(1))) == 0;
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

// W channels of a tile, 16-byte pieces of a thread on their way from memory (rows of
// C::kRow bytes) to LDS; rows from `live` on are zeros.
template <typename T, typename C, int W>
struct TileLoad {
  using L = Lay<T, W, C::Wide::kSwizzled>;
  static constexpr int per = L::kRow / 16, N = kTile * per / C::NT;
  u32x4_t x[N];
  __device__ __forceinline__ void load(const void* first, int live) {
    const int rows = live < 0 ? 0 : live > kTile ? kTile : live;
    const __amdgpu_buffer_rsrc_t r =
        make_rsrc(first, rows > 0 ? (uint32_t)((rows - 1) * C::kRow + L::kRow) : 0u);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = i * C::NT + threadIdx.x;
      x[i] = __builtin_amdgcn_raw_buffer_load_b128(r, (uint32_t)((at / per) * C::kRow + (at % per) * 16), 0, 0);
    }
  }
  __device__ __forceinline__ void store(unsigned char* lds) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = i * C::NT + threadIdx.x;
      *reinterpret_cast<u32x4_t*>(lds + L::unit_at(at / per, at % per)) = x[i];
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

// The channels of a wave's own rows that its results have: c0 + 16 o + 4 g + r of lane
// n's row.
template <typename T, typename C>
struct OwnPieces {
  u32x4_t v[C::OB];
  __device__ __forceinline__ void load(const void* row0, int live, int row, int c0, int g) {
    const int rows = live < 0 ? 0 : live > kTile ? kTile : live;
    const __amdgpu_buffer_rsrc_t r = make_rsrc(row0, (uint32_t)(rows * C::kRow));
    const uint32_t at = (uint32_t)(row * C::kRow + (c0 + 4 * g) * C::ES);
#pragma unroll
    for (int o = 0; o < C::OB; ++o) {
      if constexpr (sizeof(T) == 2) {
        const u32x2_t x = __builtin_amdgcn_raw_buffer_load_b64(r, at + 16 * o * C::ES, 0, 0);
        v[o][0] = x[0];
        v[o][1] = x[1];
      } else {
        v[o] = __builtin_amdgcn_raw_buffer_load_b128(r, at + 16 * o * C::ES, 0, 0);
      }
    }
  }
  // sum over them of their products with a result
  __device__ __forceinline__ float dot(const f32x4_t* acc) const {
    float sum = 0.0f;
#pragma unroll
    for (int o = 0; o < C::OB; ++o)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float x = sizeof(T) == 4 ? __uint_as_float(v[o][r]) : r & 1 ? bf16_hi(v[o][r >> 1]) : bf16_lo(v[o][r >> 1]);
        sum = fmaf(x, acc[o][r], sum);
      }
    return sum;
  }
};

// A value that the compiler takes for a new one: addresses made from it are worked out
// where they are used, instead of being held in registers all through a loop.
__device__ __forceinline__ int fresh(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Row 16 b + n of a tile in LDS, channels 32 ks + 8 g + j.
template <typename T, typename L>
__device__ __forceinline__ typename Num<T>::V8 row_at(const unsigned char* lds, int b, int n, int ks, int g) {
  const unsigned char* p = lds + 16 * b * L::kPitch;  // row 16 b + n has row n's swizzle
  if constexpr (sizeof(T) == 2) {
    return *reinterpret_cast<const u32x4_t*>(p + L::unit_at(n, 4 * ks + g));
  } else {
    const f32x4_t* q = reinterpret_cast<const f32x4_t*>(p + L::unit_at(n, 8 * ks + 2 * g));
    return {q[0], q[1]};
  }
}

// Column 16 cb + n of a tile in LDS, rows 32 ks + .. in split or natural order.
template <typename T, typename L, bool Split>
__device__ __forceinline__ typename Num<T>::V8 col_at(const unsigned char* lds, int cb, int ks, int lane) {
  const int n = lane & 15, g = lane >> 4;
  const unsigned char* p = lds + 32 * ks * L::kPitch;
  const int r0 = (Split ? 4 : 8) * g;
  if constexpr (sizeof(T) == 2) {
    // four rows of 32 bytes a group of 16 lanes, lane n the (n & 3)-th 8 bytes of row
    // n / 4; 16 rows on the swizzle is the same, 4 rows on one bit of it is the other
    int at = L::unit_at(r0 + (n >> 2), (n >> 1) & 1) + 8 * (n & 1), next = at;
    if constexpr (L::kSwizzled) {
      at ^= cb << 5;
      next = Split ? at : at ^ (128 >> L::kShift);
    } else {
      at += cb << 5;
      next = at;
    }
    const u32x2_t x = tr_read16(p + at), y = tr_read16(p + (Split ? 16 : 4) * L::kPitch + next);
    return (u32x4_t){x[0], x[1], y[0], y[1]};
  } else {
    constexpr int P = L::kPitch / 4, next = (Split ? 16 : 4) * P;
    const float* q = reinterpret_cast<const float*>(p + r0 * L::kPitch) + 16 * cb + n;
    return {{q[0], q[P], q[2 * P], q[3 * P]}, {q[next], q[next + P], q[next + 2 * P], q[next + 3 * P]}};
  }
}

// Order of N products that each take one operand from LDS (by one read of 16 bytes in
// bf16, two in fp32), and M more beside which vector work goes on, two at a time with
// `pair` reads for the two in bf16: eight operands ahead, eight vector instructions after
// each two of the M.  Left to itself the compiler keeps one or two reads in flight, so
// that the wave waits for LDS before every product, and puts the vector work behind the
// products.
template <typename T, int N, int M, int Pair = 2>
__device__ __forceinline__ void pipeline() {
  constexpr int kValu = 0x2, kMfma = 0x8, kRead = 0x100;
  constexpr bool half = sizeof(T) == 2;
  constexpr int reads = half ? 1 : 2, mfmas = half ? 1 : 8;
  constexpr int pair = half ? Pair : Pair == 2 ? 4 : 16;
  __builtin_amdgcn_sched_group_barrier(kRead, 8 * reads, 0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_group_barrier(kMfma, mfmas, 0);
    __builtin_amdgcn_sched_group_barrier(kRead, reads, 0);
  }
#pragma unroll
  for (int i = 0; i < M / 2; ++i) {
    __builtin_amdgcn_sched_group_barrier(kMfma, 2 * mfmas, 0);
    if (i < M / 2 - 4) __builtin_amdgcn_sched_group_barrier(kRead, pair, 0);
    __builtin_amdgcn_sched_group_barrier(kValu, 8, 0);
  }
}

// Powers of the decay in LDS: up[i] = scale lam^(i+1); down[i] = lam^(63-i), zeros
// from 64 on, so that down + 64 - L holds the weights lam^(L-1-t) of a tile of L
// tokens and nothing for the rows behind it.
struct Powers {
  float up[kTile];
  float down[2 * kTile];
  __device__ __forceinline__ void fill(const Decay& lam, float scale) {
    const int i = threadIdx.x;
    if (i < kTile) {
      up[i] = scale * lam(i + 1);
      down[i] = lam(kTile - 1 - i);
      down[kTile + i] = 0.0f;
    }
  }
};

// A wave's blocks of a state X[row][column] in fp32; the workgroup's columns start at
// col0 of D.
template <typename T, typename C>
struct State {
  f32x4_t s[C::SR];  // block i: rows 16 (rb + i) + 4 g + r, column 16 cb + n

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < C::SR; ++i) s[i] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
  }
  // from / to memory [row][column] (or [column][row])
  __device__ __forceinline__ void load(const float* m, bool transposed, int col0, int w, int lane) {
    const int col = col0 + 16 * C::col_block(w) + (lane & 15), row = 16 * C::row_block(w) + 4 * (lane >> 4);
#pragma unroll
    for (int i = 0; i < C::SR; ++i) {
      if (transposed) {
        s[i] = *reinterpret_cast<const f32x4_t*>(m + col * C::D + row + 16 * i);
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) s[i][r] = m[(row + 16 * i + r) * C::D + col];
      }
    }
  }
  __device__ __forceinline__ void store(float* m, int col0, int w, int lane) const {
    const int col = col0 + 16 * C::col_block(w) + (lane & 15), row = 16 * C::row_block(w) + 4 * (lane >> 4);
#pragma unroll
    for (int i = 0; i < C::SR; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) m[(row + 16 * i + r) * C::D + col] = s[i][r];
  }
  // into the planes [the workgroup's column][row]
  __device__ __forceinline__ void to_planes(unsigned char* planes, int w, int lane) const {
    const int g = lane >> 4, col = 16 * C::col_block(w) + (lane & 15);
#pragma unroll
    for (int i = 0; i < C::SR; ++i) {
      const f32x4_t x = s[i];
      const int row = 16 * (C::row_block(w) + i) + 4 * g;
      if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<f32x4_t*>(planes + C::Wide::unit_at(col, row >> 2)) = x;
      } else {
        unsigned char* p = planes + C::Wide::unit_at(col, row >> 3) + 8 * (g & 1);
        f32x4_t rest = x;
#pragma unroll
        for (int j = 0; j < C::NP; ++j) {
          const uint32_t a = pack_bf16x2(rest[0], rest[1]), b = pack_bf16x2(rest[2], rest[3]);
          *reinterpret_cast<u32x2_t*>(p + j * C::kPlane) = (u32x2_t){a, b};
          rest -= (f32x4_t){bf16_lo(a), bf16_hi(a), bf16_lo(b), bf16_hi(b)};
        }
      }
    }
  }
  // s = f s + A^T (weight B) over a tile's tokens: rows are A's channels, columns
  // B's (its value channels), weight[t] token t's.  The weighted operand enters in three
  // parts and the tile's products are summed by themselves, so the state has fp32's
  // accuracy.
  __device__ __forceinline__ void advance(float f, const unsigned char* A, const unsigned char* B,
                                          const float* weight, int w, int lane) {
    Parts<T, 3> b[2];
#pragma unroll
    for (int ks = 0; ks < kTile / 32; ++ks) {
      float x[8];
      Num<T>::widen(col_at<T, typename C::Slim, true>(B, C::col_block(w), ks, lane), x);
      const float* p = weight + 32 * ks + 4 * (lane >> 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[j] *= p[j];
        x[4 + j] *= p[16 + j];
      }
      b[ks].set(x);
    }
    constexpr int G = C::SR < 4 ? C::SR : 4;  // blocks at a time, as independent chains
#pragma unroll
    for (int i0 = 0; i0 < C::SR; i0 += G) {
      f32x4_t x[G];
#pragma unroll
      for (int i = 0; i < G; ++i) x[i] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int ks = 0; ks < kTile / 32; ++ks) {
        typename Num<T>::V8 a[G];
#pragma unroll
        for (int i = 0; i < G; ++i)
          a[i] = col_at<T, typename C::Wide, true>(A, C::row_block(w) + i0 + i, ks, lane);
#pragma unroll
        for (int y = Parts<T, 3>::kN - 1; y >= 0; --y)
#pragma unroll
          for (int i = 0; i < G; ++i) Num<T>::mma(x[i], a[i], b[ks].v[y]);
      }
#pragma unroll
      for (int i = 0; i < G; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[i0 + i][r] = fmaf(f, s[i0 + i][r], x[i][r]);
    }
  }
};

// Decays of a wave's scores: scale lam^(distance) of row 16 b + 4 g + i and the
// wave's own token 16 tw + n.  Own tokens are the later ones (Later) or the earlier
// ones; pairs of the wrong order are zero.
template <bool Later>
struct Scores {
  float same[4], next[4], far[2];  // block tw; 16 tokens away; factors for 32 and 48
  __device__ __forceinline__ void fill(const Decay& lam, float scale, int n, int g) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = Later ? n - 4 * g - i : 4 * g + i - n;
      same[i] = scale * lam(max(0, d));
      next[i] = scale * lam(16 + d);
    }
    far[0] = lam(16);
    far[1] = lam(32);
  }
  // `away`: blocks between the rows' block and the own one, negative where all pairs
  // are of the wrong order.  Selects only: with branches here the compiler left one to
  // five wait states between the product that forms x and its first use, where seven
  // are due (and the results were wrong).
  __device__ __forceinline__ void apply(f32x4_t& x, int away, int n, int g) const {
    const float f = away <= 1 ? 1.0f : away == 2 ? far[0] : far[1];
    const bool near = away == 0, none = away < 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool wrong = Later ? 4 * g + i > n : 4 * g + i < n;
      const float w = near ? same[i] : next[i] * f;
      x[i] = none | (near & wrong) ? 0.0f : x[i] * w;
    }
  }
};

// acc += (rows of a tile, K step ks)^T scores, the scores of its two 16-row blocks
// [rows] x [own tokens], in N parts; the rows' blocks from block `first` on.
template <typename T, typename C, typename L, int N>
__device__ __forceinline__ void add_scored(f32x4_t* acc, const f32x4_t& a, const f32x4_t& b,
                                           const unsigned char* rows, int ks, int first, int lane) {
  const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  Parts<T, N> p;
  p.set(x);
  typename Num<T>::V8 v[C::OB];
#pragma unroll
  for (int o = 0; o < C::OB; ++o) v[o] = col_at<T, L, true>(rows, first + o, ks, lane);
#pragma unroll
  for (int y = Parts<T, N>::kN - 1; y >= 0; --y)
#pragma unroll
    for (int o = 0; o < C::OB; ++o) Num<T>::mma(acc[o], v[o], p.v[y]);
}

// Products with an infinite or NaN row of a tile give NaN to tokens that the row has no part
// in, since a pair of the wrong order enters as 0 times the row.  Results that are not finite
// though all that takes part in them is are therefore formed again, pair by pair; the others
// stay.  What follows serves that: single elements, in loops that hold few registers, which
// only such inputs reach.  Looking for them costs 0 to 2 % of a forward and none of a backward.

// z stays 0 while all of x is finite, and is NaN from then on.
template <int N>
__device__ __forceinline__ void watch(float& z, const f32x4_t* x) {
#pragma unroll
  for (int o = 0; o < N; ++o)
#pragma unroll
    for (int r = 0; r < 4; ++r) z = fmaf(x[o][r], 0.0f, z);
}
__device__ __forceinline__ bool seen(float z) { return __ballot(z != 0.0f) != 0; }
template <typename T>
__device__ __forceinline__ float widen1(T x) {
  if constexpr (sizeof(T) == 2) return __uint_as_float((uint32_t)x << 16);
  else return x;
}
template <typename T>
__device__ __forceinline__ T narrow1(float x) {
  if constexpr (sizeof(T) == 2) return (T)(pack_bf16x2(x, 0.0f) & 0xffffu);
  else return x;
}
// The four values that this lane has stored at p: all finite?  y where one is not.
template <typename T>
__device__ __forceinline__ bool finite4(const T* p) {
  return isfinite(widen1(p[0])) && isfinite(widen1(p[1])) && isfinite(widen1(p[2])) && isfinite(widen1(p[3]));
}
template <typename T>
__device__ __forceinline__ void mend4(T* p, const f32x4_t& y) {
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (!isfinite(widen1(p[r]))) p[r] = narrow1<T>(y[r]);
}
// Channel c of row r of a tile in LDS.
template <typename T, typename L>
__device__ __forceinline__ float tile_at(const unsigned char* lds, int r, int c) {
  constexpr int per = 16 / (int)sizeof(T);
  return widen1(reinterpret_cast<const T*>(lds + L::unit_at(r, c / per))[c % per]);
}
// X[row][column] from its planes.
template <typename T, typename C>
__device__ __forceinline__ float plane_at(const unsigned char* planes, int row, int col) {
  const float x = tile_at<T, typename C::Wide>(planes, col, row);
  float rest = 0.0f;
#pragma unroll
  for (int p = C::NP - 1; p > 0; --p) rest += tile_at<T, typename C::Wide>(planes + p * C::kPlane, col, row);
  return isfinite(x) ? x + rest : x;
}
// Sum of the products of two rows' channels; the four lanes of a row (g) take a quarter each.
template <int D, typename A, typename B>
__device__ __forceinline__ float row_dot(int g, A a, B b) {
  float sum = 0.0f;
#pragma unroll 2
  for (int c = D / 4 * g; c < D / 4 * (g + 1); ++c) sum = fmaf(a(c), b(c), sum);
  sum += __shfl_xor(sum, 16);
  return sum + __shfl_xor(sum, 32);
}

// Rows a lane at 16 bytes: a wave holds kRows of them.  For the heads without memory.
template <typename T, int D>
struct RowPieces {
  static constexpr int kPer = 16 / (int)sizeof(T), kLanes = D / kPer, kRows = 64 / kLanes;
  using Piece = float[kPer];
  static __device__ __forceinline__ void load(Piece x, const T* p) {
    const u32x4_t v = load16(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) x[2 * i] = bf16_lo(v[i]), x[2 * i + 1] = bf16_hi(v[i]);
      else x[i] = __uint_as_float(v[i]);
    }
  }
  static __device__ __forceinline__ void store(T* p, const Piece x) {
    u32x4_t v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) v[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
      else v[i] = __float_as_uint(x[i]);
    }
    *reinterpret_cast<u32x4_t*>(p) = v;
  }
  static __device__ __forceinline__ float dot(const Piece a, const Piece b) {
    float x = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) x = fmaf(a[i], b[i], x);
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1) x += __shfl_xor(x, o);
    return x;
  }
};

// 0 if `count` pieces of 16 bytes of a row are finite, else NaN; at(u): where piece u lies.
template <typename T, int D, typename At>
__device__ __forceinline__ float row_watch(int count, At at) {
  float z = 0.0f;
#pragma unroll 1
  for (int u = 0; u < count; ++u) {
    typename RowPieces<T, D>::Piece x;
    RowPieces<T, D>::load(x, at(u));
#pragma unroll
    for (int i = 0; i < RowPieces<T, D>::kPer; ++i) z = fmaf(x[i], 0.0f, z);
  }
  return z;
}
// The same for a row in memory that four lanes (g) share.
template <typename T, int D>
__device__ __forceinline__ bool shared_row_finite(const T* row, int g) {
  float z = row_watch<T, D>(RowPieces<T, D>::kLanes / 4,
                            [&](int u) { return row + D / 4 * g + u * RowPieces<T, D>::kPer; });
  z += __shfl_xor(z, 16);
  return z + __shfl_xor(z, 32) == 0.0f;
}
// Whether four values (stored at p) are to be formed again: not finite, though what takes part
// in them (watched by z) is.
template <typename T>
__device__ __forceinline__ bool wanted4(const T* p, const f32x4_t& z) {
  bool any = false;
#pragma unroll
  for (int r = 0; r < 4; ++r) any |= !isfinite(widen1(p[r])) && isfinite(z[r]);
  return any;
}

// The record slot of the first unit of a packed sequence that starts at row c: slots
// of different sequences never meet (the next starts at least ceil(len / unit) later),
// and no prefix sum over the lengths is needed.  The last slot is below T / unit + N.
template <typename Plan>
__device__ __forceinline__ int first_slot(const Plan& P, int c, int s) { return c / P.unit + s; }

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
// there is none (a slot that no unit has).
// Plan: any with DecayPlan's members of the split (single .. units_per_seq, rows, nseq, ragged).
template <int NT, typename Plan>
__device__ __forceinline__ bool find_span(const Plan& P, const int32_t* cu, int u, Span* o) {
  if (P.single) {
    o->s = u;
  } else if (P.ragged) {
    // The last sequence whose first slot is at most u (they increase), by rounds of NT
    // probes each: one round for up to NT sequences.
    __shared__ int found;
    int lo = 0, count = P.nseq;
    while (count > 1) {
      const int step = (count + NT - 1) / NT, end = lo + count;
      const int at = lo + (int)threadIdx.x * step;
      if (threadIdx.x == 0) found = lo;
      __syncthreads();
      if (at < end && first_slot(P, cu[at], at) <= u &&
          (at + step >= end || first_slot(P, cu[at + step], at + step) > u))
        found = at;
      __syncthreads();
      const int f = __builtin_amdgcn_readfirstlane(found);
      __syncthreads();  // read by all before the next round's write
      count = min(step, end - f);
      lo = f;
    }
    o->s = lo;
    if (u - first_slot(P, cu[lo], lo) >= units_of((int64_t)cu[lo + 1] - cu[lo], P.unit)) return false;
  } else {
    o->s = u / P.units_per_seq;
  }
  if (P.ragged) {
    o->row0 = cu[o->s];
    o->len = cu[o->s + 1] - cu[o->s];
    o->slot = first_slot(P, cu[o->s], o->s);
  } else {
    o->row0 = 0;
    o->len = P.rows;
    o->slot = o->s * P.units_per_seq;
  }
  o->idx = P.single ? 0 : u - o->slot;
  o->slot += o->idx;
  o->begin = o->idx * P.unit;
  o->end = P.single ? o->len : min(o->len, o->begin + P.unit);
  o->last = o->end >= o->len;
  return true;
}

// Row of the first token of span s in head h (of `heads`) of a [.., D] tensor; the rows
// of head h + 1 are P.rows further.
template <typename Plan>
__device__ __forceinline__ int64_t first_row(const Plan& P, const Span& s, int heads, int h) {
  return P.ragged ? (int64_t)h * P.rows + s.row0 : ((int64_t)s.s * heads + h) * P.rows;
}

}  // namespace gbla
