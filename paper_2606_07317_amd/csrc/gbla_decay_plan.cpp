// gbla_decay_plan.cpp -- plans of the decoder's operators: split sizes and
// workspace layouts, a function of the shape alone.
#include <math.h>
#include <stdint.h>

#include "gbla.h"
#include "gbla_decay.h"

namespace gbla {
namespace {

// A grid's first dimension has fewer than 2^32 threads; the workgroups here have up to 512
// (or two of 256 to a unit) and 256.
constexpr int64_t kMaxGroups512 = 4294967295LL / 512, kMaxGroups256 = 4294967295LL / 256;
constexpr int kMaxGridY = 65535;
constexpr int kMaxPasses = 16;  // of a workgroup of the rotation's backward

bool head_dim_ok(int32_t d) { return d == 32 || d == 64 || d == 128; }
bool dtype_ok(int32_t t) { return t == GBLA_F32 || t == GBLA_BF16; }

// Tokens of a unit (a power of two): short enough for two workgroups a CU, long enough
// that the d x d record of a unit stays small beside its tokens.  Whole calls in us,
// units of 256 / 512 / 1024: forward bf16 B = 1, n = 32768, H = 8, d = 64 57 / 49 / 49;
// packed, 64 sequences, T = 177,929, d = 128, H = 8, K = 2 405 / 406 / 405; backward B = 8, n =
// 2048, H = 16, d = 64 165 / 141 / 140; 16 sequences, T = 57,511, H = 8, d = 128 880 / 762 / 761.
int32_t unit_tokens(const DecayPlan& p) {
  int32_t unit = kMaxUnit;
  while (unit > 2 * kTile && p.tokens * p.kv_heads < (int64_t)unit * 512) unit /= 2;
  return unit;
}

// Whether a workgroup walks a whole sequence.  One launch instead of three (three of
// five): its time is a + b longest while there are few (sequence, key head) pairs, that of
// the split a' + b' pairs longest, so the single walk wins where
//   longest (full - tokens of all pairs / longest) <= few,
// `full` pairs filling the chip at any length and few / full tokens passing for short
// whatever the pairs.  Single / split in us:
//   forward bf16 d = 64: B K = 8 n = 257 12 / 13, 384 14 / 13, 1024 32 / 14; 32 n = 384 14 / 14;
//   128 n = 768 26 / 29, 1024 34 / 33; 256 n = 4096 152 / 187.  d = 32: 8 n = 512 11 / 11, 768
//   15 / 11; 128 n = 1024 20 / 20.  d = 128: 8 n = 257 17 / 19, 384 20 / 19; 32 n = 512 27 / 25;
//   128 n = 2048 102 / 132.
//   forward fp32 d = 32: 2 n = 257 13 / 13, 320 14 / 13; 8 n = 257 14 / 13; 128 n = 512 22 / 21.
//   d = 64: 8 n = 192 17 / 20, 257 26 / 20; 128 n = 384 35 / 37, 512 45 / 41.  d = 128: 8 n = 192
//   26 / 33, 257 43 / 35; 128 n = 2048 293 / 375.
//   backward bf16 d = 32: 8 n = 192 19 / 21, 257 25 / 22; 64 n = 192 19 / 22, 257 26 / 23; 128 n =
//   384 30 / 31, 512 37 / 34; 192 n = 768 50 / 52, 1024 64 / 58; 256 n = 4096 234 / 242.  d = 64: 8
//   n = 128 23 / 27, 192 31 / 29; 64 n = 192 32 / 33, 257 45 / 38; 128 n = 320 49 / 50, 384 56 / 51;
//   192 n = 768 99 / 108, 1024 126 / 122; 256 n = 4096 499 / 560.  d = 128: 8 n = 128 37 / 41, 160
//   52 / 47; 64 n = 192 56 / 61, 257 81 / 73; 128 n = 768 191 / 199, 1024 238 / 226; 192 n = 2048
//   521 / 581.
//   backward fp32 d = 32: 8 n = 192 29 / 28; 128 n = 257 44 / 44.  d = 64: 8 n = 192 52 / 46; 128
//   n = 257 85 / 84; 256 n = 2048 495 / 553.  d = 128: 8 n = 192 131 / 105; 128 n = 384 279 / 297.
bool walk_whole(const DecayPlan& p, int64_t longest, bool backward) {
  struct Rule {
    int32_t full, few;
  };
  static constexpr Rule rules[2][2][3] = {  // forward, backward; bf16, fp32; d = 32, 64, 128
      {{{272, 148000}, {192, 61000}, {72, 20000}}, {{262, 68000}, {233, 47000}, {128, 27000}}},
      {{{240, 45000}, {245, 43000}, {150, 21500}}, {{256, 47000}, {256, 40000}, {190, 27000}}}};
  const Rule r = rules[backward][p.dtype == GBLA_F32][p.d == 32 ? 0 : p.d == 64 ? 1 : 2];
  return longest * r.full - p.tokens * p.kv_heads <= r.few;
}

}  // namespace

gbla_status make_decay_plan(const gbla_decay_shape* s, bool ragged, bool backward, DecayPlan* p) {
  if (!s || !p) return GBLA_ERR_INVALID_ARGUMENT;
  if (s->batch < 1 || s->seqlen < 0 || s->heads < 1 || s->kv_heads < 1)
    return GBLA_ERR_INVALID_ARGUMENT;
  if (s->heads % s->kv_heads != 0) return GBLA_ERR_INVALID_ARGUMENT;
  if (!isfinite(s->scale)) return GBLA_ERR_INVALID_ARGUMENT;
  if (ragged && s->max_seqlen < 0) return GBLA_ERR_INVALID_ARGUMENT;
  if (!head_dim_ok(s->head_dim) || !dtype_ok(s->dtype)) return GBLA_ERR_UNSUPPORTED;
  if (s->heads > kMaxGridY) return GBLA_ERR_UNSUPPORTED;
  DecayPlan q{};
  q.nseq = s->batch;
  q.rows = s->seqlen;
  q.heads = s->heads;
  q.kv_heads = s->kv_heads;
  q.group = s->heads / s->kv_heads;
  q.d = s->head_dim;
  q.dtype = s->dtype;
  q.ragged = ragged ? 1 : 0;
  q.scale = s->scale;
  q.tokens = ragged ? (int64_t)s->seqlen : (int64_t)s->batch * s->seqlen;
  if (q.tokens > kMaxGroups512 * kMaxUnit) return GBLA_ERR_UNSUPPORTED;  // before products with them
  q.unit = unit_tokens(q);
  // sum over the sequences of max(1, ceil(len / unit)) <= tokens / unit + N
  const int64_t cap = q.tokens / q.unit + q.nseq;
  if (cap > kMaxGroups512 - 8) return GBLA_ERR_UNSUPPORTED;
  if (ragged) {
    q.units = (int32_t)cap;
  } else {
    int64_t each = ((int64_t)q.rows + q.unit - 1) / q.unit;
    if (each < 1) each = 1;
    q.units_per_seq = (int32_t)each;
    q.units = (int32_t)(each * q.nseq);
  }
  q.single = walk_whole(q, ragged && s->max_seqlen < q.rows ? s->max_seqlen : q.rows, backward) ? 1 : 0;
  // the split's scan has a workgroup for every 256 elements of a sequence's states
  if ((int64_t)q.nseq * (q.d * q.d / 128) > kMaxGroups256) q.single = 1;
  q.grid_units = q.single ? q.nseq : q.units;
  const size_t states = (size_t)cap * q.kv_heads * q.d * q.d * sizeof(float);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = align_up(off + bytes, 256);
    return at;
  };
  q.off_S = take(states);
  if (backward) {
    q.off_D = take(states);
    q.off_dg = take(2 * (size_t)cap * q.kv_heads * 8 * sizeof(double));
  }
  q.total_bytes = off;
  *p = q;
  return GBLA_OK;
}

gbla_status make_rope_plan(const gbla_rope_shape* s, bool ragged, bool backward, RopePlan* p) {
  if (!s || !p) return GBLA_ERR_INVALID_ARGUMENT;
  if (s->batch < 1 || s->seqlen < 0 || s->heads < 1 || s->kv_heads < 1)
    return GBLA_ERR_INVALID_ARGUMENT;
  if (!(s->eps >= 0.0f) || !isfinite(s->eps)) return GBLA_ERR_INVALID_ARGUMENT;
  if (!(s->theta > 0.0f) || !isfinite(s->theta)) return GBLA_ERR_INVALID_ARGUMENT;
  if (s->flags & ~(uint32_t)(GBLA_NO_NORM | GBLA_ROPE_PAIRS)) return GBLA_ERR_INVALID_ARGUMENT;
  if (!head_dim_ok(s->head_dim) || !dtype_ok(s->dtype)) return GBLA_ERR_UNSUPPORTED;
  if (s->rotary_dim < 0 || s->rotary_dim > s->head_dim || s->rotary_dim % 8 != 0)
    return GBLA_ERR_UNSUPPORTED;
  if (s->heads > kMaxGridY || s->kv_heads > kMaxGridY) return GBLA_ERR_UNSUPPORTED;
  RopePlan q{};
  q.nseq = s->batch;
  q.rows = s->seqlen;
  q.heads = s->heads;
  q.kv_heads = s->kv_heads;
  q.d = s->head_dim;
  q.rotary = s->rotary_dim;
  q.dtype = s->dtype;
  q.ragged = ragged ? 1 : 0;
  q.eps = s->eps;
  q.flags = s->flags;
  q.tokens = ragged ? (int64_t)s->seqlen : (int64_t)s->batch * s->seqlen;
  q.tile = 256 / (q.d / 8);
  const int64_t tiles = (q.tokens + q.tile - 1) / q.tile;
  if (tiles > kMaxGroups256 * kMaxPasses) return GBLA_ERR_UNSUPPORTED;  // before products with them
  // Workgroups of one pass and up to eight heads; fewer heads while that gives
  // few workgroups.
  const int32_t all = q.heads + q.kv_heads;
  q.heads_each = 8;
  while (q.heads_each > 1 && tiles * ((all + q.heads_each - 1) / q.heads_each) < 1024)
    q.heads_each /= 2;
  q.head_blocks = (all + q.heads_each - 1) / q.heads_each;
  if (q.head_blocks > kMaxGridY) return GBLA_ERR_UNSUPPORTED;
  // The backward's workgroups leave a partial sum each: more passes where there
  // are many, so that few are added up.
  int64_t passes = 1;
  if (backward)
    while (tiles / passes * q.head_blocks > 2048 && passes < kMaxPasses) passes *= 2;
  q.passes = (int32_t)passes;
  const int64_t blocks = (tiles + passes - 1) / passes;
  if (blocks > kMaxGroups256) return GBLA_ERR_UNSUPPORTED;
  q.blocks = (int32_t)blocks;
  for (int i = 0; i < q.rotary / 2; ++i)
    q.turns[i] = pow((double)s->theta, -2.0 * i / q.rotary) / (2.0 * 3.14159265358979323846);
  *p = q;
  return GBLA_OK;
}

size_t rope_partial_bytes(const RopePlan& p) {
  return align_up((size_t)p.blocks * (p.heads + p.kv_heads) * p.d * sizeof(float), 256);
}

}  // namespace gbla
