// gbla_delta_plan.cpp -- plans of the gated delta rule: split sizes and workspace
// layouts, a function of the shape alone.
#include <math.h>
#include <stdint.h>

#include "gbla.h"
#include "gbla_delta.h"

namespace gbla {
namespace {

// A grid's first dimension has fewer than 2^32 threads; the workgroups here have up to 512.
constexpr int64_t kMaxGroups = 4294967295LL / 512;
constexpr int kMaxGridY = 65535;

// Tokens of a unit (a power of two): the largest that leaves 256 walks, a workgroup for each
// compute unit; 1024 only where that leaves four times as many.  Measured (bf16, us): 8192
// tokens, 8 heads of 64 with units of 128, 256, 512: 81, 69, 80; 16384 tokens, 8 heads of 128
// with 256, 512, 1024: 279, 233, 268; 178000 packed tokens, 8 heads of 128 with 512, 1024:
// 1916, 1786; backward, 58000 packed tokens, 8 heads of 128 with 256, 512, 1024: 2327, 2031, 2188.
int32_t unit_tokens(const DeltaPlan& p) {
  const int64_t all = p.tokens * p.value_heads;
  int32_t unit = all >= 1024 * kDeltaMaxUnit ? kDeltaMaxUnit : kDeltaMaxUnit / 2;
  while (unit > kDeltaTile && all < (int64_t)unit * 256) unit /= 2;
  return unit;
}

// Whether a workgroup walks a whole sequence: all are of a few tiles, or there are walks enough
// of the longest's length.  Measured (split, whole, in us; 8 heads of 64 in bf16 where nothing
// else is said): 1 x 192 tokens 28, 23; 1 x 256 28, 27; 1 x 320 27, 30; 1 x 128 in fp32 28, 23
// (heads of 32); 1 x 192 in fp32 31, 34; 8 x 512 41, 45; 16 x 1024 92, 88; 16 x 4096 296, 315;
// 32 x 4096 583, 386; backward, where a split sequence takes two launches more: 1 x 192 64, 57;
// 1 x 256 62, 70; 16 x 512 164, 148; 16 x 1024 288, 278; 8 x 2048, 16 heads 460, 545; 16 x 2048,
// 16 heads 874, 695.
bool walk_whole(const DeltaPlan& p, int64_t longest, bool backward) {
  const int few = p.dtype == GBLA_F32 ? 2 : backward ? 3 : 4;
  return longest <= few * kDeltaTile || longest * (longest <= 1024 ? 128 : 256) <= p.tokens * p.value_heads;
}

}  // namespace

gbla_status make_delta_plan(const gbla_delta_shape* s, bool ragged, bool backward, DeltaPlan* p) {
  if (!s || !p) return GBLA_ERR_INVALID_ARGUMENT;
  if (s->batch < 1 || s->seqlen < 0 || s->heads < 1 || s->value_heads < 1)
    return GBLA_ERR_INVALID_ARGUMENT;
  if (s->value_heads % s->heads != 0) return GBLA_ERR_INVALID_ARGUMENT;
  if (!isfinite(s->scale)) return GBLA_ERR_INVALID_ARGUMENT;
  if (ragged && s->max_seqlen < 0) return GBLA_ERR_INVALID_ARGUMENT;
  if (s->head_dim != 32 && s->head_dim != 64 && s->head_dim != 128) return GBLA_ERR_UNSUPPORTED;
  if (s->dtype != GBLA_F32 && s->dtype != GBLA_BF16) return GBLA_ERR_UNSUPPORTED;
  if (s->value_heads > kMaxGridY) return GBLA_ERR_UNSUPPORTED;
  DeltaPlan q{};
  q.nseq = s->batch;
  q.rows = s->seqlen;
  q.heads = s->heads;
  q.value_heads = s->value_heads;
  q.group = s->value_heads / s->heads;
  q.d = s->head_dim;
  q.dtype = s->dtype;
  q.ragged = ragged ? 1 : 0;
  q.scale = s->scale;
  q.tokens = ragged ? (int64_t)s->seqlen : (int64_t)s->batch * s->seqlen;
  if (q.tokens > kMaxGroups * kDeltaTile) return GBLA_ERR_UNSUPPORTED;  // before products with them
  // sum over the sequences of max(1, ceil(len / tile)) <= tokens / tile + N
  const int64_t most = q.tokens / kDeltaTile + q.nseq;
  if (most > kMaxGroups) return GBLA_ERR_UNSUPPORTED;
  q.unit = unit_tokens(q);
  const int64_t cap = q.tokens / q.unit + q.nseq;
  if (ragged) {
    q.tiles = (int32_t)most;
    q.units = (int32_t)cap;
  } else {
    const auto pieces = [&](int64_t size) {
      const int64_t each = ((int64_t)q.rows + size - 1) / size;
      return (int32_t)(each < 1 ? 1 : each);
    };
    q.tiles_per_seq = pieces(kDeltaTile);
    q.tiles = q.tiles_per_seq * q.nseq;
    q.units_per_seq = pieces(q.unit);
    q.units = q.units_per_seq * q.nseq;
  }
  q.single = walk_whole(q, ragged && s->max_seqlen < q.rows ? s->max_seqlen : q.rows, backward) ? 1 : 0;
  // the split's scan has a workgroup for every 16 value channels of a state, in groups of eight
  if (((int64_t)q.nseq * q.value_heads + 7) * (q.d / 16) > kMaxGroups) q.single = 1;
  q.grid_units = q.single ? q.nseq : q.units;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = align_up(off + bytes, 256);
    return at;
  };
  q.off_pack = take((size_t)most * q.value_heads * kPackBytes);
  const size_t states = (size_t)cap * q.value_heads * q.d * q.d * sizeof(float);
  q.off_B = take(states);
  q.off_M = take(states);
  if (backward) {
    const size_t each = (size_t)most * q.value_heads, state = (size_t)q.d * q.d * sizeof(float);
    const size_t vectors = (size_t)q.d * kDeltaTile * sizeof(float);
    const size_t gate = (size_t)q.tokens * q.value_heads * sizeof(float);
    q.off_MT = take(states);
    q.off_packT = take(each * kPackBytes);
    q.off_D = take(states);
    q.off_S = take(each * state);
    q.off_N = take(each * state);
    q.off_E = take(each * vectors);
    q.off_F = take(each * vectors);
    q.off_from = take(gate);
    q.off_on = take(gate);
    q.off_sums = take(each * sizeof(DeltaTileSums));
    q.off_dS0 = take((size_t)q.nseq * q.value_heads * state);
  }
  q.total_bytes = off;
  *p = q;
  return GBLA_OK;
}

}  // namespace gbla
