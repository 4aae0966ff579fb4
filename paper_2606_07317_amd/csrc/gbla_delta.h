// gbla_delta.h -- host-side plans and launchers of the gated delta rule.  Internal to
// libgbla.so; not part of the public boundary.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "gbla.h"
#include "gbla_plan.h"

namespace gbla {

constexpr int kDeltaTile = 64;      // tokens of a tile
constexpr int kDeltaMaxUnit = 1024;  // tokens of a unit, at most
constexpr int kGateBytes = 1792;         // a tile's gates (struct Gates)
constexpr int kPackBytes = 6 * 64 * 48 + kGateBytes;  // a tile's triangle as operands (Packed), at most, and gates

// The launches of gbla_delta_forward / gbla_delta_backward; a function of the shape
// alone (and of max_seqlen, which only sets `single`).
struct DeltaPlan {
  int32_t nseq, rows, heads, value_heads, group;  // group = value_heads / heads
  int32_t d, dtype, ragged;
  float scale;
  int64_t tokens;
  // The tokens of a (sequence, value head) are cut into units.  Split: a workgroup a
  // unit, with the states between units joined by a launch of their own.  Single: a
  // workgroup walks the whole sequence.
  int32_t single;
  int32_t unit;           // tokens of a unit, a multiple of kDeltaTile
  int32_t units_per_seq;  // dense: ceil(n / unit), at least 1
  int32_t units;          // units of a value head (dense exact, ragged bound)
  int32_t grid_units;     // workgroups of a value head: nseq (single) or units
  int32_t tiles_per_seq;  // dense: ceil(n / kDeltaTile), at least 1
  int32_t tiles;          // tile slots of a value head (dense exact, ragged bound)
  // Workspace (bytes from its base)
  size_t off_pack;   // [V, tiles] packed triangles and gates
  size_t off_B;      // [V, units, d, d] fp32: what a unit adds; then the state before each unit
  size_t off_M;      // [V, units, d, d] fp32: what a unit does to the state before it, transposed
  // Backward:
  size_t off_MT;     // [V, units, d, d] fp32: the maps, transposed against off_M
  size_t off_packT;  // ... with the triangles transposed
  size_t off_D;      // [V, units, d, d] fp32: the gradient of the state after each unit
  size_t off_S;      // [V, tiles, d, d] fp32: the state before each tile, [value][key channel]
  size_t off_N;      // ... the gradient of the state after each tile
  size_t off_E;      // [V, tiles, d, 64] fp32: the tiles' e, [value channel][token]; before that, what
                     // of the gradient of u comes from the state after the tile
  size_t off_F;      // ... the gradient of u
  size_t off_from;   // fp32, like the gates: what of the decays' gradient ends at each token and
                     // comes from the state before its tile
  size_t off_on;     // ... begins at each token and goes on to the state after its tile
  size_t off_sums;   // [V, tiles] DeltaTileSums
  size_t off_dS0;    // [N, V, d, d] fp32: dinitial_state where the caller wants none
  size_t total_bytes;
};

// What a tile has of its decays' gradient (gbla_delta_grads.hip).
struct DeltaTileSums {
  double from, on;  // sums of off_from's and off_on's tokens
  double over;      // what passes over the whole tile
  float steps;      // tiles from where the sum that `over` comes of is known
  int32_t direct;   // `over` was formed of the states themselves
};

gbla_status make_delta_plan(const gbla_delta_shape* s, bool ragged, bool backward, DeltaPlan* p);

gbla_status launch_delta_forward(const DeltaPlan& p, const void* q, const void* k, const void* v,
                                 const float* log_decay, const float* beta, const float* S0,
                                 const int32_t* cu, void* ws, void* out, float* final_state,
                                 hipStream_t st);
gbla_status launch_delta_backward(const DeltaPlan& p, const void* q, const void* k, const void* v,
                                  const float* log_decay, const float* beta, const float* S0,
                                  const int32_t* cu, const void* dout, const float* dfinal, void* ws,
                                  void* dq, void* dk, void* dv, float* dlog_decay, float* dbeta,
                                  float* dS0, hipStream_t st);
// Its pass from the last tile to the first (gbla_delta_back.hip): the units' records, and the
// walk; and its last launches (gbla_delta_grads.hip): the gradients of q, k, v and log_decay.
gbla_status launch_delta_back_records(const DeltaPlan& p, const void* q, const void* k, const int32_t* cu,
                                      const void* dout, void* ws, hipStream_t st);
gbla_status launch_delta_back_walk(const DeltaPlan& p, const void* q, const void* k, const int32_t* cu,
                                   const void* dout, const float* dfinal, void* ws, float* dS0,
                                   hipStream_t st);
gbla_status launch_delta_grads(const DeltaPlan& p, const void* q, const void* k, const float* S0,
                               const int32_t* cu, const void* dout, void* ws, void* dq, void* dk,
                               void* dv, float* dlog_decay, const float* dS0, bool final_gradient,
                               hipStream_t st);
gbla_status launch_delta_step(const gbla_delta_shape& s, const void* q, const void* k,
                              const void* v, const float* log_decay, const float* beta,
                              const int32_t* indices, int32_t slots, float* state, void* out,
                              hipStream_t st);

}  // namespace gbla
