// gbla_delta.h -- host-side plans and launchers of the gated delta rule and of the
// residual stream's norm.  Internal to libgbla.so; not part of the public boundary.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "gbla.h"
#include "gbla_plan.h"

namespace gbla {

constexpr int kDeltaTile = 64;      // tokens of a tile
constexpr int kDeltaMaxUnit = 512;  // tokens of a unit, at most
constexpr int kPackBytes = 6 * 64 * 48;  // a tile's 64 x 64 triangle as operands (Packed), at most
constexpr int kGateBytes = 1536;         // a tile's gates (struct Gates)

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
  size_t off_gates;  // [V, tiles] Gates
  size_t off_pack;   // [V, tiles] packed triangles
  size_t off_B;      // [V, units, d, d] fp32: what a unit adds; then the state before each unit
  size_t off_M;      // [V, units, d, d] fp32: what a unit does to the state before it
  size_t total_bytes;
};

gbla_status make_delta_plan(const gbla_delta_shape* s, bool ragged, bool backward, DeltaPlan* p);

gbla_status launch_delta_forward(const DeltaPlan& p, const void* q, const void* k, const void* v,
                                 const float* log_decay, const float* beta, const float* S0,
                                 const int32_t* cu, void* ws, void* out, float* final_state,
                                 hipStream_t st);
gbla_status launch_delta_step(const gbla_delta_shape& s, const void* q, const void* k,
                              const void* v, const float* log_decay, const float* beta,
                              const int32_t* indices, int32_t slots, float* state, void* out,
                              hipStream_t st);

}  // namespace gbla
