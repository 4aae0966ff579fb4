// gbla_decay.h -- host-side plans and launchers of the decoder's operators: the
// norm and rotation of queries and keys, and causal linear attention with a
// decay.  Internal to libgbla.so; not part of the public boundary.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "gbla.h"
#include "gbla_plan.h"

namespace gbla {

constexpr int kTile = 64;       // tokens of a tile of the decay kernels
constexpr int kMaxUnit = 512;   // tokens of a unit, at most

// The launches of gbla_decay_forward / gbla_decay_backward; a function of the
// shape alone (and of max_seqlen, which only sets `single`).
struct DecayPlan {
  int32_t nseq, rows, heads, kv_heads, group;  // group = heads / kv_heads
  int32_t d, dtype, ragged;
  float scale;
  int64_t tokens;
  // The tokens of a (sequence, key head) are cut into units.  Split: a
  // workgroup a unit, with the states between units joined by a launch of their
  // own.  Single: a workgroup walks the whole sequence.
  int32_t single;
  int32_t unit;           // tokens of a unit, a multiple of kTile
  int32_t units_per_seq;  // dense: ceil(n / unit), at least 1
  int32_t units;          // units of a key head (dense exact, ragged bound)
  int32_t grid_units;     // workgroups of a key head: nseq (single) or units
  // Workspace (bytes from its base)
  size_t off_S;   // [K, units, d, d] fp32: the state before each unit
  size_t off_D;   // backward: [K, units, d, d] the gradient of the state after each unit
  size_t off_dg;  // backward: [2, K, grid_units, 4 or 8] double, parts of dlog_decay
  size_t total_bytes;
};

gbla_status make_decay_plan(const gbla_decay_shape* s, bool ragged, bool backward, DecayPlan* p);

gbla_status launch_decay_forward(const DecayPlan& p, const void* q, const void* k, const void* v,
                                 const float* log_decay, const float* S0, const int32_t* cu,
                                 void* ws, void* out, float* final_state, hipStream_t st);
gbla_status launch_decay_backward(const DecayPlan& p, const void* q, const void* k, const void* v,
                                  const float* log_decay, const float* S0, const int32_t* cu,
                                  const void* dout, const float* dfinal, void* ws, void* dq,
                                  void* dk, void* dv, float* dlog_decay, float* dS0,
                                  hipStream_t st);
// The gradients of k, v, the decay and the initial state (gbla_decay_back.hip):
// the last launches of the backward.
gbla_status launch_decay_keys(const DecayPlan& p, const void* q, const void* k, const void* v,
                              const float* log_decay, const float* S0, const int32_t* cu,
                              const void* dout, const float* dfinal, void* ws, void* dk, void* dv,
                              float* dlog_decay, float* dS0, hipStream_t st);
gbla_status launch_decay_step(const gbla_decay_shape& s, const void* q, const void* k,
                              const void* v, const float* log_decay, const int32_t* indices,
                              int32_t slots, float* state, void* out, hipStream_t st);

// The norm and rotation of queries and keys.
struct RopePlan {
  int32_t nseq, rows, heads, kv_heads, d, rotary, dtype, ragged;
  float eps;
  uint32_t flags;
  int64_t tokens;
  int32_t tile;          // tokens of a pass of a workgroup
  int32_t passes;        // passes of a workgroup
  int32_t blocks;        // workgroups over the tokens
  int32_t heads_each;    // heads (of H + K) of a workgroup
  int32_t head_blocks;
  double turns[64];      // turns of the pair i per position: theta^(-2 i / R) / (2 pi)
};
// Kernels' arguments are small: the plan goes by value, 600 bytes.
gbla_status make_rope_plan(const gbla_rope_shape* s, bool ragged, bool backward, RopePlan* p);
size_t rope_partial_bytes(const RopePlan& p);
gbla_status launch_rope(const RopePlan& p, const void* q, const void* k, const float* q_w,
                        const float* k_w, const int32_t* pos, const int32_t* cu, void* q_out,
                        void* k_out, hipStream_t st);
gbla_status launch_rope_backward(const RopePlan& p, const void* q, const void* k, const float* q_w,
                                 const float* k_w, const int32_t* pos, const int32_t* cu,
                                 const void* dq_out, const void* dk_out, void* ws, void* dq,
                                 void* dk, float* dq_w, float* dk_w, hipStream_t st);

}  // namespace gbla
