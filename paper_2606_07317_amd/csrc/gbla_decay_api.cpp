// gbla_decay_api.cpp -- the C entry points of the decoder's operators
// (include/gbla.h).  Every check runs on the host before anything is enqueued.
#include <stdint.h>

#include <initializer_list>

#include "gbla.h"
#include "gbla_decay.h"

namespace {

// Arrays in use: present, and aligned to `a` bytes.
gbla_status present(std::initializer_list<const void*> ptrs, size_t a = 16) {
  for (const void* p : ptrs) {
    if (!p) return GBLA_ERR_INVALID_ARGUMENT;
    if (!gbla::aligned(p, a)) return GBLA_ERR_MISALIGNED;
  }
  return GBLA_OK;
}

// Arrays over the tokens: of no elements, and so possibly NULL, where there are none.
gbla_status rows_present(int64_t tokens, std::initializer_list<const void*> ptrs) {
  return tokens > 0 ? present(ptrs) : GBLA_OK;
}

// Arrays that may be NULL.
gbla_status optional(std::initializer_list<const void*> ptrs, size_t a = 16) {
  for (const void* p : ptrs)
    if (p && !gbla::aligned(p, a)) return GBLA_ERR_MISALIGNED;
  return GBLA_OK;
}

gbla_status scratch(const void* ws, size_t have, size_t need) {
  if (!ws) return GBLA_ERR_WORKSPACE;
  if (!gbla::aligned(ws, 256)) return GBLA_ERR_MISALIGNED;
  return have < need ? GBLA_ERR_WORKSPACE : GBLA_OK;
}

size_t decay_bytes(const gbla_decay_shape* shape, bool ragged, bool backward) {
  gbla::DecayPlan p;
  return gbla::make_decay_plan(shape, ragged, backward, &p) == GBLA_OK ? p.total_bytes : 0;
}

size_t rope_bytes(const gbla_rope_shape* shape, bool ragged) {
  gbla::RopePlan p;
  if (gbla::make_rope_plan(shape, ragged, true, &p) != GBLA_OK) return 0;
  const size_t bytes = gbla::rope_partial_bytes(p);
  return bytes < 256 ? 256 : bytes;
}

size_t larger(size_t a, size_t b) { return a > b ? a : b; }

#define GBLA_TRY(expr)                  \
  do {                                  \
    gbla_status _st = (expr);           \
    if (_st != GBLA_OK) return _st;     \
  } while (0)

}  // namespace

extern "C" {

gbla_status gbla_qk_norm_rope(const gbla_rope_shape* shape, const void* q, const void* k,
                              const float* q_w, const float* k_w, const int32_t* positions,
                              const int32_t* cu_seqlens, void* q_out, void* k_out, void* stream) {
  gbla::RopePlan p;
  GBLA_TRY(gbla::make_rope_plan(shape, cu_seqlens != nullptr, false, &p));
  GBLA_TRY(rows_present(p.tokens, {q, k, q_out, k_out}));
  if (!(p.flags & GBLA_NO_NORM)) GBLA_TRY(present({q_w, k_w}));
  GBLA_TRY(optional({positions, cu_seqlens}, 4));
  return gbla::launch_rope(p, q, k, q_w, k_w, positions, cu_seqlens, q_out, k_out,
                           static_cast<hipStream_t>(stream));
}

size_t gbla_qk_norm_rope_backward_workspace_bytes(const gbla_rope_shape* shape) {
  return larger(rope_bytes(shape, false), rope_bytes(shape, true));
}

size_t gbla_qk_norm_rope_backward_ragged_workspace_bytes(const gbla_rope_shape* shape) {
  return rope_bytes(shape, true);
}

gbla_status gbla_qk_norm_rope_backward(const gbla_rope_shape* shape, const void* q, const void* k,
                                       const float* q_w, const float* k_w,
                                       const int32_t* positions, const int32_t* cu_seqlens,
                                       const void* dq_out, const void* dk_out, void* workspace,
                                       size_t workspace_bytes, void* dq, void* dk, float* dq_w,
                                       float* dk_w, void* stream) {
  gbla::RopePlan p;
  GBLA_TRY(gbla::make_rope_plan(shape, cu_seqlens != nullptr, true, &p));
  GBLA_TRY(rows_present(p.tokens, {q, k, dq_out, dk_out, dq, dk}));
  if (!(p.flags & GBLA_NO_NORM)) GBLA_TRY(present({q_w, k_w, dq_w, dk_w}));
  GBLA_TRY(optional({positions, cu_seqlens}, 4));
  GBLA_TRY(scratch(workspace, workspace_bytes, gbla::rope_partial_bytes(p)));
  return gbla::launch_rope_backward(p, q, k, q_w, k_w, positions, cu_seqlens, dq_out, dk_out,
                                    workspace, dq, dk, dq_w, dk_w,
                                    static_cast<hipStream_t>(stream));
}

size_t gbla_decay_workspace_bytes(const gbla_decay_shape* shape) {
  return larger(decay_bytes(shape, false, false), decay_bytes(shape, true, false));
}

size_t gbla_decay_backward_workspace_bytes(const gbla_decay_shape* shape) {
  return larger(decay_bytes(shape, false, true), decay_bytes(shape, true, true));
}

size_t gbla_decay_ragged_workspace_bytes(const gbla_decay_shape* shape) {
  return decay_bytes(shape, true, false);
}

size_t gbla_decay_backward_ragged_workspace_bytes(const gbla_decay_shape* shape) {
  return decay_bytes(shape, true, true);
}

gbla_status gbla_decay_forward(const gbla_decay_shape* shape, const void* q, const void* k,
                               const void* v, const float* log_decay,
                               const float* initial_state, const int32_t* cu_seqlens,
                               void* workspace, size_t workspace_bytes, void* out,
                               float* final_state, void* stream) {
  gbla::DecayPlan p;
  GBLA_TRY(gbla::make_decay_plan(shape, cu_seqlens != nullptr, false, &p));
  GBLA_TRY(rows_present(p.tokens, {q, k, v, out}));
  GBLA_TRY(present({log_decay}, 4));
  GBLA_TRY(optional({initial_state, final_state}));
  GBLA_TRY(optional({cu_seqlens}, 4));
  GBLA_TRY(scratch(workspace, workspace_bytes, p.total_bytes));
  return gbla::launch_decay_forward(p, q, k, v, log_decay, initial_state, cu_seqlens, workspace,
                                    out, final_state, static_cast<hipStream_t>(stream));
}

gbla_status gbla_decay_backward(const gbla_decay_shape* shape, const void* q, const void* k,
                                const void* v, const float* log_decay,
                                const float* initial_state, const int32_t* cu_seqlens,
                                const void* dout, const float* dfinal_state, void* workspace,
                                size_t workspace_bytes, void* dq, void* dk, void* dv,
                                float* dlog_decay, float* dinitial_state, void* stream) {
  gbla::DecayPlan p;
  GBLA_TRY(gbla::make_decay_plan(shape, cu_seqlens != nullptr, true, &p));
  GBLA_TRY(rows_present(p.tokens, {q, k, v, dout, dq, dk, dv}));
  GBLA_TRY(present({log_decay}, 4));
  GBLA_TRY(optional({initial_state, dfinal_state, dinitial_state}));
  GBLA_TRY(optional({cu_seqlens, dlog_decay}, 4));
  GBLA_TRY(scratch(workspace, workspace_bytes, p.total_bytes));
  return gbla::launch_decay_backward(p, q, k, v, log_decay, initial_state, cu_seqlens, dout,
                                     dfinal_state, workspace, dq, dk, dv, dlog_decay,
                                     dinitial_state, static_cast<hipStream_t>(stream));
}

gbla_status gbla_decay_step(const gbla_decay_shape* shape, const void* q, const void* k,
                            const void* v, const float* log_decay, const int32_t* state_indices,
                            int32_t slots, float* state, void* out, void* stream) {
  gbla::DecayPlan p;  // the shape's checks
  GBLA_TRY(gbla::make_decay_plan(shape, false, false, &p));
  if (shape->seqlen != 1 || slots < 1) return GBLA_ERR_INVALID_ARGUMENT;
  if (!state_indices && slots < shape->batch) return GBLA_ERR_INVALID_ARGUMENT;
  GBLA_TRY(present({q, k, v, state, out}));
  GBLA_TRY(present({log_decay}, 4));
  GBLA_TRY(optional({state_indices}, 4));
  return gbla::launch_decay_step(*shape, q, k, v, log_decay, state_indices, slots, state, out,
                                 static_cast<hipStream_t>(stream));
}

}  // extern "C"
