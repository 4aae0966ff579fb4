// gbla_delta_api.cpp -- the C entry points of the gated delta rule (include/gbla.h).
// Every check runs on the host before anything is enqueued.
#include <stdint.h>

#include "gbla.h"
#include "gbla_checks.h"
#include "gbla_delta.h"

namespace {

size_t delta_bytes(const gbla_delta_shape* shape, bool ragged, bool backward) {
  gbla::DeltaPlan p;
  return gbla::make_delta_plan(shape, ragged, backward, &p) == GBLA_OK ? p.total_bytes : 0;
}

}  // namespace

using namespace gbla::checks;

extern "C" {

size_t gbla_delta_workspace_bytes(const gbla_delta_shape* shape) {
  return larger(delta_bytes(shape, false, false), delta_bytes(shape, true, false));
}

size_t gbla_delta_ragged_workspace_bytes(const gbla_delta_shape* shape) {
  return delta_bytes(shape, true, false);
}

gbla_status gbla_delta_forward(const gbla_delta_shape* shape, const void* q, const void* k,
                               const void* v, const float* log_decay, const float* beta,
                               const float* initial_state, const int32_t* cu_seqlens,
                               void* workspace, size_t workspace_bytes, void* out,
                               float* final_state, void* stream) {
  gbla::DeltaPlan p;
  GBLA_TRY(gbla::make_delta_plan(shape, cu_seqlens != nullptr, false, &p));
  GBLA_TRY(rows_present(p.tokens, {q, k, v, out}));
  GBLA_TRY(rows_present(p.tokens, {log_decay, beta}, 4));
  GBLA_TRY(optional({initial_state, final_state}));
  GBLA_TRY(optional({cu_seqlens}, 4));
  GBLA_TRY(scratch(workspace, workspace_bytes, p.total_bytes));
  return gbla::launch_delta_forward(p, q, k, v, log_decay, beta, initial_state, cu_seqlens,
                                    workspace, out, final_state, static_cast<hipStream_t>(stream));
}

size_t gbla_delta_backward_workspace_bytes(const gbla_delta_shape* shape) {
  return larger(delta_bytes(shape, false, true), delta_bytes(shape, true, true));
}

size_t gbla_delta_backward_ragged_workspace_bytes(const gbla_delta_shape* shape) {
  return delta_bytes(shape, true, true);
}

gbla_status gbla_delta_backward(const gbla_delta_shape* shape, const void* q, const void* k,
                                const void* v, const float* log_decay, const float* beta,
                                const float* initial_state, const int32_t* cu_seqlens,
                                const void* dout, const float* dfinal_state, void* workspace,
                                size_t workspace_bytes, void* dq, void* dk, void* dv,
                                float* dlog_decay, float* dbeta, float* dinitial_state,
                                void* stream) {
  gbla::DeltaPlan p;
  GBLA_TRY(gbla::make_delta_plan(shape, cu_seqlens != nullptr, true, &p));
  GBLA_TRY(rows_present(p.tokens, {q, k, v, dout, dq, dk, dv}));
  GBLA_TRY(rows_present(p.tokens, {log_decay, beta, dlog_decay, dbeta}, 4));
  GBLA_TRY(optional({initial_state, dfinal_state, dinitial_state}));
  GBLA_TRY(optional({cu_seqlens}, 4));
  GBLA_TRY(scratch(workspace, workspace_bytes, p.total_bytes));
  return gbla::launch_delta_backward(p, q, k, v, log_decay, beta, initial_state, cu_seqlens, dout,
                                     dfinal_state, workspace, dq, dk, dv, dlog_decay, dbeta,
                                     dinitial_state, static_cast<hipStream_t>(stream));
}

gbla_status gbla_delta_step(const gbla_delta_shape* shape, const void* q, const void* k,
                            const void* v, const float* log_decay, const float* beta,
                            const int32_t* state_indices, int32_t slots, float* state, void* out,
                            void* stream) {
  gbla::DeltaPlan p;  // the shape's checks
  GBLA_TRY(gbla::make_delta_plan(shape, false, false, &p));
  if (shape->seqlen != 1 || slots < 1) return GBLA_ERR_INVALID_ARGUMENT;
  if (!state_indices && slots < shape->batch) return GBLA_ERR_INVALID_ARGUMENT;
  GBLA_TRY(present({q, k, v, state, out}));
  GBLA_TRY(present({log_decay, beta}, 4));
  GBLA_TRY(optional({state_indices}, 4));
  return gbla::launch_delta_step(*shape, q, k, v, log_decay, beta, state_indices, slots, state, out,
                                 static_cast<hipStream_t>(stream));
}

}  // extern "C"
