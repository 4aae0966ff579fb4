// gbla_norm_api.cpp -- plan and C entry points of the residual stream's norm
// (include/gbla.h).  Every check runs on the host before anything is enqueued.
#include <math.h>
#include <stdint.h>

#include "gbla.h"
#include "gbla_checks.h"
#include "gbla_norm.h"

namespace gbla {
namespace {

constexpr int32_t kMaxWidth = 16384;
constexpr int64_t kMaxBlocks = 1 << 20;

}  // namespace

gbla_status make_norm_plan(const gbla_norm_shape* s, bool backward, NormPlan* p) {
  if (!s || !p) return GBLA_ERR_INVALID_ARGUMENT;
  if (s->rows < 0 || s->width < 1 || s->group < 0) return GBLA_ERR_INVALID_ARGUMENT;
  if (!(s->eps >= 0.0f) || !isfinite(s->eps)) return GBLA_ERR_INVALID_ARGUMENT;
  if (s->dtype != GBLA_F32 && s->dtype != GBLA_BF16) return GBLA_ERR_UNSUPPORTED;
  if (s->width % 8 != 0 || s->width > kMaxWidth) return GBLA_ERR_UNSUPPORTED;
  // 2^60 bytes of rows are more than any machine has, and the products below stay in range
  if (s->rows > ((int64_t)1 << 60) / s->width) return GBLA_ERR_UNSUPPORTED;
  if (!backward) {
    if (s->out_dtype != s->dtype && s->out_dtype != GBLA_E4M3) return GBLA_ERR_UNSUPPORTED;
    if (s->group != 0 && (s->out_dtype != GBLA_E4M3 || s->group != 128 || s->width % 128 != 0))
      return GBLA_ERR_UNSUPPORTED;
  }
  NormPlan q{};
  q.rows = s->rows;
  q.width = s->width;
  q.dtype = s->dtype;
  q.out_dtype = s->out_dtype;
  q.group = s->group;
  q.eps = s->eps;
  q.inv_width = (float)(1.0 / s->width);
  const int32_t eights = s->width / 8;
  q.lanes = 8;
  while (q.lanes < 64 && q.lanes < eights) q.lanes *= 2;
  if (eights > 4 * 64) q.lanes = 256;
  q.pieces = 1;
  while (q.lanes * q.pieces < eights) q.pieces *= 2;
  const int32_t each = 256 / q.lanes;
  const int64_t groups = (q.rows + each - 1) / each;
  // The backward's workgroups leave a partial sum each.  One workgroup for up to four groups of
  // rows writes its sum as the gradient and saves the launch that adds them (a call from Python
  // with 4 rows of 1024: 13.9 us with it, 10.9 without).
  const int64_t most = backward ? (q.lanes == 256 ? 512 : 1024) : kMaxBlocks;
  q.blocks = (int32_t)(backward && groups <= 4 ? groups > 0 : groups < most ? groups : most);
  *p = q;
  return GBLA_OK;
}

size_t norm_partial_bytes(const NormPlan& p) {
  const size_t bytes = align_up((size_t)p.blocks * p.width * sizeof(float), 256);
  return bytes < 256 ? 256 : bytes;
}

}  // namespace gbla

using namespace gbla::checks;

extern "C" {

gbla_status gbla_add_norm(const gbla_norm_shape* shape, const void* x, const void* residual,
                          const float* weight, void* sum, void* out, float* scales, void* stream) {
  gbla::NormPlan p;
  GBLA_TRY(gbla::make_norm_plan(shape, false, &p));
  GBLA_TRY(rows_present(p.rows, {x, out}));
  GBLA_TRY(present({weight}));
  GBLA_TRY(optional({residual, sum}));
  if (p.out_dtype == GBLA_E4M3) GBLA_TRY(rows_present(p.rows, {scales}, 4));
  return gbla::launch_norm(p, x, residual, weight, sum, out, scales, static_cast<hipStream_t>(stream));
}

size_t gbla_add_norm_backward_workspace_bytes(const gbla_norm_shape* shape) {
  gbla::NormPlan p;
  return gbla::make_norm_plan(shape, true, &p) == GBLA_OK ? gbla::norm_partial_bytes(p) : 0;
}

gbla_status gbla_add_norm_backward(const gbla_norm_shape* shape, const void* sum,
                                   const float* weight, const void* dout, const void* dsum,
                                   void* workspace, size_t workspace_bytes, void* dx,
                                   float* dweight, void* stream) {
  gbla::NormPlan p;
  GBLA_TRY(gbla::make_norm_plan(shape, true, &p));
  GBLA_TRY(rows_present(p.rows, {sum, dout, dx}));
  GBLA_TRY(present({weight, dweight}));
  GBLA_TRY(optional({dsum}));
  GBLA_TRY(scratch(workspace, workspace_bytes, gbla::norm_partial_bytes(p)));
  return gbla::launch_norm_backward(p, sum, weight, dout, dsum, workspace, dx, dweight,
                                    static_cast<hipStream_t>(stream));
}

}  // extern "C"
