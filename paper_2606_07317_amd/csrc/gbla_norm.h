// gbla_norm.h -- host-side plan and launchers of the residual stream's norm.  Internal to
// libgbla.so; not part of the public boundary.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "gbla.h"
#include "gbla_plan.h"

namespace gbla {

struct NormPlan {
  int64_t rows;
  int32_t width, dtype, out_dtype, group;
  float eps, inv_width;
  int32_t lanes;   // of a row: 8, 16, 32, 64, or a workgroup's 256
  int32_t pieces;  // of eight channels a lane: 1, 2, 4 or 8
  int32_t blocks;  // workgroups; each takes every blocks-th group of 256 / lanes rows
};

gbla_status make_norm_plan(const gbla_norm_shape* s, bool backward, NormPlan* p);
size_t norm_partial_bytes(const NormPlan& p);
gbla_status launch_norm(const NormPlan& p, const void* x, const void* residual, const float* w,
                        void* sum, void* out, float* scales, hipStream_t st);
gbla_status launch_norm_backward(const NormPlan& p, const void* sum, const float* w,
                                 const void* dout, const void* dsum, void* ws, void* dx, float* dw,
                                 hipStream_t st);

}  // namespace gbla
