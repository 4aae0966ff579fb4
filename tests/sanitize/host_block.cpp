// Host-only driver for the sanitizer test: the plans and the argument checks of the decoder
// block's operators (gbla_delta_plan.cpp, gbla_delta_api.cpp, gbla_norm_api.cpp), built with
// -fsanitize=address,undefined and the kernel launchers replaced by stubs that check the
// grids and the workspaces they would use.  Prints "host block ok" at the end.
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include "gbla.h"
#include "gbla_delta.h"
#include "gbla_norm.h"

#define REQUIRE(cond)                                                          \
  do {                                                                         \
    if (!(cond)) {                                                             \
      fprintf(stderr, "host_block: %s failed at line %d\n", #cond, __LINE__); \
      abort();                                                                 \
    }                                                                          \
  } while (0)

namespace gbla {
static int g_launches = 0;

static bool grid_ok(int64_t x, int64_t y, int threads) {
  return x >= 1 && x * threads <= (int64_t)UINT32_MAX && y >= 1 && y <= 65535;
}

static void check(const DeltaPlan& p, bool backward) {
  REQUIRE(grid_ok(p.tiles, p.value_heads, 256));
  REQUIRE(grid_ok(p.grid_units, p.value_heads, 4 * p.d));
  if (!p.single) REQUIRE(grid_ok(((int64_t)p.nseq * p.value_heads + 7) / 8 * 8 * (p.d / 16), 1, 4 * p.d));
  REQUIRE(p.group * p.heads == p.value_heads);
  REQUIRE(p.unit % kDeltaTile == 0 && p.unit >= kDeltaTile);
  REQUIRE(p.units >= 1 && p.tiles >= p.units && (p.single ? p.grid_units == p.nseq : p.grid_units == p.units));
  const size_t tiles = (size_t)p.tiles * p.value_heads, units = (size_t)p.units * p.value_heads;
  const size_t state = (size_t)p.d * p.d * sizeof(float);
  REQUIRE(p.off_pack + tiles * kPackBytes <= p.off_B);
  REQUIRE(p.off_B + units * state <= p.off_M);
  REQUIRE(p.off_M + units * state <= p.total_bytes);
  if (backward) REQUIRE(p.off_M + units * state <= p.off_packT && p.off_packT < p.off_D && p.off_D < p.total_bytes);
  ++g_launches;
}

gbla_status launch_delta_forward(const DeltaPlan& p, const void*, const void*, const void*, const float*, const float*,
                                 const float*, const int32_t*, void*, void*, float*, hipStream_t) {
  check(p, false);
  return GBLA_OK;
}
gbla_status launch_delta_backward(const DeltaPlan& p, const void*, const void*, const void*, const float*, const float*,
                                  const float*, const int32_t*, const void*, const float*, void*, void*, void*, void*,
                                  float*, float*, float*, hipStream_t) {
  check(p, true);
  return GBLA_OK;
}
gbla_status launch_delta_step(const gbla_delta_shape& s, const void*, const void*, const void*, const float*,
                              const float*, const int32_t*, int32_t slots, float*, void*, hipStream_t) {
  REQUIRE(grid_ok(s.batch, s.value_heads, 256) && slots >= 1);
  ++g_launches;
  return GBLA_OK;
}
static void check(const NormPlan& p) {
  REQUIRE(p.rows == 0 || grid_ok(p.blocks, 1, 256));
  REQUIRE(p.lanes * p.pieces * 8 >= p.width && (p.lanes == 8 || p.lanes * p.pieces * 4 < p.width));
  REQUIRE(p.lanes == 8 || p.lanes == 16 || p.lanes == 32 || p.lanes == 64 || p.lanes == 256);
  REQUIRE(p.pieces == 1 || p.pieces == 2 || p.pieces == 4 || (p.pieces == 8 && p.lanes == 256));
  REQUIRE(p.lanes < 256 || p.pieces > 1);
  ++g_launches;
}
gbla_status launch_norm(const NormPlan& p, const void*, const void*, const float*, void*, void*, float*, hipStream_t) {
  check(p);
  return GBLA_OK;
}
gbla_status launch_norm_backward(const NormPlan& p, const void*, const float*, const void*, const void*, void*, void*,
                                 float*, hipStream_t) {
  check(p);
  REQUIRE(norm_partial_bytes(p) >= (size_t)p.blocks * p.width * sizeof(float));
  return GBLA_OK;
}
}  // namespace gbla

namespace {

// Stand-in device pointers: aligned, never dereferenced by host code.
alignas(256) unsigned char g_buf[1024];
void* A() { return g_buf; }
float* F() { return reinterpret_cast<float*>(g_buf); }
const int32_t* I() { return reinterpret_cast<const int32_t*>(g_buf); }

void delta(int32_t B, int32_t n, int32_t H, int32_t V, int32_t d, int32_t msl, int32_t dtype, float scale = 0.125f) {
  fprintf(stderr, "delta B=%d n=%d H=%d V=%d d=%d max=%d dtype=%d\n", B, n, H, V, d, msl, dtype);
  const gbla_delta_shape s = {B, n, H, V, d, msl, dtype, scale};
  const size_t fwd = gbla_delta_workspace_bytes(&s), bwd = gbla_delta_backward_workspace_bytes(&s);
  REQUIRE((fwd == 0) == (bwd == 0) && bwd >= fwd && gbla_delta_ragged_workspace_bytes(&s) <= fwd);
  for (int ragged = 0; ragged < 2; ++ragged) {
    const int32_t* cu = ragged ? I() : nullptr;
    const int before = gbla::g_launches;
    const gbla_status a = gbla_delta_forward(&s, A(), A(), A(), F(), F(), F(), cu, A(), fwd, A(), F(), nullptr);
    const gbla_status b = gbla_delta_backward(&s, A(), A(), A(), F(), F(), F(), cu, A(), F(), A(), bwd, A(), A(), A(),
                                              F(), F(), F(), nullptr);
    REQUIRE(gbla::g_launches - before == (a == GBLA_OK) + (b == GBLA_OK));
    REQUIRE(fwd > 0 || (a != GBLA_OK && b != GBLA_OK));
    if (a == GBLA_OK)
      REQUIRE(gbla_delta_forward(&s, A(), A(), A(), F(), F(), F(), cu, A(), 0, A(), F(), nullptr) == GBLA_ERR_WORKSPACE);
  }
  gbla_delta_step(&s, A(), A(), A(), F(), F(), I(), 1, F(), A(), nullptr);
}

void norm(int64_t rows, int32_t width, int32_t dtype, int32_t out, int32_t group, float eps = 1e-6f) {
  fprintf(stderr, "norm rows=%lld width=%d dtype=%d out=%d group=%d\n", (long long)rows, width, dtype, out, group);
  const gbla_norm_shape s = {rows, width, dtype, out, group, eps};
  const size_t bytes = gbla_add_norm_backward_workspace_bytes(&s);
  gbla_add_norm(&s, A(), A(), F(), A(), A(), F(), nullptr);
  gbla_add_norm(&s, A(), nullptr, F(), nullptr, A(), F(), nullptr);
  const gbla_status st = gbla_add_norm_backward(&s, A(), F(), A(), A(), A(), bytes, A(), F(), nullptr);
  REQUIRE((st == GBLA_OK) == (bytes > 0));
}

}  // namespace

int main() {
  const int32_t dims[3] = {32, 64, 128}, types[2] = {GBLA_F32, GBLA_BF16};
  for (int32_t d : dims)
    for (int32_t t : types) {
      delta(1, 1, 1, 1, d, 0, t);
      delta(1, 0, 2, 8, d, 0, t);
      delta(64, 0, 8, 8, d, 0, t);
      delta(8, 257, 3, 6, d, 257, t);
      delta(1, 32768, 8, 8, d, 0, t);
      delta(64, 177929, 4, 8, d, 17201, t);
      delta(1, INT32_MAX, 1, 1, d, INT32_MAX, t);
      delta(1, INT32_MAX, 65535, 65535, d, 0, t);
      delta(INT32_MAX, 1, 1, 1, d, 1, t);
      delta(INT32_MAX, INT32_MAX, 65535, 65535, d, 1, t);
      delta(131072, 4096, 1, 1, d, 4096, t);
      delta(1100000, 200, 1, 1, d, 200, t);
      delta(8388607, 1, 1, 2, d, 1, t);
      delta(8388608, 1, 1, 2, d, 1, t);
      delta(1, 64, 5, 65535, d, 64, t);
    }
  for (int32_t t : types)
    for (int32_t width = 8; width <= 16384; width += width < 600 ? 8 : 1144) {
      for (int64_t rows : {(int64_t)0, (int64_t)1, (int64_t)31, (int64_t)100000, (int64_t)1 << 40}) {
        norm(rows, width, t, t, 0);
        norm(rows, width, t, GBLA_E4M3, 0);
        norm(rows, width, t, GBLA_E4M3, 128);
      }
    }
  // refused before any arithmetic
  delta(0, 1, 1, 1, 64, 0, GBLA_BF16);
  delta(1, -1, 1, 1, 64, 0, GBLA_BF16);
  delta(1, 1, 0, 1, 64, 0, GBLA_BF16);
  delta(1, 1, 1, 0, 64, 0, GBLA_BF16);
  delta(1, 1, 2, 3, 64, 0, GBLA_BF16);
  delta(1, 1, 1, 1, 48, 0, GBLA_BF16);
  delta(1, 1, 1, 1, 64, 0, 2);
  delta(1, 1, 1, 1, 64, INT32_MIN, GBLA_BF16);
  delta(1, 1, 1, 65536, 64, 0, GBLA_BF16);
  delta(1, 1, 1, 1, 64, 0, GBLA_BF16, INFINITY);
  delta(1, 1, 1, 1, 64, 0, GBLA_BF16, NAN);
  norm(-1, 64, GBLA_BF16, GBLA_BF16, 0);
  norm(INT64_MAX, 16384, GBLA_BF16, GBLA_BF16, 0);
  norm(INT64_MIN, 64, GBLA_BF16, GBLA_BF16, 0);
  norm(1, INT32_MIN, GBLA_BF16, GBLA_BF16, 0);
  norm(1, INT32_MAX, GBLA_BF16, GBLA_BF16, 0);
  norm(1, 64, 5, 5, 0);
  norm(1, 64, GBLA_BF16, GBLA_BF16, INT32_MIN);
  norm(1, 64, GBLA_BF16, GBLA_BF16, 0, NAN);
  REQUIRE(gbla_delta_workspace_bytes(nullptr) == 0 && gbla_add_norm_backward_workspace_bytes(nullptr) == 0);
  printf("host block ok (%d stub launches)\n", gbla::g_launches);
  return 0;
}
