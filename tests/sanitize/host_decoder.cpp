// Host-only driver for the sanitizer test: the plans and the argument checks of the
// decoder's operators (gbla_decay_plan.cpp, gbla_decay_api.cpp), built with
// -fsanitize=address,undefined and the kernel launchers replaced by stubs that check
// the grids they would build.  Prints "host decoder ok" at the end.
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include "gbla.h"
#include "gbla_decay.h"

#define REQUIRE(cond)                                                            \
  do {                                                                           \
    if (!(cond)) {                                                               \
      fprintf(stderr, "host_decoder: %s failed at line %d\n", #cond, __LINE__); \
      abort();                                                                   \
    }                                                                            \
  } while (0)

namespace gbla {
static int g_launches = 0;

static bool grid_ok(int64_t x, int64_t y, int threads) {
  return x >= 1 && x * threads <= (int64_t)UINT32_MAX && y >= 1 && y <= 65535;
}

static void check(const DecayPlan& p, bool backward) {
  const int64_t groups = p.grid_units;
  REQUIRE(grid_ok(groups, p.kv_heads, p.d == 128 ? 512 : 256));
  REQUIRE(grid_ok((groups + 7) / 8 * 16, p.kv_heads, p.d == 128 ? 256 : 1));  // walks of two halves
  if (!p.single) REQUIRE(grid_ok((int64_t)p.nseq * (p.d * p.d / (backward ? 128 : 256)), p.kv_heads, 256));
  REQUIRE(p.group * p.kv_heads == p.heads);
  REQUIRE(p.unit >= 2 * kTile && p.unit <= kMaxUnit && (p.unit & (p.unit - 1)) == 0);
  REQUIRE(p.units >= 1 && (p.single ? p.grid_units == p.nseq : p.grid_units == p.units));
  const size_t state = (size_t)p.d * p.d * sizeof(float);
  REQUIRE(p.off_S + (size_t)p.units * p.kv_heads * state <= p.total_bytes);
  if (backward) {
    REQUIRE(p.off_D >= p.off_S + (size_t)p.units * p.kv_heads * state);
    REQUIRE(p.off_dg >= p.off_D + (size_t)p.units * p.kv_heads * state);
    REQUIRE(p.off_dg + 2 * (size_t)p.kv_heads * p.grid_units * 8 * sizeof(double) <= p.total_bytes);
  }
  ++g_launches;
}

gbla_status launch_decay_forward(const DecayPlan& p, const void*, const void*, const void*, const float*,
                                 const float*, const int32_t*, void*, void*, float*, hipStream_t) {
  check(p, false);
  return GBLA_OK;
}
gbla_status launch_decay_backward(const DecayPlan& p, const void*, const void*, const void*, const float*,
                                  const float*, const int32_t*, const void*, const float*, void*, void*,
                                  void*, void*, float*, float*, hipStream_t) {
  check(p, true);
  return GBLA_OK;
}
gbla_status launch_decay_step(const gbla_decay_shape& s, const void*, const void*, const void*, const float*,
                              const int32_t*, int32_t slots, float*, void*, hipStream_t) {
  REQUIRE(grid_ok(s.batch, s.kv_heads, 256) && slots >= 1);
  ++g_launches;
  return GBLA_OK;
}
static void check(const RopePlan& p) {
  REQUIRE(grid_ok(p.tokens > 0 ? p.blocks : 1, p.head_blocks, 256));
  REQUIRE((int64_t)p.blocks * p.passes * p.tile >= p.tokens);
  REQUIRE((int64_t)p.head_blocks * p.heads_each >= (int64_t)p.heads + p.kv_heads && p.heads_each <= 8);
  for (int i = 0; i < p.rotary / 2; ++i) REQUIRE(p.turns[i] > 0.0);
  ++g_launches;
}
gbla_status launch_rope(const RopePlan& p, const void*, const void*, const float*, const float*,
                        const int32_t*, const int32_t*, void*, void*, hipStream_t) {
  check(p);
  return GBLA_OK;
}
gbla_status launch_rope_backward(const RopePlan& p, const void*, const void*, const float*, const float*,
                                 const int32_t*, const int32_t*, const void*, const void*, void*, void*,
                                 void*, float*, float*, hipStream_t) {
  check(p);
  return GBLA_OK;
}
}  // namespace gbla

namespace {

// Stand-in device pointers: aligned, never dereferenced by host code.
alignas(256) unsigned char g_buf[1024];
void* A() { return g_buf; }
float* F() { return reinterpret_cast<float*>(g_buf); }
const int32_t* I() { return reinterpret_cast<const int32_t*>(g_buf); }

void decay(int32_t B, int32_t n, int32_t H, int32_t K, int32_t d, int32_t msl, int32_t dtype,
           float scale = 0.125f) {
  fprintf(stderr, "decay B=%d n=%d H=%d K=%d d=%d max=%d dtype=%d\n", B, n, H, K, d, msl, dtype);
  const gbla_decay_shape s = {B, n, H, K, d, msl, dtype, scale};
  const size_t fwd = gbla_decay_workspace_bytes(&s), bwd = gbla_decay_backward_workspace_bytes(&s);
  REQUIRE((fwd == 0) == (bwd == 0) && bwd >= fwd);
  for (int ragged = 0; ragged < 2; ++ragged) {
    const int32_t* cu = ragged ? I() : nullptr;
    const int before = gbla::g_launches;
    const gbla_status a = gbla_decay_forward(&s, A(), A(), A(), F(), F(), cu, A(), fwd, A(), F(), nullptr);
    const gbla_status b = gbla_decay_backward(&s, A(), A(), A(), F(), F(), cu, A(), F(), A(), bwd, A(), A(),
                                              A(), F(), F(), nullptr);
    REQUIRE(gbla::g_launches - before == (a == GBLA_OK) + (b == GBLA_OK));
    REQUIRE(fwd > 0 || (a != GBLA_OK && b != GBLA_OK));
    if (a == GBLA_OK)  // one byte less than the shape may need refuses at least one reading
      REQUIRE(gbla_decay_forward(&s, A(), A(), A(), F(), F(), cu, A(), 0, A(), F(), nullptr) ==
              GBLA_ERR_WORKSPACE);
  }
  gbla_decay_step(&s, A(), A(), A(), F(), I(), 1, F(), A(), nullptr);
}

void rope(int32_t B, int32_t n, int32_t H, int32_t K, int32_t d, int32_t R, int32_t dtype, float eps,
          float theta, uint32_t flags) {
  fprintf(stderr, "rope B=%d n=%d H=%d K=%d d=%d R=%d dtype=%d flags=%u\n", B, n, H, K, d, R, dtype, flags);
  const gbla_rope_shape s = {B, n, H, K, d, R, dtype, eps, theta, flags};
  const size_t bytes = gbla_qk_norm_rope_backward_workspace_bytes(&s);
  for (int ragged = 0; ragged < 2; ++ragged) {
    const int32_t* cu = ragged ? I() : nullptr;
    gbla_qk_norm_rope(&s, A(), A(), F(), F(), I(), cu, A(), A(), nullptr);
    gbla_qk_norm_rope(&s, A(), A(), nullptr, nullptr, nullptr, cu, A(), A(), nullptr);
    gbla_qk_norm_rope_backward(&s, A(), A(), F(), F(), I(), cu, A(), A(), A(), bytes, A(), A(), F(), F(),
                               nullptr);
  }
}

}  // namespace

int main() {
  const int32_t dims[3] = {32, 64, 128}, types[2] = {GBLA_F32, GBLA_BF16};
  for (int32_t d : dims)
    for (int32_t t : types) {
      decay(1, 1, 1, 1, d, 0, t);
      decay(1, 0, 8, 2, d, 0, t);
      decay(64, 0, 8, 8, d, 0, t);
      decay(8, 257, 6, 3, d, 257, t);
      decay(1, 32768, 8, 8, d, 0, t);
      decay(64, 177929, 8, 2, d, 8000, t);
      decay(1, INT32_MAX, 1, 1, d, INT32_MAX, t);
      decay(1, INT32_MAX, 65535, 65535, d, 0, t);
      decay(INT32_MAX, 1, 1, 1, d, 1, t);
      decay(INT32_MAX, INT32_MAX, 65535, 65535, d, 1, t);
      decay(131072, 4096, 1, 1, d, 4096, t);   // more states than a scan's grid takes at d = 128
      decay(8388599, 1, 2, 1, d, 1, t);
      decay(8388600, 1, 2, 1, d, 1, t);
      decay(1, 64, 65535, 5, d, 64, t);
      rope(1, 1, 1, 1, d, d, t, 1e-6f, 1e4f, 0);
      rope(1, 0, 8, 2, d, 0, t, 0.0f, 1e4f, GBLA_NO_NORM);
      rope(3, 33, 5, 1, d, 8, t, 1e-6f, 1e-30f, GBLA_ROPE_PAIRS);
      rope(1, INT32_MAX, 1, 1, d, d, t, 1e-6f, 3e38f, 0);
      rope(INT32_MAX, INT32_MAX, 65535, 65535, d, d, t, 1e-6f, 1e4f, 0);
      rope(INT32_MAX, 1, 65535, 1, d, d, t, 1e-6f, 1e4f, GBLA_ROPE_PAIRS);
    }
  // refused before any arithmetic
  decay(0, 1, 1, 1, 64, 0, GBLA_BF16);
  decay(1, -1, 1, 1, 64, 0, GBLA_BF16);
  decay(1, 1, 0, 1, 64, 0, GBLA_BF16);
  decay(1, 1, 1, 0, 64, 0, GBLA_BF16);
  decay(1, 1, 3, 2, 64, 0, GBLA_BF16);
  decay(1, 1, 1, 1, 48, 0, GBLA_BF16);
  decay(1, 1, 1, 1, 64, 0, 2);
  decay(1, 1, 1, 1, 64, -1, GBLA_BF16);
  decay(1, 1, 1, 1, 64, INT32_MIN, GBLA_BF16);
  decay(1, 1, 65536, 1, 64, 0, GBLA_BF16);
  decay(1, 1, 1, 1, 64, 0, GBLA_BF16, INFINITY);
  decay(1, 1, 1, 1, 64, 0, GBLA_BF16, NAN);
  rope(0, 1, 1, 1, 64, 64, GBLA_BF16, 1e-6f, 1e4f, 0);
  rope(1, -1, 1, 1, 64, 64, GBLA_BF16, 1e-6f, 1e4f, 0);
  rope(1, 1, 1, 1, 64, 4, GBLA_BF16, 1e-6f, 1e4f, 0);
  rope(1, 1, 1, 1, 64, 72, GBLA_BF16, 1e-6f, 1e4f, 0);
  rope(1, 1, 1, 1, 64, -8, GBLA_BF16, 1e-6f, 1e4f, 0);
  rope(1, 1, 1, 1, 64, 64, GBLA_BF16, -1.0f, 1e4f, 0);
  rope(1, 1, 1, 1, 64, 64, GBLA_BF16, 1e-6f, 0.0f, 0);
  rope(1, 1, 1, 1, 64, 64, GBLA_BF16, 1e-6f, NAN, 0);
  rope(1, 1, 1, 1, 64, 64, GBLA_BF16, 1e-6f, 1e4f, 64);
  REQUIRE(gbla_decay_workspace_bytes(nullptr) == 0 && gbla_qk_norm_rope_backward_workspace_bytes(nullptr) == 0);
  printf("host decoder ok (%d stub launches)\n", gbla::g_launches);
  return 0;
}
