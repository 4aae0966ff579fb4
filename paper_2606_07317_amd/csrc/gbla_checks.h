// gbla_checks.h -- argument checks of the C entry points of the decoder's operators.
// Internal to libgbla.so; host code.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <initializer_list>

#include "gbla.h"
#include "gbla_plan.h"

#define GBLA_TRY(expr)                  \
  do {                                  \
    gbla_status _st = (expr);           \
    if (_st != GBLA_OK) return _st;     \
  } while (0)

namespace gbla {
namespace checks {

// Arrays in use: present, and aligned to `a` bytes.
inline gbla_status present(std::initializer_list<const void*> ptrs, size_t a = 16) {
  for (const void* p : ptrs) {
    if (!p) return GBLA_ERR_INVALID_ARGUMENT;
    if (!aligned(p, a)) return GBLA_ERR_MISALIGNED;
  }
  return GBLA_OK;
}

// Arrays over the tokens: of no elements, and so possibly NULL, where there are none.
inline gbla_status rows_present(int64_t tokens, std::initializer_list<const void*> ptrs, size_t a = 16) {
  return tokens > 0 ? present(ptrs, a) : GBLA_OK;
}

// Arrays that may be NULL.
inline gbla_status optional(std::initializer_list<const void*> ptrs, size_t a = 16) {
  for (const void* p : ptrs)
    if (p && !aligned(p, a)) return GBLA_ERR_MISALIGNED;
  return GBLA_OK;
}

inline gbla_status scratch(const void* ws, size_t have, size_t need) {
  if (!ws) return GBLA_ERR_WORKSPACE;
  if (!aligned(ws, 256)) return GBLA_ERR_MISALIGNED;
  return have < need ? GBLA_ERR_WORKSPACE : GBLA_OK;
}

inline size_t larger(size_t a, size_t b) { return a > b ? a : b; }

}  // namespace checks
}  // namespace gbla
