// Error reporting of the C ABI entry points: a thread's last message, and the
// checks that return it.
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/gart.h"

namespace gart {

// Stores the formatted message for gart_last_error and returns s.
gart_status fail(gart_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
void clear_error();

}  // namespace gart

#define GART_HIP(expr)                                                                   \
  do {                                                                                   \
    const hipError_t e_ = (expr);                                                        \
    if (e_ != hipSuccess) return fail(GART_ERR_HIP, "%s: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

#define GART_REQUIRE(cond, ...)                                   \
  do {                                                            \
    if (!(cond)) return fail(GART_ERR_INVALID_ARG, __VA_ARGS__); \
  } while (0)
