// What the C entry points of every source file share: the thread's last error message and the macros that return it.
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/jacobi_made.h"

namespace jm {

// Keeps the message for made_last_error() and returns `code`.
__attribute__((visibility("hidden"), format(printf, 2, 3))) int fail(int code, const char* fmt, ...);

}  // namespace jm

#define HIP_TRY(expr)                                                                               \
  do {                                                                                              \
    hipError_t e_ = (expr);                                                                         \
    if (e_ != hipSuccess)                                                                           \
      return fail(e_ == hipErrorOutOfMemory ? MADE_ERR_NOMEM : MADE_ERR_HIP, "%s failed: %s (%s:%d)", #expr, \
                  hipGetErrorString(e_), __FILE__, __LINE__);                                       \
  } while (0)

#define TRY(expr)            \
  do {                       \
    int rc_ = (expr);        \
    if (rc_ != MADE_OK) return rc_; \
  } while (0)
