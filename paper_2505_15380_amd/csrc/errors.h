// The message behind ssd_last_error() and the checks of HIP calls, for every file of the library.
#pragma once
#include "../../include/ssd.h"

#include <hip/hip_runtime.h>

namespace ssd {
// Remembers the message for the calling thread and returns `code`.
__attribute__((visibility("hidden"))) int fail(int code, const char* fmt, ...);
}  // namespace ssd

#define HIP_TRY(expr)                                                                      \
  do {                                                                                     \
    hipError_t e_ = (expr);                                                                \
    if (e_ != hipSuccess) return fail(SSD_EHIP, "%s: %s", #expr, hipGetErrorString(e_));   \
  } while (0)
#define LAUNCH_CHECK() HIP_TRY(hipGetLastError())
