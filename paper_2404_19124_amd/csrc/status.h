// Errors of the C ABI's entry points: the message of the calling thread (spec_last_error) and the status to return.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/spec.h"

namespace specdraft {

spec_status_t fail(spec_status_t code, const char* fmt, ...);
spec_status_t hip_fail(hipError_t e, const char* what);

}  // namespace specdraft

#define HIP_TRY(expr)                                  \
  do {                                                 \
    hipError_t e_ = (expr);                            \
    if (e_ != hipSuccess) return hip_fail(e_, #expr);  \
  } while (0)
