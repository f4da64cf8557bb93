// How a failing HIP call becomes a status (host code).
#pragma once

#include <hip/hip_runtime_api.h>

namespace pipesd {

int hip_fail(hipError_t e, const char* what);  // keeps the text for pipesd_last_hip_error(); PIPESD_EHIP

}  // namespace pipesd

#define HIP_TRY(expr)                                 \
  do {                                                \
    hipError_t _e = (expr);                           \
    if (_e != hipSuccess) return hip_fail(_e, #expr); \
  } while (0)
