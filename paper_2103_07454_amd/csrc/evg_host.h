// What the host sides of the library share: error texts and the checks of device pointers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/evg.h"

namespace evg {

// Leaves the text for evg_error_text and returns the status.
evg_status fail(evg_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

// Device memory of the current device, and `bytes` of it from p on?
evg_status check_device_array(const void* p, uint64_t bytes, const char* what);

}  // namespace evg

#define HIP_TRY(expr)                                                                             \
  do {                                                                                            \
    hipError_t e_ = (expr);                                                                       \
    if (e_ != hipSuccess)                                                                         \
      return evg::fail(e_ == hipErrorOutOfMemory ? EVG_ERR_OOM : EVG_ERR_HIP, "%s: %s", #expr,    \
                       hipGetErrorString(e_));                                                    \
  } while (0)
