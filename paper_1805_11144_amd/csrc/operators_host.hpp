// Host-side helpers of operators.hip: a failed runtime call as an ms::Error, and
// the calling thread's device for the length of a scope.
#pragma once

#include <hip/hip_runtime.h>

#include <string>

#include "host.hpp"

#define HIPCHECK(expr)                                                                    \
  do {                                                                                    \
    hipError_t _e = (expr);                                                               \
    if (_e != hipSuccess)                                                                 \
      ms::fail(MS_E_HIP, std::string(#expr) + ": " + hipGetErrorString(_e));              \
  } while (0)

namespace ms {

struct DeviceGuard {
  int prev = 0;
  explicit DeviceGuard(int dev) {
    HIPCHECK(hipGetDevice(&prev));
    if (prev != dev) HIPCHECK(hipSetDevice(dev));
  }
  ~DeviceGuard() {
    int cur = 0;
    if (hipGetDevice(&cur) == hipSuccess && cur != prev) (void)hipSetDevice(prev);
  }
};

}  // namespace ms
