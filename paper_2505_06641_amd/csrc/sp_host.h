// Host-side helpers that the C entry points share.
#pragma once
#include <hip/hip_runtime.h>

#include <string>

namespace sp {

struct DeviceGuard {
  int prev = -1;
  bool ok = true;
  explicit DeviceGuard(int dev) {
    if (hipGetDevice(&prev) != hipSuccess) prev = -1;
    if (prev != dev) ok = hipSetDevice(dev) == hipSuccess;
  }
  ~DeviceGuard() {
    if (prev >= 0) (void)hipSetDevice(prev);
  }
};

}  // namespace sp

#define SP_HIP(ctx, call)                                                          \
  do {                                                                             \
    hipError_t e_ = (call);                                                        \
    if (e_ != hipSuccess) {                                                        \
      (ctx)->hip_err = std::string(#call) + ": " + hipGetErrorString(e_);          \
      return SP_EDEVICE;                                                           \
    }                                                                              \
  } while (0)
