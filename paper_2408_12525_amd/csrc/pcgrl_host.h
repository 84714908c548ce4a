// What the host sides of the library's translation units share.
#pragma once
#include <hip/hip_runtime.h>

struct pcgrl_ctx;

namespace pcgrl {

// The device that a context lives on and its numbers of tile types and of environments.
int device_of(const pcgrl_ctx* ctx);
int tiles_in(const pcgrl_ctx* ctx);
int levels_of(const pcgrl_ctx* ctx);

struct DeviceGuard {
  int prev = -1;
  bool ok = true;
  explicit DeviceGuard(int dev) {
    if (hipGetDevice(&prev) != hipSuccess) prev = -1;
    ok = hipSetDevice(dev) == hipSuccess;
  }
  ~DeviceGuard() {
    if (prev >= 0) (void)hipSetDevice(prev);
  }
};

}  // namespace pcgrl
