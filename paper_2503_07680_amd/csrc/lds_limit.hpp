// Kernels with more dynamic LDS than a launch has by default.
#pragma once
#include <hip/hip_runtime.h>

#include <atomic>

namespace hbp {

// Raises the kernel's limit on the current device, once for each device and kernel; returns hipError_t as int.  `done`: of that
// kernel, static.
struct LdsLimitDone {
  std::atomic<unsigned long long> devices{0};  // a bit each; further ones are asked every time
};
inline int raise_lds_limit(const void* kernel, int bytes, LdsLimitDone& done) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return (int)e;
  const unsigned long long bit = dev >= 0 && dev < 64 ? 1ull << dev : 0;
  if (done.devices.load(std::memory_order_relaxed) & bit) return 0;
  e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) done.devices.fetch_or(bit, std::memory_order_relaxed);
  return (int)e;
}

}  // namespace hbp
