// What the host side of the operators around the decision step shares: checks and
// launches.

#ifndef ASYMSPEC_STEP_LAUNCH_H_
#define ASYMSPEC_STEP_LAUNCH_H_

#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <cstring>

#include "asymspec.h"

namespace asym_step {

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

// Compute units of the current device, or 0 when it is no gfx950.
inline int device_cus() {
  static std::atomic<int> cus[64];       // 0: not looked at; -1: not a gfx950
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) {
    (void)hipGetLastError();
    return 0;
  }
  int n = cus[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    hipDeviceProp_t pr;
    if (hipGetDeviceProperties(&pr, dev) != hipSuccess) {
      (void)hipGetLastError();
      return 0;
    }
    n = std::strncmp(pr.gcnArchName, "gfx950", 6) == 0 ? pr.multiProcessorCount : -1;
    cus[dev].store(n, std::memory_order_relaxed);
  }
  return std::max(n, 0);
}

// A launch has fewer than 2^32 threads.
inline bool fits(long long grid, int threads) { return grid <= 0xFFFFFFFFll / threads; }

// Enqueues a kernel of one argument.
template <class Args>
inline int launch(void (*kernel)(Args), unsigned grid, int threads, size_t lds, void* stream, Args& args) {
  void* p[] = {&args};
  if (hipLaunchKernel((const void*)kernel, dim3(grid), dim3(threads), p, lds, (hipStream_t)stream) == hipSuccess)
    return ASYMSPEC_OK;
  (void)hipGetLastError();
  return ASYMSPEC_E_DEVICE;
}

}  // namespace asym_step

#endif  // ASYMSPEC_STEP_LAUNCH_H_
