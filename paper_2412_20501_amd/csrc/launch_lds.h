// Launches with more LDS than the default limit.
#pragma once
#include <atomic>

#include "tr_internal.h"

namespace tr {
namespace {

// Lets a kernel ask for more LDS than the default limit, once for each device.
template <typename Kernel>
hipError_t raise_lds(Kernel kernel, std::atomic<uint64_t>& raised, int lds_bytes) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev >= 0 && dev < 64 ? (uint64_t)1 << dev : 0;
  if (!(raised.load(std::memory_order_acquire) & bit)) {
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes);
    if (e != hipSuccess) return e;
    raised.fetch_or(bit, std::memory_order_release);
  }
  return hipSuccess;
}
template <typename Kernel, typename... Args>
hipError_t launch_lds(Kernel kernel, std::atomic<uint64_t>& raised, dim3 grid, dim3 block, int lds_bytes, hipStream_t stream, Args... args) {
  const hipError_t e = raise_lds(kernel, raised, lds_bytes);
  return e != hipSuccess ? e : launch_kernel(kernel, grid, block, lds_bytes, stream, args...);
}

}  // namespace
}  // namespace tr
