// launch.cuh -- host side of the layer operators' launches.
#pragma once
#include <atomic>
#include <cstdint>

#include <cuda_runtime.h>

namespace rdn {
// Lets a kernel have `bytes` of dynamic shared memory (beyond 48 KB, always as many for one kernel) on the
// current device.  A call of a few microseconds on the device asks once, not every time (a microsecond).
template <auto kKernel>
cudaError_t let_smem(int bytes) {
  static std::atomic<uint64_t> done{0};  // a bit for each device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
  return e;
}
}  // namespace rdn
