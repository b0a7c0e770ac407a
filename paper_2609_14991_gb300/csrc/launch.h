// What a launch asks of the runtime, kept per device.
#pragma once

#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

namespace tsd {

// Lets a kernel take that much dynamic shared memory; asked of the runtime once per device.
template <auto KERNEL>
cudaError_t smem_opt_in(int bytes) {
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (dev < 64 && (done.load() >> dev & 1))) return e;
  e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess && dev < 64) done.fetch_or(uint64_t(1) << dev);
  return e;
}

// The current device's SMs.
cudaError_t device_sms(int* sms);

}  // namespace tsd
