// pdl.cuh -- launches that overlap with the end of the kernel before them
// (programmatic dependent launch).  A kernel launched by launch_overlapped
// may start while its predecessor's last CTAs still run; it sets up what is
// its own (barriers, tensor memory, shared memory) and calls
// after_predecessor() before its first access to global memory, which returns
// when the predecessor has finished and its writes are visible.
#pragma once

#include <atomic>
#include <cstdint>
#include <cuda_runtime.h>
#include <utility>

namespace soma {

__device__ __forceinline__ void after_predecessor() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
}
// The successor may be set up from here on (it still waits for this kernel's
// end before it touches memory).
__device__ __forceinline__ void admit_successor() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

template <typename... P, typename... A>
cudaError_t launch_overlapped(void (*kernel)(P...), dim3 grid, int threads, size_t smem,
                              cudaStream_t stream, A&&... args) {
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(std::forward<A>(args))...);
}

// Allows launches of KERNEL with up to `bytes` of dynamic shared memory on the
// current device; asked once for each device.
template <auto KERNEL>
cudaError_t allow_shared(size_t bytes) {
  static std::atomic<uint64_t> asked{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
  if (bit && (asked.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
  e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == cudaSuccess) asked.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

}  // namespace soma
