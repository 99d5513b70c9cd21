// Host-side launch helpers of the language-model operators.  Launches report their own status, so an error that
// an earlier, unrelated call left pending is neither taken for theirs nor cleared.
#pragma once
#include <atomic>
#include <utility>

#include <cuda_runtime.h>

namespace lp {

// Raises a kernel's dynamic shared-memory limit once per device.
struct SmemLimit {
  std::atomic<unsigned long long> done{0};
  cudaError_t raise(const void* kernel, int bytes) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = 1ull << (dev & 63);
    if (dev < 64 && (done.load(std::memory_order_acquire) & bit)) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && dev < 64) done.fetch_or(bit, std::memory_order_release);
    return e;
  }
};

// Launches a kernel that waits for its predecessor on the stream itself: cudaGridDependencySynchronize() before anything
// else, so its blocks are set up while the predecessor drains.
template <typename... KArgs, typename... Args>
cudaError_t launch_after(void (*kernel)(KArgs...), dim3 grid, int threads, size_t smem, cudaStream_t s, Args&&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}

}  // namespace lp
