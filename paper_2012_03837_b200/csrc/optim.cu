// Fused multi-tensor optimizer update over the whole parameter arena (each chunk's parameters are
// updated from that chunk's own gradients only, Sec. 1 / Sec. 6: the update is element-wise, so one
// flat sweep applies all K per-chunk updates).
#include "common.cuh"
#include "optim_update.cuh"

namespace lp {
namespace {

// 4 elements per thread, 128-bit accesses (optim_update4).
template <bool PER_CHUNK>
__global__ void __launch_bounds__(256) optim_kernel(OptimArgs a) {
  long long i4 = ((long long)blockIdx.x * blockDim.x + threadIdx.x) * 4;
  if (i4 >= a.n_total) return;   // the arena length is a multiple of 4
  optim_update4<PER_CHUNK>(a, i4);
}

__global__ void __launch_bounds__(256) mask_losses_kernel(float* losses, const float4* chunk_tab, int K) {
  int k = blockIdx.x * blockDim.x + threadIdx.x;
  if (k < K && chunk_tab[k].x == 0.f) losses[k] = __int_as_float(0x7fc00000);
}

}  // namespace

void launch_optim(const OptimArgs& a, cudaStream_t s) {
  long long threads = (a.n_total + 3) / 4;
  if (threads == 0) return;
  if (a.seg_end) optim_kernel<true><<<(unsigned)((threads + 255) / 256), 256, 0, s>>>(a);
  else optim_kernel<false><<<(unsigned)((threads + 255) / 256), 256, 0, s>>>(a);
}

void launch_mask_losses(float* losses, const float4* chunk_tab, int K, cudaStream_t s) {
  mask_losses_kernel<<<(K + 255) / 256, 256, 0, s>>>(losses, chunk_tab, K);
}

}  // namespace lp
