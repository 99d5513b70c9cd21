// Dropout whose mask is never stored: element i is kept or dropped by one word of a counter-based generator, so the
// gradient's pass forms the same mask again from the same key and counters.
//
//   word(i) = word i mod 4 of Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2,
//             3", SC 2011) with key = seed and counter = {lo(o + i div 4), hi(o + i div 4), w2, w3}
//   y[i]    = resid[i] + (word(i) >= floor(p 2^32) ? x[i] * 1/(1-p) : 0)
//
// A dropped element is selected away, not multiplied by zero: a NaN or an infinity there does not reach y.
// Sums and products are in fp32 and rounded once, on storing.
#include "common.cuh"
#include "launch.cuh"

namespace lp {
namespace {

__device__ __forceinline__ uint4 philox10(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const unsigned long long a = (unsigned long long)c0 * 0xD2511F53u, b = (unsigned long long)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}

__device__ __forceinline__ uint4 words(const DropoutArgs& a, unsigned long long first, long long group) {
  const unsigned long long c = first + (unsigned long long)group;
  return philox10((uint32_t)c, (uint32_t)(c >> 32), a.w2, a.w3, (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
}

__device__ __forceinline__ float drop(const DropoutArgs& a, uint32_t w, float x, float r) {
  return w >= a.threshold ? fmaf(x, a.scale, r) : r;
}

// One thread per group of four elements; any alignment.
template <typename T>
__global__ void __launch_bounds__(256) dropout_kernel(DropoutArgs a) {
  const long long groups = (a.n + 3) / 4;
  const unsigned long long first = a.offset + (a.offset_dev ? *a.offset_dev : 0ull);
  for (long long g = (long long)blockIdx.x * blockDim.x + threadIdx.x; g < groups; g += (long long)gridDim.x * blockDim.x) {
    const uint4 w = words(a, first, g);
    const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const long long i = 4 * g + e;
      if (i < a.n) {
        const float r = a.resid ? to_f(((const T*)a.resid)[i]) : 0.f;
        ((T*)a.y)[i] = from_f<T>(drop(a, ww[e], to_f(((const T*)a.x)[i]), r));
      }
    }
  }
}

}  // namespace

cudaError_t launch_dropout(const DropoutArgs& a, bool is_bf16, cudaStream_t s) {
  if (a.n <= 0) return cudaSuccess;
  const long long groups = (a.n + 3) / 4;
  const unsigned blocks = (unsigned)std::min<long long>((groups + 255) / 256, 148 * 16);
  return is_bf16 ? launch_kernel(dropout_kernel<bf16>, dim3(blocks), 256, 0, s, a)
                 : launch_kernel(dropout_kernel<float>, dim3(blocks), 256, 0, s, a);
}

}  // namespace lp
