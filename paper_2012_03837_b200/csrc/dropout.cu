// Dropout whose mask is never stored: element i is kept or dropped by one word of a counter-based generator, so the
// gradient's pass forms the same mask again from the same key and counters.
//
//   word(i) = word i mod 4 of Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2,
//             3", SC 2011) with key = seed and counter = {lo(o + i div 4), hi(o + i div 4), w2, w3}
//   y[i]    = resid[i] + (word(i) >= floor(p 2^32) ? x[i] * 1/(1-p) : 0)
//
// A dropped element is selected away, not multiplied by zero: a NaN or an infinity there does not reach y.
// Sums and products are in fp32 and rounded once, on storing.
//
// What bounds it: memory where three tensors pass (33.5 M bf16 with residual: 31 to 33 us in a replayed graph, 6.1 to 6.5 TB/s, 33
// to 35 us as a call among others; fp32 60 us, 6.7 TB/s), the generator's instructions where two bf16 tensors do (30 to 33 us
// against 20 for the bytes: twenty wide products and twenty three-way exclusive-ors per four elements, about 150 instructions
// per eight; fp32 45 against 41).  Sixteen random bits per element would
// halve that and tie p to multiples of 2^-16; a loop over blocks that fetches ahead was slower (35 to 41 us).
#include <algorithm>

#include "common.cuh"
#include "launch.cuh"

namespace lp {
namespace {

// The arguments and the ten rounds' keys, formed on the host: as kernel parameters they are operands of the rounds' own
// instructions.
struct Args : DropoutArgs {
  uint32_t k0[10], k1[10];
  explicit Args(const DropoutArgs& a) : DropoutArgs(a) {
    for (uint32_t r = 0; r < 10; ++r) {
      k0[r] = (uint32_t)seed + r * 0x9E3779B9u;
      k1[r] = (uint32_t)(seed >> 32) + r * 0xBB67AE85u;
    }
  }
};

__device__ __forceinline__ uint4 words(const Args& a, unsigned long long first, long long group) {
  const unsigned long long c = first + (unsigned long long)group;
  uint32_t c0 = (uint32_t)c, c1 = (uint32_t)(c >> 32), c2 = a.w2, c3 = a.w3;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const unsigned long long x = (unsigned long long)c0 * 0xD2511F53u, y = (unsigned long long)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(y >> 32) ^ c1 ^ a.k0[r];
    c1 = (uint32_t)y;
    c2 = (uint32_t)(x >> 32) ^ c3 ^ a.k1[r];
    c3 = (uint32_t)x;
  }
  return make_uint4(c0, c1, c2, c3);
}

// A predicated multiply-add: selecting an operand would go through the pipe that the generator's rounds keep busy.
__device__ __forceinline__ float drop(const Args& a, uint32_t w, float x, float r) {
  if (w >= a.threshold) r = fmaf(x, a.scale, r);
  return r;
}

// 16 bytes per thread and load, U of them in flight (with the residual's); the generator's arithmetic fills the wait.
// A block covers U * 256 consecutive vectors; the elements behind the last whole vector go one by one.
template <typename T, bool RESID, int U>
__global__ void __launch_bounds__(256) dropout_vec_kernel(const __grid_constant__ Args a) {
  cudaGridDependencySynchronize();
  constexpr int VEC = 16 / sizeof(T);
  const long long vecs = a.n / VEC, v0 = (long long)blockIdx.x * (256 * U) + threadIdx.x;
  const unsigned long long first = a.offset + (a.offset_dev ? *a.offset_dev : 0ull);
  uint4 x[U], r[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (v0 + 256 * u < vecs) {
      x[u] = ((const uint4*)a.x)[v0 + 256 * u];
      if (RESID) r[u] = ((const uint4*)a.resid)[v0 + 256 * u];
    }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long long v = v0 + 256 * u;
    if (v >= vecs) break;
    const uint32_t xs[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
    const uint32_t rs[4] = {r[u].x, r[u].y, r[u].z, r[u].w};
    uint32_t ys[4];
#pragma unroll
    for (int k = 0; k < VEC / 4; ++k) {          // a counter per four elements
      const uint4 w = words(a, first, v * (VEC / 4) + k);
      const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
      if (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          ys[e] = __float_as_uint(drop(a, ww[e], __uint_as_float(xs[e]), RESID ? __uint_as_float(rs[e]) : 0.f));
      } else {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t xx = xs[2 * k + e], rr = RESID ? rs[2 * k + e] : 0u;
          float lo = __uint_as_float(rr << 16), hi = __uint_as_float(rr & 0xffff0000u);
          if (ww[2 * e] >= a.threshold) lo = fmaf(__uint_as_float(xx << 16), a.scale, lo);
          if (ww[2 * e + 1] >= a.threshold) hi = fmaf(__uint_as_float(xx & 0xffff0000u), a.scale, hi);
          __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
          ys[2 * k + e] = *(uint32_t*)&b;
        }
      }
    }
    ((uint4*)a.y)[v] = make_uint4(ys[0], ys[1], ys[2], ys[3]);
  }
  const long long i = vecs * VEC + threadIdx.x;
  if (blockIdx.x == 0 && i < a.n) {
    const uint4 w = words(a, first, i >> 2);
    const uint32_t ww = (i & 3) == 0 ? w.x : (i & 3) == 1 ? w.y : (i & 3) == 2 ? w.z : w.w;
    ((T*)a.y)[i] = from_f<T>(drop(a, ww, to_f(((const T*)a.x)[i]), RESID ? to_f(((const T*)a.resid)[i]) : 0.f));
  }
}

// One thread per group of four elements; any alignment.
template <typename T>
__global__ void __launch_bounds__(256) dropout_kernel(const __grid_constant__ Args a) {
  cudaGridDependencySynchronize();
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

template <typename T>
cudaError_t run_vec(const Args& a, cudaStream_t s) {
  const long long vecs = a.n / (16 / (int)sizeof(T));
  const bool many = vecs >= 148LL * 8 * 256 * 2;   // more than two waves of single loads: four in flight per thread
  const unsigned blocks = (unsigned)std::max<long long>(1, many ? (vecs + 1023) / 1024 : (vecs + 255) / 256);
  if (a.resid) return many ? launch_after(dropout_vec_kernel<T, true, 4>, dim3(blocks), 256, 0, s, a) : launch_after(dropout_vec_kernel<T, true, 1>, dim3(blocks), 256, 0, s, a);
  return many ? launch_after(dropout_vec_kernel<T, false, 4>, dim3(blocks), 256, 0, s, a) : launch_after(dropout_vec_kernel<T, false, 1>, dim3(blocks), 256, 0, s, a);
}

}  // namespace

cudaError_t launch_dropout(const DropoutArgs& in, bool is_bf16, cudaStream_t s) {
  const Args a(in);
  if (a.n <= 0) return cudaSuccess;
  if ((((uintptr_t)a.x | (uintptr_t)a.resid | (uintptr_t)a.y) & 15) == 0) return is_bf16 ? run_vec<bf16>(a, s) : run_vec<float>(a, s);
  const long long groups = (a.n + 3) / 4;
  const unsigned blocks = (unsigned)std::min<long long>((groups + 255) / 256, 148 * 16);
  return is_bf16 ? launch_after(dropout_kernel<bf16>, dim3(blocks), 256, 0, s, a)
                 : launch_after(dropout_kernel<float>, dim3(blocks), 256, 0, s, a);
}

}  // namespace lp
