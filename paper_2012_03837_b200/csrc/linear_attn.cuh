// Shared by the two forms of the linear-attention scan (linear_attn.cu, linear_attn_tc.cu).
#pragma once
#include "common.cuh"
#include "launch.cuh"

namespace lp {

constexpr int LA_D = 64;                         // width of a head
constexpr int LA_STATE = LA_D * LA_D;            // elements of a state

// l^n for n >= 0, l = exp(lg), l^0 = 1 also for l = 0.  n lg is formed as a product and its rounding error, so that
// the error of the result stays that of one expf.
__device__ __forceinline__ float decay_pow(float lg, float n) {
  if (n == 0.f) return 1.f;
  const float x = n * lg, r = fmaf(n, lg, -x), e = expf(x);
  return r == r ? fmaf(e, r, e) : e;             // lg = -infinity: no correction
}

// Tokens [t0, t1) of sequence (b, h) that a block covers.
struct LaSpan { int b, h, t0, t1; };
__device__ __forceinline__ LaSpan la_span(const LinAttnArgs& a, int item) {
  LaSpan s;
  const int seg = item % a.n_seg, bh = item / a.n_seg;
  s.h = bh % a.H;
  s.b = bh / a.H;
  const int len = a.lengths ? min(max(a.lengths[s.b], 0), a.T) : a.T;
  s.t0 = (int)min((long long)seg * a.seg_len, (long long)len);
  s.t1 = (int)min((long long)s.t0 + a.seg_len, (long long)len);
  return s;
}
__device__ __forceinline__ const bf16* la_at(const LinAttnTok& x, const LaSpan& s, long long t) { return x.p + s.b * x.bs + t * x.ts + s.h * LA_D; }

__device__ __forceinline__ uint32_t la_pack(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *(uint32_t*)&v;
}
__device__ __forceinline__ float la_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float la_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
// The bf16 pair nearest to (x, y); x and y become what is left.
__device__ __forceinline__ uint32_t la_take(float& x, float& y) {
  const uint32_t h = la_pack(x, y);
  x -= la_lo(h);
  y -= la_hi(h);
  return h;
}

}  // namespace lp
