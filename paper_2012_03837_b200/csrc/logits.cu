// Operators that read a model's logits: log probabilities of given tokens with entropy and top alternatives, their
// gradient, and distillation from a teacher's top logits.
//
// x: a row, z = x / T, M = max x, S = sum exp((x - M) / T), W = sum exp((x - M) / T) (x - M)
//   log p_j = (x_j - M) / T - log S      lse = M / T + log S      entropy H = log S - W / (S T)
//   gradient of a logp_tok + b H + c lse:   dx_j = 1/T [ p_j (c - a - b H - b log p_j) + a 1[j = tok] ]
// Distillation, q_j the teacher's listed probabilities, q_r its rest, Q = sum q_j + q_r; R = sum over the tokens not listed:
//   KL = sum q_j (log q_j - log p_j) + q_r (log q_r - log (R / S))
//   dx_i = 1/T [ Q p_i - q_i ] where listed,   1/T e_i [ Q / S - q_r / R ] elsewhere, e_i = exp((x_i - M) / T)
// Differences to the maximum are formed before the temperature, so rows of the type's lowest value are rows like others.
// Everything is summed in fp32; what a row hands out is formed from its sums once.
#include <cfloat>

#include "common.cuh"
#include "launch.cuh"

namespace lp {
namespace {

constexpr int TOP_MAX = 128;                  // LP_TOP_MAX
constexpr float SMALLEST_REST = 0x1p-20f;

struct Row {
  float c, inv_t;                             // log2(e) / T, 1 / T
};
__device__ __forceinline__ float exp_of(float d, float c) { return exp2f(d * c); }

// A logit's place in the order: larger logits above, NaN below everything, equal ones by ascending index.
__device__ __forceinline__ unsigned long long order_key(float v, int j) {
  uint32_t u = __float_as_uint(v == 0.f ? 0.f : v);
  u = (u & 0x80000000u) ? ~u : u | 0x80000000u;
  if (v != v) u = 0;
  return ((unsigned long long)u << 32) | (uint32_t)~j;
}

template <typename T>
__device__ float row_max(const T* x, int n, float* red) {
  float m = -INFINITY;
  for (int j = threadIdx.x; j < n; j += blockDim.x) m = fmaxf(m, to_f(x[j]));
  return block_max(m, red);
}

template <typename T>
__global__ void __launch_bounds__(256) logprobs_kernel(const LogprobsArgs a, const Row p) {
  __shared__ float red[33];
  __shared__ unsigned long long best[8], last;
  const int r = blockIdx.x, n = a.in.vocab;
  const T* x = (const T*)a.in.x + (long long)r * a.in.ld;
  const float m = row_max(x, n, red);
  float s = 0.f, w = 0.f;
  for (int j = threadIdx.x; j < n; j += blockDim.x) {
    const float v = to_f(x[j]);
    if (v == -INFINITY) continue;
    const float d = v - m, e = exp_of(d, p.c);
    s += e;
    if (e != 0.f) w = fmaf(e, d, w);
  }
  s = block_sum(s, red);
  w = block_sum(w, red);
  const float logs = logf(s);
  auto logp = [&](float v) { return s == 0.f ? -INFINITY : fmaf(v - m, p.inv_t, -logs); };
  if (threadIdx.x == 0) {
    if (a.logp) {
      const int t = a.tokens[r];
      if (t >= n && a.in.out_of_range) atomicOr(a.in.out_of_range, 1);
      a.logp[r] = t >= 0 && t < n ? logp(to_f(x[t])) : 0.f;
    }
    if (a.entropy) a.entropy[r] = s == 0.f ? 0.f : logs - w / s * p.inv_t;
    if (a.lse) a.lse[r] = s == 0.f ? -INFINITY : fmaf(m, p.inv_t, logs);
  }
  unsigned long long bound = ~0ull;
  for (int i = 0; i < a.top_k; ++i) {
    unsigned long long b = 0;
    for (int j = threadIdx.x; j < n; j += blockDim.x) {
      const unsigned long long key = order_key(to_f(x[j]), j);
      if (key < bound && key > b) b = key;
    }
    for (int o = 16; o > 0; o >>= 1) {
      const unsigned long long y = __shfl_xor_sync(0xffffffffu, b, o);
      b = y > b ? y : b;
    }
    if ((threadIdx.x & 31) == 0) best[threadIdx.x >> 5] = b;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int k = 1; k < 8; ++k) b = best[k] > b ? best[k] : b;
      last = b;
      const int j = (int)~(uint32_t)b;
      a.top_ids[(long long)r * a.top_k + i] = j;
      a.top_logp[(long long)r * a.top_k + i] = logp(to_f(x[j]));
    }
    __syncthreads();
    bound = last;
  }
}

template <typename T>
__global__ void __launch_bounds__(256) logprobs_bwd_kernel(const LogprobsBwdArgs a, const Row p) {
  __shared__ float red[33];
  const int r = blockIdx.x, n = a.in.vocab;
  const T* x = (const T*)a.in.x + (long long)r * a.in.ld;
  T* dx = (T*)a.dx + (long long)r * a.ld_out;
  int t = -1;
  if (a.dlogp) {
    t = a.tokens[r];
    if (t >= n) {
      if (threadIdx.x == 0 && a.in.out_of_range) atomicOr(a.in.out_of_range, 1);
      t = -1;
    }
  }
  const float ga = t >= 0 ? a.dlogp[r] : 0.f, gb = a.dentropy ? a.dentropy[r] : 0.f, gc = a.dlse ? a.dlse[r] : 0.f;
  if (ga == 0.f && gb == 0.f && gc == 0.f) {
    for (int j = threadIdx.x; j < n; j += blockDim.x) dx[j] = from_f<T>(0.f);
    return;
  }
  const float m = row_max(x, n, red);
  float s = 0.f, w = 0.f;
  for (int j = threadIdx.x; j < n; j += blockDim.x) {
    const float v = to_f(x[j]);
    if (v == -INFINITY) continue;
    const float d = v - m, e = exp_of(d, p.c);
    s += e;
    if (e != 0.f) w = fmaf(e, d, w);
  }
  s = block_sum(s, red);
  w = block_sum(w, red);
  const float logs = logf(s), h = logs - w / s * p.inv_t;
  const float k0 = (gc - ga - gb * h) * p.inv_t, k1 = -gb * p.inv_t, inv_s = 1.f / s;
  for (int j = threadIdx.x; j < n; j += blockDim.x) {
    const float d = to_f(x[j]) - m, e = exp_of(d, p.c) * inv_s;
    float g = e == 0.f ? 0.f : e * fmaf(k1, fmaf(d, p.inv_t, -logs), k0);
    if (j == t) g += ga * p.inv_t;
    dx[j] = from_f<T>(s == 0.f ? 0.f : g);
  }
}

template <typename T>
__global__ void __launch_bounds__(256) distill_kernel(const DistillArgs a, const Row p) {
  __shared__ float red[33];
  __shared__ int id[TOP_MAX];
  __shared__ float q[TOP_MAX];
  const int r = blockIdx.x, n = a.in.vocab, k = a.k, tid = threadIdx.x;
  const T* x = (const T*)a.in.x + (long long)r * a.in.ld;
  T* dx = a.dx ? (T*)a.dx + (long long)r * a.ld_out : nullptr;
  float t = -INFINITY;
  int i = -1;
  if (tid < k) {
    i = a.ids[(long long)r * k + tid];
    t = a.teacher[(long long)r * k + tid];
    if (i >= n) {
      if (a.in.out_of_range) atomicOr(a.in.out_of_range, 1);
      i = -1;
    }
    if (i < 0) { i = -1; t = -INFINITY; }
    id[tid] = i;
  }
  const bool weight = __syncthreads_or(!(t == -INFINITY));
  const float dl = a.dloss ? a.dloss[r] : 1.f, g = dl * a.scale * p.inv_t;
  if (!weight || (!a.loss && dl == 0.f)) {
    if (tid == 0 && a.loss) a.loss[r] = 0.f;
    if (dx)
      for (int j = tid; j < n; j += blockDim.x) dx[j] = from_f<T>(0.f);
    return;
  }
  float qj, logq, qr = 0.f;
  if (a.rest) {
    qj = expf(t);
    logq = t;
    const float mass = block_sum(qj, red);
    qr = 1.f - mass > SMALLEST_REST ? 1.f - mass : 0.f;
  } else {
    const float mt = block_max(t, red);
    const float e = t == -INFINITY ? 0.f : expf((t - mt) * p.inv_t), st = block_sum(e, red);
    qj = e / st;
    logq = (t - mt) * p.inv_t - logf(st);
  }
  if (tid < k) q[tid] = qj;
  const float Q = block_sum(qj, red) + qr;      // its barriers make id and q visible
  bool first = i >= 0;                          // the first entry of its token
  for (int j = 0; j < tid && j < k; ++j) first = first && id[j] != i;
  auto listed = [&](int j) {
    for (int l = 0; l < k; ++l)
      if (id[l] == j) return true;
    return false;
  };
  // the tokens not listed against their own maximum, so that a small rest keeps its digits
  float mr = -INFINITY;
  for (int j = tid; j < n; j += blockDim.x)
    if (const float v = to_f(x[j]); v > mr && !listed(j)) mr = v;
  mr = block_max(mr, red);
  float R = 0.f;
  for (int j = tid; j < n; j += blockDim.x) {
    const float v = to_f(x[j]);
    if (v != -INFINITY && !listed(j)) R += exp_of(v - mr, p.c);
  }
  R = block_sum(R, red);
  const float xi = i >= 0 ? to_f(x[i]) : -INFINITY;
  const float m = fmaxf(mr, block_max(xi, red));
  const float ei = xi == -INFINITY ? 0.f : exp_of(xi - m, p.c);
  const float f = R == 0.f ? 0.f : exp_of(mr - m, p.c);
  const float S = block_sum(first ? ei : 0.f, red) + R * f, logs = logf(S);
  if (a.loss) {
    float l = qj > 0.f || qj != qj ? qj * (logq - (S == 0.f ? -INFINITY : (xi - m) * p.inv_t - logs)) : 0.f;
    l = block_sum(l, red);
    if (tid == 0) {
      if (qr > 0.f) l += qr * (logf(qr) - (R == 0.f ? -INFINITY : (mr - m) * p.inv_t + logf(R) - logs));
      a.loss[r] = a.scale * l;
    }
  }
  if (!dx) return;
  if (dl == 0.f) {
    for (int j = tid; j < n; j += blockDim.x) dx[j] = from_f<T>(0.f);
    return;
  }
  float qi = 0.f;
  if (first)
    for (int j = 0; j < k; ++j) qi += id[j] == i ? q[j] : 0.f;
  const float kappa = R == 0.f ? 0.f : (Q * f / S - (qr > 0.f ? qr / R : 0.f)) * g;
  for (int j = tid; j < n; j += blockDim.x) {
    const float v = to_f(x[j]);
    if (!listed(j)) dx[j] = from_f<T>(kappa == 0.f || v == -INFINITY ? (S != S ? S : 0.f) : kappa * exp_of(v - mr, p.c));
  }
  if (first) dx[i] = from_f<T>(S == 0.f ? 0.f : (Q * (ei / S) - qi) * g);
}

Row row_of(const LogitsIn& in) {
  return Row{(float)(1.4426950408889634 / (double)in.temperature), (float)(1.0 / (double)in.temperature)};
}

}  // namespace

cudaError_t launch_logprobs(const LogprobsArgs& a, bool is_bf16, cudaStream_t s) {
  const dim3 grid(a.in.rows);
  if (is_bf16) logprobs_kernel<bf16><<<grid, 256, 0, s>>>(a, row_of(a.in));
  else logprobs_kernel<float><<<grid, 256, 0, s>>>(a, row_of(a.in));
  return cudaPeekAtLastError();
}

cudaError_t launch_logprobs_bwd(const LogprobsBwdArgs& a, bool is_bf16, cudaStream_t s) {
  const dim3 grid(a.in.rows);
  if (is_bf16) logprobs_bwd_kernel<bf16><<<grid, 256, 0, s>>>(a, row_of(a.in));
  else logprobs_bwd_kernel<float><<<grid, 256, 0, s>>>(a, row_of(a.in));
  return cudaPeekAtLastError();
}

cudaError_t launch_distill(const DistillArgs& a, bool is_bf16, cudaStream_t s) {
  const dim3 grid(a.in.rows);
  if (is_bf16) distill_kernel<bf16><<<grid, 256, 0, s>>>(a, row_of(a.in));
  else distill_kernel<float><<<grid, 256, 0, s>>>(a, row_of(a.in));
  return cudaPeekAtLastError();
}

}  // namespace lp
