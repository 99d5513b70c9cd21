// Operators that read a model's logits: log probabilities of given tokens with entropy and top alternatives, their
// gradient, and distillation from a teacher's top logits.
//
// x: a row, c = log2(e) / T, y_j = x_j c - rho with rho = fl(c max x): the reference of all powers of two, the same for all
// terms, so that its rounding cancels.  S = sum 2^y_j, W = sum 2^y_j y_j:
//   log p_j = y_j ln 2 - log S      lse = rho ln 2 + log S      entropy H = log S - ln 2 W / S
//   gradient of a logp_tok + b H + g lse:
//     dx_j = 2^y_j (k0 + k1 y_j) + a/T 1[j = tok],  k0 = (g - a + b ln 2 W / S) / (T S),  k1 = -b ln 2 / (T S)
// Distillation: q_j the teacher's entries, q_r its rest, Q = sum q_j + q_r.  The tokens not listed are summed against their
// own maximum (rho_r; R = sum 2^(x_i c - rho_r)), so that a small rest keeps its digits; f = 2^(rho_r - rho):
//   KL = sum q_j (log q_j - log p_j) + q_r (log q_r - log p_r),   log p_r = (rho_r - rho) ln 2 + log R - log S
//   dx_i = 2^(x_i c - rho_r) kappa elsewhere, kappa = (Q f / S - q_r / R) / T;   dx_j = (Q p_j - q_j) / T where listed
// Sums are in fp32 in a fixed order.  Rows whose |rho| is above FAR (the type's lowest value in every place, infinities)
// take the differences before the factor, one element at a time.
//
// A row is read once: its piece of the row waits in shared memory (asynchronous copies of 16 bytes) for the second pass that
// a gradient or the top alternatives take.  Long rows, and rows too few for the device, are cut over a cluster of up to
// eight blocks, which exchange their sums through distributed shared memory.
#include <algorithm>
#include <cstddef>

#include <cooperative_groups.h>

#include "common.cuh"
#include "launch.cuh"

namespace lp {
namespace {

namespace cg = cooperative_groups;
typedef unsigned long long u64;

constexpr int TOP_MAX = 128;                  // LP_TOP_MAX
constexpr float SMALLEST_REST = 0x1p-20f;
constexpr float FAR = 1e23f;
constexpr float LN2 = 0.693147180559945309f;
constexpr int MAX_CLUSTER = 8, MAX_THREADS = 512, MAX_WARPS = MAX_THREADS / 32;
constexpr int CANDIDATES = 512;               // of the top alternatives

// ---------------------------------------------------------------------------------------------- two floats at a time
__device__ __forceinline__ u64 pack(float a, float b) {
  u64 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 unpack(u64 a) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a));
  return r;
}
__device__ __forceinline__ u64 fma2(u64 a, u64 b, u64 c) {
  u64 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ u64 add2(u64 a, u64 b) {
  u64 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ u64 mul2(u64 a, u64 b) {
  u64 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float ex2(float a) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(a));
  return r;
}
__device__ __forceinline__ u64 ex22(u64 a) {
  const float2 v = unpack(a);
  return pack(ex2(v.x), ex2(v.y));
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// ---------------------------------------------------------------------------------------------- vectors of 16 bytes
template <typename T> struct Vec;
template <> struct Vec<bf16> {
  static constexpr int N = 8;
  static constexpr uint32_t NEG_INF = 0xFF80FF80u;
  static __device__ __forceinline__ u64 pair(const uint4& v, int i) {
    const uint32_t w = (&v.x)[i];
    return pack(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
  static __device__ __forceinline__ __nv_bfloat162 b2(uint32_t w) { return *(__nv_bfloat162*)&w; }
  static __device__ __forceinline__ uint32_t u2(__nv_bfloat162 w) { return *(uint32_t*)&w; }
  // the largest element; a NaN only if there is nothing else
  static __device__ __forceinline__ float max1(const uint4& v) {
    const __nv_bfloat162 m = __hmax2(__hmax2(b2(v.x), b2(v.y)), __hmax2(b2(v.z), b2(v.w)));
    return __bfloat162float(__hmax(__low2bfloat16(m), __high2bfloat16(m)));
  }
  static __device__ __forceinline__ float max4(const uint4* v) {
    __nv_bfloat162 m = b2(v[0].x);
#pragma unroll
    for (int u = 0; u < 4; ++u) m = __hmax2(m, __hmax2(__hmax2(b2(v[u].x), b2(v[u].y)), __hmax2(b2(v[u].z), b2(v[u].w))));
    return __bfloat162float(__hmax(__low2bfloat16(m), __high2bfloat16(m)));
  }
  static __device__ __forceinline__ void clamp(uint4& v, float lo) {
    const __nv_bfloat162 l = __float2bfloat162_rn(lo);
#pragma unroll
    for (int i = 0; i < 4; ++i) (&v.x)[i] = u2(__hmax2_nan(b2((&v.x)[i]), l));
  }
  static __device__ __forceinline__ float get(const uint4& v, int i) {
    const uint32_t w = (&v.x)[i >> 1];
    return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
  }
  static __device__ __forceinline__ void set_pair(uint4& v, int i, u64 p) {
    const float2 f = unpack(p);
    (&v.x)[i] = u2(__floats2bfloat162_rn(f.x, f.y));
  }
};
template <> struct Vec<float> {
  static constexpr int N = 4;
  static constexpr uint32_t NEG_INF = 0xFF800000u;
  static __device__ __forceinline__ float at(const uint4& v, int i) { return __uint_as_float((&v.x)[i]); }
  static __device__ __forceinline__ u64 pair(const uint4& v, int i) { return pack(at(v, 2 * i), at(v, 2 * i + 1)); }
  static __device__ __forceinline__ float max1(const uint4& v) { return fmaxf(fmaxf(at(v, 0), at(v, 1)), fmaxf(at(v, 2), at(v, 3))); }
  static __device__ __forceinline__ float max4(const uint4* v) { return fmaxf(fmaxf(max1(v[0]), max1(v[1])), fmaxf(max1(v[2]), max1(v[3]))); }
  static __device__ __forceinline__ void clamp(uint4& v, float lo) {
#pragma unroll
    for (int i = 0; i < 4; ++i) (&v.x)[i] = __float_as_uint(max_nan(at(v, i), lo));
  }
  static __device__ __forceinline__ float get(const uint4& v, int i) { return at(v, i); }
  static __device__ __forceinline__ void set_pair(uint4& v, int i, u64 p) {
    const float2 f = unpack(p);
    (&v.x)[2 * i] = __float_as_uint(f.x);
    (&v.x)[2 * i + 1] = __float_as_uint(f.y);
  }
};

// ---------------------------------------------------------------------------------------------- a row's pieces
struct Geometry {
  float c, inv_t;                             // log2(e) / T, 1 / T
  float lo;                                   // logits below it have probability 0 in rows that are not far
  int cluster;                                // blocks per row
};

// The block's piece of its row: vectors first .. first + count of the row's lattice of aligned 16 bytes, of which vector v
// holds elements v N - shift .. v N - shift + N - 1.
template <typename T>
struct Piece {
  const T* x;                                 // the row
  int n, shift, first, count, per;
  uint4* buf;                                 // its vectors in shared memory, -infinity outside the row
  __device__ __forceinline__ Piece(const T* row, int n_, int rank, int cluster, uint4* buf_) : x(row), n(n_), buf(buf_) {
    shift = (int)(((uintptr_t)row & 15) / sizeof(T));
    const int all = (n + shift + Vec<T>::N - 1) / Vec<T>::N;
    per = (all + cluster - 1) / cluster;
    first = min(all, rank * per);
    count = min(all - first, per);
  }
  __device__ __forceinline__ int element(int v) const { return (first + v) * Vec<T>::N - shift; }     // the first of vector v
  __device__ __forceinline__ bool inside(int j) const { return j >= 0 && j + Vec<T>::N <= n; }
  // Every thread fetches the vectors that it works on: v = threadIdx.x, + blockDim.x, ...
  __device__ __forceinline__ void fetch() const {
    for (int v = threadIdx.x; v < count; v += blockDim.x) {
      const int j = element(v);
      if (inside(j)) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(buf + v)), "l"(x + j) : "memory");
      } else {
        T* e = (T*)(buf + v);
#pragma unroll
        for (int i = 0; i < Vec<T>::N; ++i) e[i] = j + i >= 0 && j + i < n ? x[j + i] : from_f<T>(-INFINITY);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  __device__ __forceinline__ static void arrived() { asm volatile("cp.async.wait_all;" ::: "memory"); }
  // The vector's place in another matrix of rows, if it is aligned there.
  __device__ __forceinline__ void store(T* dst, int v, const uint4& r) const {
    const int j = element(v);
    if (inside(j) && ((uintptr_t)(dst + j) & 15) == 0) {
      *(uint4*)(dst + j) = r;
    } else {
      const T* e = (const T*)&r;
#pragma unroll
      for (int i = 0; i < Vec<T>::N; ++i)
        if (j + i >= 0 && j + i < n) dst[j + i] = e[i];
    }
  }
  __device__ __forceinline__ void zeros(T* dst) const {
    for (int v = threadIdx.x; v < count; v += blockDim.x) store(dst, v, make_uint4(0, 0, 0, 0));
  }
};

// ---------------------------------------------------------------------------------------------- sums of a row
struct Sums { float m, s, w; };               // max x, sum 2^y, sum 2^y y against rho_of(m)

// The reference that a maximum gives; none below lo (masked tokens, of -infinity or the type's lowest value: their sum is
// 0, unless the row has nothing else and is far).
__device__ __forceinline__ float rho_of(float m, const Geometry& g) { return m < g.lo ? 0.f : __fmul_rn(m, g.c); }

// Moves a sum from its reference to that of a larger maximum.
template <bool W>
__device__ __forceinline__ void move(Sums& a, float m, const Geometry& g) {
  const float d = rho_of(a.m, g) - rho_of(m, g), f = a.m < g.lo ? 0.f : ex2(d);
  if (W) a.w = f * fmaf(a.s, fmaxf(d, -1e30f), a.w);
  a.s *= f;
  a.m = m;
}

template <typename T, bool W>
__device__ __forceinline__ Sums sweep(const Piece<T>& p, const Geometry& g) {
  constexpr int P = Vec<T>::N / 2;
  const u64 c2 = pack(g.c, g.c);
  u64 s0 = 0, s1 = 0, w0 = 0, w1 = 0, nrho = 0;
  float m = -INFINITY;
  const int nt = blockDim.x;
  for (int v = threadIdx.x; v < p.count; v += 4 * nt) {
    uint4 a[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      a[u] = v + u * nt < p.count ? p.buf[v + u * nt] : make_uint4(Vec<T>::NEG_INF, Vec<T>::NEG_INF, Vec<T>::NEG_INF, Vec<T>::NEG_INF);
    const float bm = Vec<T>::max4(a);
    if (bm > m) {
      const float d = rho_of(m, g) - rho_of(bm, g), f = ex2(d);
      if (m >= g.lo) {
        const u64 f2 = pack(f, f), d2 = pack(d, d);
        if (W) { w0 = mul2(f2, fma2(s0, d2, w0)); w1 = mul2(f2, fma2(s1, d2, w1)); }
        s0 = mul2(s0, f2);
        s1 = mul2(s1, f2);
      }
      m = bm;
      const float r = -rho_of(m, g);
      nrho = pack(r, r);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (W) Vec<T>::clamp(a[u], g.lo);
#pragma unroll
      for (int i = 0; i < P; i += 2) {
        const u64 y0 = fma2(Vec<T>::pair(a[u], i), c2, nrho), y1 = fma2(Vec<T>::pair(a[u], i + 1), c2, nrho);
        const u64 e0 = ex22(y0), e1 = ex22(y1);
        s0 = add2(s0, e0);
        s1 = add2(s1, e1);
        if (W) { w0 = fma2(e0, y0, w0); w1 = fma2(e1, y1, w1); }
      }
    }
  }
  const float2 s = unpack(add2(s0, s1)), w = unpack(add2(w0, w1));
  return Sums{m, s.x + s.y, w.x + w.y};
}

// The same against the row's maximum, for far rows.
template <typename T, bool W>
__device__ __noinline__ Sums sweep_far(const Piece<T>& p, const Geometry& g, float m) {
  Sums a{m, 0.f, 0.f};
  for (int v = threadIdx.x; v < p.count; v += blockDim.x)
    for (int i = 0; i < Vec<T>::N; ++i) {
      const float x = Vec<T>::get(p.buf[v], i);
      if (x == -INFINITY) continue;
      const float y = (x - m) * g.c, e = ex2(y);
      a.s += e;
      if (W && e != 0.f) a.w = fmaf(e, y, a.w);
    }
  return a;
}

struct Exchange {                             // what the warps of a row's blocks tell one another
  float4 part[2][MAX_CLUSTER * MAX_WARPS];
};

template <bool CL>
__device__ __forceinline__ void sync_row() {
  if (CL) {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  } else {
    __syncthreads();
  }
}

// The row's sums, the same bits in every thread of its blocks.  FARROW: all parts have the row's maximum as their reference.
template <bool W, bool CL, bool FARROW>
__device__ __forceinline__ Sums join(Sums a, Exchange& ex, const Geometry& g, int rank) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  if (!FARROW) move<W>(a, warp_max(a.m), g);
  a.s = warp_sum(a.s);
  if (W) a.w = warp_sum(a.w);
  float4* part = ex.part[FARROW ? 1 : 0];
  const float4 mine = make_float4(a.m, a.s, a.w, 0.f);
  if (CL) {
    if (lane < g.cluster) cg::this_cluster().map_shared_rank(part, lane)[rank * warps + warp] = mine;
  } else if (lane == 0) {
    part[warp] = mine;
  }
  sync_row<CL>();
  const int parts = CL ? g.cluster * warps : warps;
  float m = a.m;
  if (!FARROW) {
    m = -INFINITY;
    for (int i = lane; i < parts; i += 32) m = fmaxf(m, part[i].x);
    m = warp_max(m);
  }
  Sums t{m, 0.f, 0.f};
  for (int i = lane; i < parts; i += 32) {
    Sums b{part[i].x, part[i].y, part[i].z};
    if (!FARROW) move<W>(b, m, g);
    t.s += b.s;
    if (W) t.w += b.w;
  }
  t.s = warp_sum(t.s);
  if (W) t.w = warp_sum(t.w);
  return t;
}

// A row's reference.
struct Ref {
  float m, rho, c, inv_t;
  bool far;
  __device__ __forceinline__ Ref(float m_, const Geometry& g) : m(m_), rho(rho_of(m_, g)), c(g.c), inv_t(g.inv_t),
                                                              far(m_ != -INFINITY && !(fabsf(m_) * g.c <= FAR)) {}
  __device__ __forceinline__ bool apart(float x) const { return far || fabsf(x) * c > FAR; }
  __device__ __forceinline__ float y(float x) const { return far ? (x - m) * c : fmaf(x, c, -rho); }
  // (x - m) / T, of a masked token's lowest value too
  __device__ __forceinline__ float nat(float x) const { return apart(x) ? (x - m) * inv_t : fmaf(x, c, -rho) * LN2; }
};

template <typename T, bool W, bool CL>
__device__ __forceinline__ Sums row_sums(const Piece<T>& p, const Geometry& g, Exchange& ex, int rank, float& thread_max) {
  const Sums own = sweep<T, W>(p, g);
  thread_max = own.m;
  Sums a = join<W, CL, false>(own, ex, g, rank);
  if (Ref(a.m, g).far) a = join<W, CL, true>(sweep_far<T, W>(p, g, a.m), ex, g, rank);
  return a;
}

extern __shared__ uint4 dynamic[];

template <bool CL>
__device__ __forceinline__ void cluster_start() {        // every block of the cluster runs: its memory may be written
  if (CL) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
template <bool CL>
__device__ __forceinline__ void cluster_started() {
  if (CL) {
    __syncwarp();
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
  }
}

// A token id, or -1 where there is none.
__device__ __forceinline__ int token_of(const int* tokens, long long i, int n, int* out_of_range, bool report) {
  const int t = tokens[i];
  if (t < n) return t < 0 ? -1 : t;
  if (report && out_of_range) atomicOr(out_of_range, 1);
  return -1;
}

// ---------------------------------------------------------------------------------------------- top alternatives
// A logit's place in the order: larger logits above, NaN below everything; with the id, equal ones by ascending id.
__device__ __forceinline__ uint32_t order_of(float v) {
  uint32_t u = __float_as_uint(v + 0.f);                 // -0 becomes 0
  u = (u & 0x80000000u) ? ~u : u | 0x80000000u;
  return v != v ? 0u : u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
  return o == 0 ? __uint_as_float(0x7fc00000u) : __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ u64 key_of(uint32_t order, int j) { return ((u64)order << 32) | (uint32_t)~j; }

struct TopSpace {
  u64 list[CANDIDATES];
  int count, base, warp_total[MAX_WARPS];
  u64 sorted[MAX_CLUSTER][TOP_MAX];           // of the row's first block: what each block found
};

// Puts the keys of the block's k largest logits (all of them, if there are fewer) into ts.list and returns how many are
// there: at least min(k, logits), at most CANDIDATES.
//   bound: the k-th largest of the threads' maxima, or a little less: at least k logits reach it, and of logits in no
//   particular order hardly more (k = 64 of 256 threads: 74).  Halving an interval of the order, one count per step.
//   Where more than CANDIDATES reach it (many equal logits, or large ones side by side), the k-th largest value itself is
//   found the same way among all logits, and the equal ones are taken in the order of their ids.
template <typename T>
__device__ int top_candidates(const Piece<T>& p, int k, float thread_max, TopSpace& ts) {
  const int tid = threadIdx.x, nt = blockDim.x;
  // bounds of the thread's largest logit: what counts as -infinity may be a NaN, which stands below
  const uint32_t most = tid < p.count ? order_of(thread_max) : 0u, least = thread_max == -INFINITY ? 0u : most;
  if (tid == 0) ts.count = 0;
  uint32_t lo = 0, hi = 0xffffffffu;                     // at least k reach lo (0: all), fewer than k reach hi
  while (hi - lo > 1) {
    const uint32_t mid = lo + (hi - lo) / 2;
    const int n = __syncthreads_count(least >= mid);
    if (n >= k) {
      lo = mid;
      if (n <= k + k / 4) break;
    } else {
      hi = mid;
    }
  }
  __syncthreads();
  auto add = [&](uint32_t o, int j) {
    const int at = atomicAdd(&ts.count, 1);
    if (at < CANDIDATES) ts.list[at] = key_of(o, j);
  };
  if (most >= lo) {
    for (int v = tid; v < p.count; v += nt) {
      const uint4 a = p.buf[v];
      if (order_of(Vec<T>::max1(a)) < lo) continue;
      const int j = p.element(v);
      for (int i = 0; i < Vec<T>::N; ++i) {
        const uint32_t o = order_of(Vec<T>::get(a, i));
        if (o >= lo && j + i >= 0 && j + i < p.n) add(o, j + i);
      }
    }
  }
  __syncthreads();
  const int found = ts.count;
  if (found <= CANDIDATES) return found;

  // exactly: the largest value that at least k logits reach
  auto reaching = [&](uint32_t bound) {
    int n = 0;
    if (most >= bound)
      for (int v = tid; v < p.count; v += nt) {
        const int j = p.element(v);
        for (int i = 0; i < Vec<T>::N; ++i) n += j + i >= 0 && j + i < p.n && order_of(Vec<T>::get(p.buf[v], i)) >= bound;
      }
    n = __reduce_add_sync(0xffffffffu, n);
    __syncthreads();
    if (tid == 0) ts.base = 0;
    __syncthreads();
    if ((tid & 31) == 0) atomicAdd(&ts.base, n);
    __syncthreads();
    return ts.base;
  };
  hi = 0xffffffffu;
  uint32_t probe = lo + 1;                               // often lo itself is the value
  int above = 0;
  while (hi - lo > 1) {
    const int n = reaching(probe);
    if (n >= k) lo = probe;
    else { hi = probe; above = n; }
    probe = lo + (hi - lo) / 2;
  }
  __syncthreads();
  if (tid == 0) { ts.count = 0; ts.base = 0; }
  __syncthreads();
  if (most > lo)
    for (int v = tid; v < p.count; v += nt) {
      const int j = p.element(v);
      for (int i = 0; i < Vec<T>::N; ++i) {
        const uint32_t o = order_of(Vec<T>::get(p.buf[v], i));
        if (o > lo && j + i >= 0 && j + i < p.n) add(o, j + i);
      }
    }
  int taken = above;                                     // ids ascend with v, and within a step with the thread
  for (int v0 = 0; v0 < p.count && taken < k; v0 += nt) {
    const int v = v0 + tid;
    unsigned same = 0;
    int j = 0;
    if (v < p.count) {
      j = p.element(v);
      for (int i = 0; i < Vec<T>::N; ++i)
        if (j + i >= 0 && j + i < p.n && order_of(Vec<T>::get(p.buf[v], i)) == lo) same |= 1u << i;
    }
    int before = __popc(same);
    const int own = before;
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, before, o);
      if ((tid & 31) >= o) before += y;
    }
    __syncthreads();
    if ((tid & 31) == 31) ts.warp_total[tid >> 5] = before;
    __syncthreads();
    int total = 0;
    before -= own;
    for (int w = 0; w < nt >> 5; ++w) {
      if (w < tid >> 5) before += ts.warp_total[w];
      total += ts.warp_total[w];
    }
    for (int i = 0, at = taken + before; same && at < k; ++i)
      if (same >> i & 1) { add(lo, j + i); ++at; same &= ~(1u << i); }
    taken += total;
  }
  __syncthreads();
  return min(ts.count, CANDIDATES);
}

// ---------------------------------------------------------------------------------------------- kernels
template <typename T, bool W, bool CL>
__global__ void __launch_bounds__(MAX_THREADS) logprobs_kernel(const __grid_constant__ LogprobsArgs a, const __grid_constant__ Geometry g) {
  __shared__ Exchange ex;
  cudaGridDependencySynchronize();
  cluster_start<CL>();
  const int rank = CL ? (int)(blockIdx.x % g.cluster) : 0, tid = threadIdx.x, nt = blockDim.x;
  const long long r = CL ? blockIdx.x / g.cluster : blockIdx.x;
  const T* x = (const T*)a.in.x + r * a.in.ld;
  const Piece<T> p(x, a.in.vocab, rank, CL ? g.cluster : 1, dynamic);
  p.fetch();
  const bool speaks = rank == 0 && tid == 0;             // for the row
  int t = -1;
  float xt = 0.f;
  if (speaks && a.tokens) {
    t = token_of(a.tokens, r, p.n, a.in.out_of_range, true);
    if (t >= 0) xt = to_f(x[t]);
  }
  p.arrived();
  cluster_started<CL>();
  float thread_max;
  const Sums s = row_sums<T, W, CL>(p, g, ex, rank, thread_max);
  const Ref ref(s.m, g);
  const float logs = logf(s.s);
  auto logp = [&](float v) { return s.s == 0.f ? -INFINITY : ref.nat(v) - logs; };
  if (speaks) {
    if (a.logp) a.logp[r] = t >= 0 ? logp(xt) : 0.f;
    if (W && a.entropy) a.entropy[r] = s.s == 0.f ? 0.f : fmaf(-LN2, s.w / s.s, logs);
    if (a.lse) a.lse[r] = s.s == 0.f ? -INFINITY : ref.far ? fmaf(s.m, g.inv_t, logs) : fmaf(ref.rho, LN2, logs);
  }
  if (a.top_k == 0) return;
  const int k = a.top_k;
  TopSpace& ts = *(TopSpace*)(dynamic + p.per);
  auto put = [&](int at, u64 key) {
    a.top_ids[r * k + at] = (int)~(uint32_t)key;
    a.top_logp[r * k + at] = logp(value_of((uint32_t)(key >> 32)));
  };
  const int found = top_candidates(p, k, thread_max, ts);
  u64* sorted = CL ? cg::this_cluster().map_shared_rank(&ts.sorted[rank][0], 0) : nullptr;
  for (int i = tid; i < found; i += nt) {                // a candidate's place is the number of larger ones
    const u64 key = ts.list[i];
    int at = 0;
    for (int j = 0; j < found; ++j) at += ts.list[j] > key;
    if (at >= k) continue;
    if (CL) sorted[at] = key;
    else put(at, key);
  }
  if constexpr (CL) {
    for (int i = found + tid; i < k; i += nt) sorted[i] = 0;   // fewer logits than k in this piece
    sync_row<true>();
    if (rank != 0) return;
    for (int i = tid; i < g.cluster * k; i += nt) {        // the place among all: the larger ones of every block's list
      const int q = i / k;
      const u64 key = ts.sorted[q][i - q * k];
      if (key == 0) continue;
      int at = i - q * k;
      for (int o = 0; o < g.cluster; ++o) {
        if (o == q) continue;
        int lo = 0, hi = k;
        while (lo < hi) {
          const int mid = (lo + hi) / 2;
          if (ts.sorted[o][mid] > key) lo = mid + 1;
          else hi = mid;
        }
        at += lo;
      }
      if (at < k) put(at, key);
    }
  }
}

// The row's second pass: dst = 2^y (k0 + k1 y), a token's own term added.
template <typename T, bool W>
__device__ __forceinline__ void gradient(const Piece<T>& p, const Geometry& g, const Ref& ref, float k0, float k1, int t, float at_t, T* dst) {
  constexpr int N = Vec<T>::N;
  if (ref.far) {
    for (int v = threadIdx.x; v < p.count; v += blockDim.x) {
      uint4 o;
      const int j = p.element(v);
      float d[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float y = ref.y(Vec<T>::get(p.buf[v], i)), e = ex2(y);
        d[i] = e == 0.f && k0 == k0 ? 0.f : W ? e * fmaf(k1, y, k0) : e * k0;
        if (j + i == t) d[i] += at_t;
      }
#pragma unroll
      for (int i = 0; i < N / 2; ++i) Vec<T>::set_pair(o, i, pack(d[2 * i], d[2 * i + 1]));
      p.store(dst, v, o);
    }
    return;
  }
  const u64 c2 = pack(g.c, g.c), nrho = pack(-ref.rho, -ref.rho), k02 = pack(k0, k0), k12 = pack(k1, k1);
#pragma unroll 2
  for (int v = threadIdx.x; v < p.count; v += blockDim.x) {
    uint4 a = p.buf[v], o;
    if (W) Vec<T>::clamp(a, g.lo);
    u64 d[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const u64 y = fma2(Vec<T>::pair(a, i), c2, nrho), e = ex22(y);
      d[i] = mul2(e, W ? fma2(k12, y, k02) : k02);
    }
    const unsigned off = (unsigned)(t - p.element(v));
    if (t >= 0 && off < N) {
#pragma unroll
      for (int i = 0; i < N / 2; ++i)
        if (off >> 1 == i) d[i] = add2(d[i], off & 1 ? pack(0.f, at_t) : pack(at_t, 0.f));
    }
#pragma unroll
    for (int i = 0; i < N / 2; ++i) Vec<T>::set_pair(o, i, d[i]);
    p.store(dst, v, o);
  }
}

template <typename T, bool W, bool CL>
__global__ void __launch_bounds__(MAX_THREADS) logprobs_bwd_kernel(const __grid_constant__ LogprobsBwdArgs a, const __grid_constant__ Geometry g) {
  __shared__ Exchange ex;
  cudaGridDependencySynchronize();
  cluster_start<CL>();
  const int rank = CL ? (int)(blockIdx.x % g.cluster) : 0;
  const long long r = CL ? blockIdx.x / g.cluster : blockIdx.x;
  const Piece<T> p((const T*)a.in.x + r * a.in.ld, a.in.vocab, rank, CL ? g.cluster : 1, dynamic);
  T* dx = (T*)a.dx + r * a.ld_out;
  const int t = a.dlogp ? token_of(a.tokens, r, p.n, a.in.out_of_range, rank == 0 && threadIdx.x == 0) : -1;
  const float ga = t >= 0 ? a.dlogp[r] : 0.f, gb = W ? a.dentropy[r] : 0.f, gl = a.dlse ? a.dlse[r] : 0.f;
  if (ga == 0.f && gb == 0.f && gl == 0.f) {
    p.zeros(dx);
    cluster_started<CL>();
    return;
  }
  p.fetch();
  p.arrived();
  cluster_started<CL>();
  float thread_max;
  const Sums s = row_sums<T, W, CL>(p, g, ex, rank, thread_max);
  if (s.s == 0.f) {                                      // no token
    p.zeros(dx);
    return;
  }
  const Ref ref(s.m, g);
  const float k = g.inv_t / s.s;
  gradient<T, W>(p, g, ref, W ? (gl - ga + gb * (LN2 * (s.w / s.s))) * k : (gl - ga) * k, -gb * LN2 * k, t, ga * g.inv_t, dx);
}

__device__ __forceinline__ void sync_teacher() { asm volatile("bar.sync 1, 128;" ::: "memory"); }   // the first four warps

template <typename T, bool CL>
__global__ void __launch_bounds__(MAX_THREADS) distill_kernel(const __grid_constant__ DistillArgs a, const __grid_constant__ Geometry g) {
  __shared__ Exchange ex;
  __shared__ __align__(16) int id[TOP_MAX];
  __shared__ float weight[TOP_MAX];
  __shared__ float red[4][4];
  __shared__ double red_mass[4];
  __shared__ int any_weight;
  cudaGridDependencySynchronize();
  cluster_start<CL>();
  const int rank = CL ? (int)(blockIdx.x % g.cluster) : 0, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, k = a.k;
  const long long r = CL ? blockIdx.x / g.cluster : blockIdx.x;
  const T* x = (const T*)a.in.x + r * a.in.ld;
  const Piece<T> p(x, a.in.vocab, rank, CL ? g.cluster : 1, dynamic);
  T* dx = a.dx ? (T*)a.dx + r * a.ld_out : nullptr;
  p.fetch();
  const float dl = a.dloss ? a.dloss[r] : 1.f;

  // The teacher's row and what the student gives its tokens, an entry per thread of four warps, while the logits arrive.
  float q = 0.f, lq = 0.f, xi = -INFINITY;
  int i = -1, twins = 0;
  bool first = false;
  if (warp < 4) {
    float t = -INFINITY;
    if (tid < k) {
      i = token_of(a.ids, r * k + tid, p.n, a.in.out_of_range, rank == 0);
      if (i >= 0) { t = a.teacher[r * k + tid]; xi = to_f(x[i]); }
    }
    id[tid] = i;
    const float wt = warp_max(t), wx = warp_max(xi);
    const bool some = __any_sync(0xffffffffu, !(t == -INFINITY));
    if (lane == 0) { red[warp][0] = wt; red[warp][1] = wx; red[warp][2] = some ? 1.f : 0.f; }
    sync_teacher();
    float mt = -INFINITY, ml = -INFINITY, has = 0.f;
    for (int w = 0; w < 4; ++w) {
      mt = fmaxf(mt, red[w][0]);
      ml = fmaxf(ml, red[w][1]);
      has += red[w][2];
    }
    const double e = t == -INFINITY ? 0.0 : a.rest ? exp((double)t) : (double)expf((t - mt) * g.inv_t);
    first = i >= 0;
    for (int j = 0; j < k; j += 4) {
      const int4 o = *(const int4*)&id[j];
      const int same = (o.x == i) + (o.y == i) + (o.z == i) + (o.w == i);
      twins += same;                                     // entries of the same token; the first one stands for it
      if (same && (o.x == i ? j : o.y == i ? j + 1 : o.z == i ? j + 2 : j + 3) < tid) first = false;
    }
    const Ref rl(ml, g);
    const float el = first && xi != -INFINITY ? ex2(rl.y(xi)) : 0.f;
    double mass = e;
    for (int o = 16; o > 0; o >>= 1) mass += __shfl_xor_sync(0xffffffffu, mass, o);
    const float sl = warp_sum(el);
    sync_teacher();                                      // red is read
    if (lane == 0) { red_mass[warp] = mass; red[warp][3] = sl; red[warp][1] = ml; }
    if (tid == 0) any_weight = has != 0.f;
    sync_teacher();
    mass = red_mass[0] + red_mass[1] + red_mass[2] + red_mass[3];
    q = a.rest ? (float)e : (float)(e / mass);
    lq = a.rest ? t : (t - mt) * g.inv_t - logf((float)mass);
    weight[tid] = q;
  }
  p.arrived();
  cluster_started<CL>();
  __syncthreads();
  if (!any_weight) {
    if (rank == 0 && tid == 0 && a.loss) a.loss[r] = 0.f;
    if (dx) p.zeros(dx);
    return;
  }
  const int spot = i + p.shift - p.first * Vec<T>::N;    // the token's place in the piece, if it is there
  const bool here = i >= 0 && spot >= 0 && spot < p.count * Vec<T>::N;
  if (here) ((T*)p.buf)[spot] = from_f<T>(-INFINITY);    // what stays are the tokens not listed
  __syncthreads();
  float unused;
  const Sums rest = row_sums<T, false, CL>(p, g, ex, rank, unused);
  const double mass = red_mass[0] + red_mass[1] + red_mass[2] + red_mass[3];
  const float qr = a.rest && 1.0 - mass > SMALLEST_REST ? (float)(1.0 - mass) : 0.f;
  const float Q = a.rest ? (float)(qr > 0.f ? 1.0 : mass) : (float)(mass / mass);
  const float ml = red[0][1], R = rest.s, m = fmaxf(rest.m, ml);
  const Ref ref(m, g), rr(rest.m, g), rl(ml, g);
  const bool far = ref.far || rr.far;
  auto factor = [&](const Ref& o) { return o.m == -INFINITY ? 0.f : ex2(ref.far ? (o.m - m) * g.c : o.rho - ref.rho); };
  const float f = factor(rr), S = R * f + (red[0][3] + red[1][3] + red[2][3] + red[3][3]) * factor(rl), logs = logf(S);
  if (a.loss && rank == 0 && warp < 4) {
    float l = i >= 0 && !(q == 0.f) ? q * (lq - (S == 0.f ? -INFINITY : ref.nat(xi) - logs)) : 0.f;
    l = warp_sum(l);
    if (lane == 0) red[warp][2] = l;
    sync_teacher();
    if (tid == 0) {
      l = red[0][2] + red[1][2] + red[2][2] + red[3][2];
      if (qr > 0.f) l += qr * (logf(qr) - (R == 0.f ? -INFINITY : (far ? (rest.m - m) * g.inv_t : (rr.rho - ref.rho) * LN2) + logf(R) - logs));
      a.loss[r] = a.scale * l;
    }
  }
  if (!dx) return;
  if (dl == 0.f) {
    p.zeros(dx);
    return;
  }
  const float w = dl * a.scale * g.inv_t;
  const float kappa = S != S ? S : R == 0.f ? 0.f : (Q * f / S - (qr > 0.f ? qr / R : 0.f)) * w;
  gradient<T, false>(p, g, rr, kappa, 0.f, -1, 0.f, dx);
  __syncthreads();
  if (first && here) {
    float qi = q;
    if (twins > 1) {
      qi = 0.f;
      for (int j = 0; j < k; ++j) qi += id[j] == i ? weight[j] : 0.f;
    }
    const float pi = (xi == -INFINITY ? 0.f : ex2(ref.y(xi))) / S;
    dx[i] = from_f<T>(S == 0.f ? 0.f : (Q * pi - qi) * w);
  }
}

// ---------------------------------------------------------------------------------------------- launches
constexpr int PIECE = 4160;                   // vectors of a block's piece that let three blocks stay on an SM

struct Plan {
  Geometry g;
  dim3 grid;
  int threads, per;                           // vectors of the longest piece
};
Plan plan_rows(const LogitsIn& in, int elem_bytes, int min_threads) {
  Plan p{};
  const int N = 16 / elem_bytes, all = (in.vocab + 2 * N - 2) / N;      // a row may begin inside its first vector
  int c = std::min(MAX_CLUSTER, (all + PIECE - 1) / PIECE);
  while (2 * c <= MAX_CLUSTER && (long long)in.rows * c < 2 * 148 && all / (2 * c) >= 256) c *= 2;
  p.per = (all + c - 1) / c;
  p.threads = p.per > PIECE ? 512 : std::max(min_threads, std::min(256, (p.per + 31) / 32 * 32));
  p.grid = dim3((unsigned)((long long)in.rows * c));
  const double cc = 1.4426950408889634 / (double)in.temperature;
  p.g = Geometry{(float)cc, (float)(1.0 / (double)in.temperature), (float)(-1e30 * std::min(1.0, 1.0 / cc)), c};
  return p;
}

template <typename... KArgs, typename A>
cudaError_t run(void (*kernel)(KArgs...), SmemLimit& limit, const Plan& p, size_t extra, cudaStream_t s, const A& a) {
  const cudaError_t e = limit.raise((const void*)kernel, 160 * 1024);
  if (e != cudaSuccess) return e;
  return launch_cluster_after(kernel, p.g.cluster, p.grid, p.threads, (size_t)p.per * 16 + extra, s, a, p.g);
}

template <typename T, bool W, bool CL>
cudaError_t run_logprobs(const LogprobsArgs& a, const Plan& p, cudaStream_t s) {
  static SmemLimit limit;
  return run(logprobs_kernel<T, W, CL>, limit, p, a.top_k == 0 ? 0 : CL ? sizeof(TopSpace) : offsetof(TopSpace, sorted), s, a);
}
template <typename T, bool W, bool CL>
cudaError_t run_bwd(const LogprobsBwdArgs& a, const Plan& p, cudaStream_t s) {
  static SmemLimit limit;
  return run(logprobs_bwd_kernel<T, W, CL>, limit, p, 0, s, a);
}
template <typename T, bool CL>
cudaError_t run_distill(const DistillArgs& a, const Plan& p, cudaStream_t s) {
  static SmemLimit limit;
  return run(distill_kernel<T, CL>, limit, p, 0, s, a);
}

}  // namespace

cudaError_t launch_logprobs(const LogprobsArgs& a, bool is_bf16, cudaStream_t s) {
  const Plan p = plan_rows(a.in, is_bf16 ? 2 : 4, 64);
  const bool w = a.entropy != nullptr, cl = p.g.cluster > 1;
  if (is_bf16) return w ? (cl ? run_logprobs<bf16, true, true>(a, p, s) : run_logprobs<bf16, true, false>(a, p, s))
                        : (cl ? run_logprobs<bf16, false, true>(a, p, s) : run_logprobs<bf16, false, false>(a, p, s));
  return w ? (cl ? run_logprobs<float, true, true>(a, p, s) : run_logprobs<float, true, false>(a, p, s))
           : (cl ? run_logprobs<float, false, true>(a, p, s) : run_logprobs<float, false, false>(a, p, s));
}

cudaError_t launch_logprobs_bwd(const LogprobsBwdArgs& a, bool is_bf16, cudaStream_t s) {
  const Plan p = plan_rows(a.in, is_bf16 ? 2 : 4, 64);
  const bool w = a.dentropy != nullptr, cl = p.g.cluster > 1;
  if (is_bf16) return w ? (cl ? run_bwd<bf16, true, true>(a, p, s) : run_bwd<bf16, true, false>(a, p, s))
                        : (cl ? run_bwd<bf16, false, true>(a, p, s) : run_bwd<bf16, false, false>(a, p, s));
  return w ? (cl ? run_bwd<float, true, true>(a, p, s) : run_bwd<float, true, false>(a, p, s))
           : (cl ? run_bwd<float, false, true>(a, p, s) : run_bwd<float, false, false>(a, p, s));
}

cudaError_t launch_distill(const DistillArgs& a, bool is_bf16, cudaStream_t s) {
  const Plan p = plan_rows(a.in, is_bf16 ? 2 : 4, TOP_MAX);
  if (is_bf16) return p.g.cluster > 1 ? run_distill<bf16, true>(a, p, s) : run_distill<bf16, false>(a, p, s);
  return p.g.cluster > 1 ? run_distill<float, true>(a, p, s) : run_distill<float, false>(a, p, s);
}

}  // namespace lp
