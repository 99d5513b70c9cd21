// Operators that read a model's logits: log probabilities of given tokens with entropy and top alternatives, their
// gradient, and distillation from a teacher's top logits.
//
// x: a row, c = log2(e) / T, y_j = x_j c - rho with rho = fl(c max x): the reference of all powers of two, the same for all
// terms, so that its rounding cancels; it is at most 2 while |rho| <= FAR, so the powers stay well within 32 bits.
// S = sum 2^y_j, W = sum 2^y_j y_j:
//   log p_j = y_j ln 2 - log S      lse = rho ln 2 + log S      entropy H = log S - ln 2 W / S
//   gradient of a logp_tok + b H + g lse:
//     dx_j = 2^y_j (k0 + k1 y_j) + a/T 1[j = tok],  k0 = (g - a + b ln 2 W / S) / (T S),  k1 = -b ln 2 / (T S)
// Distillation: q_j the teacher's entries, q_r its rest, Q = sum q_j + q_r.  The tokens not listed are summed against their
// own maximum (rho_r; R = sum 2^(x_i c - rho_r)), so that a small rest keeps its digits; f = 2^(rho_r - rho):
//   KL = sum q_j (log q_j - log p_j) + q_r (log q_r - log p_r),   log p_r = (rho_r - rho) ln 2 + log R - log S
//   dx_i = 2^(x_i c - rho_r) kappa elsewhere, kappa = (Q f / S - q_r / R) / T;   dx_j = (Q p_j - q_j) / T where listed
// Sums are in fp32 in a fixed order; what a row hands out is rounded from them once (the loss, a small difference of
// logarithms, by way of 64 bits).  Rows whose |rho| is above FAR (masked tokens' value in every place, infinities; ordinary logits
// only below temperatures of 1e-5) take the differences before the factor, one element at a time.
//
// What bounds it: memory, and close behind it the 16 exponentials a clock of an SM (one per logit, two with a gradient: 57 and
// 114 us of the 82 and 164 that 8192 x 32768 bf16 take to pass) and the instructions (5.5 a logit for a sum, 11 with a gradient).
// Hence: each logit is fetched once, by asynchronous copies of 16 bytes that only the fetching thread reads again, so no barrier
// stands between a copy and its use; two logits per instruction where one does it; a reference that moves only when a power
// would exceed 2^SLACK; one barrier per row to join its sums; and persistent blocks, several to an SM, whose copies run ahead
// into the next row.
//   Rows that are only read (logprobs_kernel) stream through a ring of two batches, whatever their length.
//   Rows that need a second pass (gradients, distillation) stay in shared memory: pieces of up to 65 KB, three blocks to an SM;
//   as the second pass leaves a batch, the next row's takes its place.  A cluster of up to eight blocks shares a longer row and
//   exchanges its sums through distributed shared memory; so do blocks that share a row because rows are few.  Above 133120 fp32
//   logits eight pieces are longer, up to 128 KB, and one or two blocks on an SM (512 x 262144: gradient 321 us against 164 to pass,
//   distillation 282; 512 x 133120: 100 and 100 against 83).
// Measured, replayed from a graph, against the bytes at 6.54 TB/s: 8192 x 32768 bf16 log probabilities 85 us (82), with entropy
// 89 (82), with 64 alternatives 158 (83), gradient with entropy 179 (164), distillation with gradient 190 (165), with a rest 209;
// 1031 x 50021 fp32 with 5 alternatives 36 (32); 1000 x 131071 bf16 distillation from 128 entries and a rest 125 (80).
#include <algorithm>
#include <atomic>
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
// The border, in powers of two, from where a row is far.  fl(c max x) is off by half a unit in its last place: by 2 at 2^26 (by 64 at
// 2^31, where a sum starts to overflow or vanish).  At the smallest temperature, 2^-20, logits of 44 lie at the border.
constexpr float FAR = 0x1p26f;
constexpr double LOWEST = -0x1p27;            // below it a logit is masked, unless the row has nothing above -FAR
constexpr float BEYOND = 1e12f;               // from here on an error of 2 is rounding, and soon x c no number of 32 bits
constexpr float LN2 = 0.693147180559945309f;
constexpr int MAX_CLUSTER = 8;
constexpr float SLACK = 8.f;                  // a sum's reference stays while no power of two exceeds 2^SLACK
constexpr int CANDIDATES = 256;               // of the top alternatives

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
__device__ __forceinline__ float warp_most(float a) {     // of numbers
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(a));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// ---------------------------------------------------------------------------------------------- vectors of 16 bytes
struct Quad { uint32_t w[4]; };
__device__ __forceinline__ Quad quad(const uint4& v) { return Quad{{v.x, v.y, v.z, v.w}}; }
__device__ __forceinline__ uint4 four(const Quad& q) { return make_uint4(q.w[0], q.w[1], q.w[2], q.w[3]); }
template <typename T> __device__ __forceinline__ Quad nothing();          // -infinity throughout
template <> __device__ __forceinline__ Quad nothing<bf16>() { return Quad{{0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u}}; }
template <> __device__ __forceinline__ Quad nothing<float>() { return Quad{{0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u}}; }
template <typename T> struct Vec;
template <> struct Vec<bf16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ u64 pair(const Quad& v, int i) {
    const uint32_t w = v.w[i];
    return pack(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
  static __device__ __forceinline__ __nv_bfloat162 b2(uint32_t w) { return *(__nv_bfloat162*)&w; }
  static __device__ __forceinline__ uint32_t u2(__nv_bfloat162 w) { return *(uint32_t*)&w; }
  // the largest element; a NaN only if there is nothing else.  First in two halves.
  typedef __nv_bfloat162 Most;
  static __device__ __forceinline__ Most lowest() { return b2(0xFF80FF80u); }
  static __device__ __forceinline__ Most most(const Quad& v) { return __hmax2(__hmax2(b2(v.w[0]), b2(v.w[1])), __hmax2(b2(v.w[2]), b2(v.w[3]))); }
  static __device__ __forceinline__ Most more(Most a, Most b) { return __hmax2(a, b); }
  static __device__ __forceinline__ float value(Most m) { return __bfloat162float(__hmax(__low2bfloat16(m), __high2bfloat16(m))); }
  static __device__ __forceinline__ void clamp(Quad& v, float lo) {
    const __nv_bfloat162 l = __float2bfloat162_rn(lo);
#pragma unroll
    for (int i = 0; i < 4; ++i) v.w[i] = u2(__hmax2_nan(b2(v.w[i]), l));
  }
  static __device__ __forceinline__ float get(const Quad& v, int i) {
    const uint32_t w = v.w[i >> 1];
    return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
  }
  static __device__ __forceinline__ void set_pair(Quad& v, int i, u64 p) {
    const float2 f = unpack(p);
    v.w[i] = u2(__floats2bfloat162_rn(f.x, f.y));
  }
};
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ float at(const Quad& v, int i) { return __uint_as_float(v.w[i]); }
  static __device__ __forceinline__ u64 pair(const Quad& v, int i) { return pack(at(v, 2 * i), at(v, 2 * i + 1)); }
  typedef float Most;
  static __device__ __forceinline__ Most lowest() { return -INFINITY; }
  static __device__ __forceinline__ Most most(const Quad& v) { return fmaxf(fmaxf(at(v, 0), at(v, 1)), fmaxf(at(v, 2), at(v, 3))); }
  static __device__ __forceinline__ Most more(Most a, Most b) { return fmaxf(a, b); }
  static __device__ __forceinline__ float value(Most m) { return m; }
  static __device__ __forceinline__ void clamp(Quad& v, float lo) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v.w[i] = __float_as_uint(max_nan(at(v, i), lo));
  }
  static __device__ __forceinline__ float get(const Quad& v, int i) { return at(v, i); }
  static __device__ __forceinline__ void set_pair(Quad& v, int i, u64 p) {
    const float2 f = unpack(p);
    v.w[2 * i] = __float_as_uint(f.x);
    v.w[2 * i + 1] = __float_as_uint(f.y);
  }
};

// ---------------------------------------------------------------------------------------------- a row's pieces
// Threads that sweep over a row that passes by, or stays in shared memory for a second pass; FEW where rows are short and many.
constexpr int STREAM = 128, STAY = 128, FEW = 32;
// Vectors that a thread takes at a time: fewer steps with eight (scoring 8192 rows of 32768 in bf16 84.5 us against 89.6), more blocks
// on an SM and less left over in short rows with four (the same with 64 alternatives 157 against 167, 16384 rows of 512 30 against 36).
__host__ __device__ constexpr int batch_of(int threads, bool top) { return threads == FEW || top ? 4 : 8; }

struct Geometry {
  float c, inv_t;                             // log2(e) / T, 1 / T
  float lo;                                   // logits below it have probability 0 in rows that are not far
  float slack;                                // SLACK in units of a logit
  int cluster, per, batches;                  // blocks per row, vectors of a block's piece, batches of them
  int shift;                                  // log2 of the fours of vectors of which a thread leaves one maximum
};

// A block's piece of a row.  Its vectors are those aligned 16 bytes that lie in the row as a whole, `first` .. `first` +
// `count` of them here; element j of the row's ends, which no vector holds, belongs to one thread of the first block.
// Thread t works on vectors t, t + NT, ..., B to a batch, and nobody else sees its copies of them.
template <typename T, int NT, int B>
struct Piece {
  static constexpr int N = Vec<T>::N;
  const T* x;                                 // the row
  int head, first, count, edge;               // elements before the first vector; the thread's own element, or -1
  __device__ __forceinline__ Piece(const LogitsIn& in, long long r, int rank, const Geometry& g) : x((const T*)in.x + r * in.ld) {
    const int n = in.vocab, t = threadIdx.x;
    head = min(n, (int)((16 - ((uintptr_t)x & 15)) / sizeof(T)) & (N - 1));
    const int all = (n - head) / N, tail = head + all * N;
    first = rank * g.per;
    count = max(0, min(all - first, g.per));
    edge = rank != 0 ? -1 : t < head ? t : t - head < n - tail ? tail + t - head : -1;
  }
  __device__ __forceinline__ int element(int v) const { return head + (first + v) * N; }     // the first of vector v
  __device__ __forceinline__ bool whole(int b) const { return (b + 1) * B * NT <= count; }
  // Asks for batch b: its vectors u arrive at to[u * NT].  One group of copies, of nothing for b beyond the piece.
  __device__ __forceinline__ void fetch(uint4* to, int b) const {
    const int v = B * b * NT + threadIdx.x;
    const uint32_t d = (uint32_t)__cvta_generic_to_shared(to);
    const T* s = x + element(v);
    if (whole(b)) {
#pragma unroll
      for (int u = 0; u < B; ++u)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d + u * NT * 16), "l"(s + u * NT * N) : "memory");
    } else {
#pragma unroll
      for (int u = 0; u < B; ++u)
        if (v + u * NT < count) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d + u * NT * 16), "l"(s + u * NT * N) : "memory");
    }
    commit();
  }
  __device__ __forceinline__ static void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
  __device__ __forceinline__ void fetch_all(uint4* buf, const Geometry& g) const {
    for (int b = 0; b < g.batches; ++b) fetch(buf + B * b * NT + threadIdx.x, b);
  }
  __device__ __forceinline__ float edge_value() const { return edge >= 0 ? to_f(x[edge]) : -INFINITY; }
  __device__ __forceinline__ void store(T* dst, int v, const Quad& r) const {
    T* d = dst + element(v);
    if (((uintptr_t)d & 15) == 0) {
      *(uint4*)d = four(r);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) d[i] = from_f<T>(Vec<T>::get(r, i));
    }
  }
  __device__ __forceinline__ void zeros(T* dst) const {
    for (int v = threadIdx.x; v < count; v += NT) store(dst, v, Quad{{0, 0, 0, 0}});
    if (edge >= 0) dst[edge] = from_f<T>(0.f);
  }
};

// Waits until at most n of the thread's latest groups of copies are on their way (a smaller number waits for more).
__device__ __forceinline__ void wait_groups(int n) {
  if (n <= 0) asm volatile("cp.async.wait_group 0;" ::: "memory");
  else if (n == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else if (n == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else asm volatile("cp.async.wait_group 3;" ::: "memory");
}

// ---------------------------------------------------------------------------------------------- sums of a row
// The reference that a maximum gives; none below lo (masked tokens, of -infinity or the type's lowest value: their sum is
// 0, unless the row has nothing else and is far).
__device__ __forceinline__ float rho_of(float m, const Geometry& g) { return m < g.lo ? 0.f : __fmul_rn(m, g.c); }

struct Sums { float m, s, w; };               // max x, sum 2^y, sum 2^y y against rho_of(m)

// A sum against the reference rho moved to that of a maximum m, which is no lower; but the sum of nothing (0, or NaN) stands
// against 0, from where a power of two could be infinite.
template <bool W>
__device__ __forceinline__ void move(float& s, float& w, float rho, float m, const Geometry& g) {
  const float d = rho - rho_of(m, g), f = ex2(fminf(d, 0.f));
  if (W) w = f * fmaf(s, fmaxf(d, -1e30f), w);
  s *= f;
}

// A thread's running sums.  The reference is the maximum of the first four vectors above lo, and is raised when later ones
// would give a power above 2^SLACK, which few do (raising it with every new maximum made every fourth step one of all warps).
template <typename T, bool W>
struct Running {
  u64 s0 = 0, s1 = 0, w0 = 0, w1 = 0, nrho = 0;
  float m = -INFINITY, rho = 0.f, top;        // max x; what a logit may be without a new reference
  __device__ __forceinline__ explicit Running(const Geometry& g) : top(g.lo) {}
  __device__ __forceinline__ void raise(float to, const Geometry& g) {
    const float r = rho_of(to, g), d = rho - r, f = ex2(fminf(d, 0.f));    // the first time the sums are 0, or NaN
    const u64 f2 = pack(f, f), d2 = pack(d, d);
    if (W) { w0 = mul2(f2, fma2(s0, d2, w0)); w1 = mul2(f2, fma2(s1, d2, w1)); }
    s0 = mul2(s0, f2);
    s1 = mul2(s1, f2);
    rho = r;
    nrho = pack(-r, -r);
    top = to + g.slack;
  }
  template <int M>
  __device__ __forceinline__ void add(Quad (&a)[M], float bm, const Geometry& g) {
    constexpr int P = Vec<T>::N / 2;
    const u64 c2 = pack(g.c, g.c);
    m = fmaxf(m, bm);
    if (bm > top) raise(bm, g);
#pragma unroll
    for (int u = 0; u < M; ++u) {
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
  // Adds batch b, which has arrived; leaf(four, maximum of its even vectors, of the odd ones) hears of every four vectors.
  // The reference goes by fours whatever the batch, so that kernels of other batches give the same bits.
  template <int NT, int B, typename Leaf>
  __device__ __forceinline__ void batch(const Piece<T, NT, B>& p, const uint4* from, int b, const Geometry& g, Leaf leaf) {
    typedef Vec<T> V;
    auto four = [&](Quad (&a)[4], int q) {
      const typename V::Most e = V::more(V::most(a[0]), V::most(a[2])), o = V::more(V::most(a[1]), V::most(a[3]));
      leaf(q, e, o);
      add<4>(a, V::value(V::more(e, o)), g);
    };
    if (p.whole(b)) {
      Quad a[B / 4][4];
#pragma unroll
      for (int u = 0; u < B; ++u) a[u / 4][u % 4] = quad(from[u * NT]);
#pragma unroll
      for (int q = 0; q < B / 4; ++q) four(a[q], B / 4 * b + q);
    } else {
      const int first = threadIdx.x & ~31;               // of the warp: what no lane has is left out
#pragma unroll 1
      for (int q = B / 4 * b; q < B / 4 * (b + 1); ++q, from += 4 * NT) {
        if (4 * (q + 1) * NT <= p.count) {
          Quad a[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) a[u] = quad(from[u * NT]);
          four(a, q);
          continue;
        }
#pragma unroll 1
        for (int u = 0; u < 4; ++u) {
          const int v = (4 * q + u) * NT;
          if (v + first >= p.count) return;
          Quad a[1] = {nothing<T>()};
          if (v + (int)threadIdx.x < p.count) a[0] = quad(from[u * NT]);
          const typename V::Most m = V::most(a[0]);
          leaf(q, u & 1 ? V::lowest() : m, u & 1 ? m : V::lowest());
          add<1>(a, V::value(m), g);
        }
      }
    }
  }
  // The thread's own element of the row's ends, if it is there (not -infinity), and the sums against the warp's maximum.
  __device__ __forceinline__ Sums end(float edge, const Geometry& g) {
    m = fmaxf(m, edge);
    if (edge > top) raise(edge, g);
    const float2 sp = unpack(add2(s0, s1)), wp = unpack(add2(w0, w1));
    float s = sp.x + sp.y, w = wp.x + wp.y;
    if (edge != -INFINITY) {
      const float y = fmaf(max_nan(edge, g.lo), g.c, -rho), e = ex2(y);
      s += e;
      if (W) w = fmaf(e, y, w);
    }
    const float wm = warp_most(m);
    if (top == g.lo) rho = rho_of(wm, g);                // nothing but masked tokens (or NaN)
    move<W>(s, w, rho, wm, g);
    return Sums{wm, s, w};
  }
};

// The same against the row's maximum, for far rows, one element after the other, without the `k` tokens of `skip`, each of them compared
// with each: 8192 x 32768 bf16 360 us (84 if not far), gradient 641 (178), distillation 820 (212), beside a rest and 64 entries 6300 (229).
template <typename T, int NT, int B, bool W>
__device__ __noinline__ Sums sweep_far(const Piece<T, NT, B> p, const Geometry g, float m, float edge, const int* skip = nullptr, int k = 0) {
  Sums a{m, 0.f, 0.f};
  auto add = [&](float x) {
    if (x == -INFINITY) return;
    const float y = (x - m) * g.c, e = ex2(y);
    a.s += e;
    if (W && e != 0.f) a.w = fmaf(e, y, a.w);
  };
  for (int v = threadIdx.x; v < p.count; v += NT)
    for (int i = 0; i < Vec<T>::N; ++i) {
      const int j = p.element(v) + i;
      bool out = false;
      for (int l = 0; l < k; ++l) out = out || skip[l] == j;
      if (!out) add(to_f(p.x[j]));
    }
  add(edge);
  return a;
}

// What the warps of a row's blocks tell one another; of two rows in turn.
template <int NT, bool CL>
struct Exchange { float4 part[2][2][(CL ? MAX_CLUSTER : 1) * NT / 32]; };

// All warps of the block, wherever in the code each of them is.
__device__ __forceinline__ void sync_block() {
  __syncwarp();
  asm volatile("bar.sync 0;" ::: "memory");
}

template <bool CL>
__device__ __forceinline__ void sync_row() {
  if (CL) {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  } else {
    sync_block();
  }
}

// Joins the warps' sums: every warp leaves its part with all blocks of the row, and behind sync_row takes the whole, the same
// bits in every thread.  The parts of a warp have one reference, its maximum's, or in a far row the row's.
template <int NT, bool W, bool CL>
__device__ __forceinline__ void leave_part(Sums a, float4* part, const Geometry& g, int rank) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  a.s = warp_sum(a.s);
  if (W) a.w = warp_sum(a.w);
  const float4 mine = make_float4(a.m, a.s, a.w, 0.f);
  if (CL) {
    if (lane < g.cluster) cg::this_cluster().map_shared_rank(part, lane)[rank * (NT / 32) + warp] = mine;
  } else if (lane == 0) {
    part[warp] = mine;
  }
}
template <int NT, bool W, bool CL, bool FARROW>
__device__ __forceinline__ Sums take_parts(const float4* part, const Geometry& g) {
  Sums t{-INFINITY, 0.f, 0.f};
  auto add = [&](float4 b) {
    if (!FARROW) move<W>(b.y, b.z, rho_of(b.x, g), t.m, g);
    t.s += b.y;
    t.w += b.z;
  };
  if constexpr (CL) {                                    // up to a part per lane
    const int lane = threadIdx.x & 31, parts = g.cluster * (NT / 32);
    static_assert(MAX_CLUSTER * NT <= 32 * 32, "a part per lane");
    if (lane < parts) t.m = part[lane].x;
    t.m = warp_most(t.m);
    if (lane < parts) add(part[lane]);
    t.s = warp_sum(t.s);
    if (W) t.w = warp_sum(t.w);
  } else {                                               // few: each thread by itself
#pragma unroll
    for (int i = 0; i < NT / 32; ++i) t.m = fmaxf(t.m, part[i].x);
#pragma unroll
    for (int i = 0; i < NT / 32; ++i) add(part[i]);
  }
  return t;
}
template <int NT, bool W, bool CL, bool FARROW>
__device__ __forceinline__ Sums join(Sums a, float4* part, const Geometry& g, int rank) {
  leave_part<NT, W, CL>(a, part, g, rank);
  sync_row<CL>();
  return take_parts<NT, W, CL, FARROW>(part, g);
}

// A row's reference.
struct Ref {
  float m, rho, c, inv_t;
  bool far;
  __device__ __forceinline__ Ref(float m_, const Geometry& g) : m(m_), rho(rho_of(m_, g)), c(g.c), inv_t(g.inv_t),
                                                              far(m_ != -INFINITY && !(fabsf(m_) * g.c <= FAR)) {}
  __device__ __forceinline__ bool apart(float x) const { return far || fabsf(x) * c > BEYOND; }
  __device__ __forceinline__ float y(float x) const { return far ? (x - m) * c : fmaf(x, c, -rho); }
  // y ln 2, of a masked token's lowest value too
  __device__ __forceinline__ float nat(float x) const { return apart(x) ? (x - m) * inv_t : fmaf(x, c, -rho) * LN2; }
  // how far v lies above it, times q: that may be a number of 32 bits where the distance is none
  __device__ __forceinline__ float above(float q, float v, float x) const {
    return apart(x) ? fmaf(q * (0.5f * m - 0.5f * x), 2.f * inv_t, q * v) : q * fmaf(-fmaf(x, c, -rho), LN2, v);
  }
};

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

constexpr int ENTRIES = 8;                    // maxima that a thread leaves of its batches

template <int NT>
struct TopSpace {
  alignas(16) u64 list[CANDIDATES];           // read two at a time
  float maxima[ENTRIES][NT];                  // of 2^shift fours of vectors each
  uint32_t halves[2 * NT];                    // the order of every thread's maxima over its even and odd vectors
  unsigned short hits[ENTRIES * NT];
  int queue[CANDIDATES];                      // vectors to look at
  uint32_t bound;
  int count, found, queued;
  u64 sorted[MAX_CLUSTER][TOP_MAX];           // of the row's first block: what each block found
};

// One warp: a bound that at least k of the values reach (0 if there are not as many), and not many more unless they are equal.
template <int COUNT>
__device__ __forceinline__ uint32_t bound_of(const uint32_t* values, int k) {
  constexpr int P = COUNT / 32;
  uint32_t v[P], lo = 0xffffffffu, hi = 0;
  int n = 0;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    v[i] = values[32 * i + (threadIdx.x & 31)];
    if (v[i]) { lo = min(lo, v[i]); ++n; }
    hi = max(hi, v[i]);
  }
  if (__reduce_add_sync(0xffffffffu, n) < k) return 0;
  if (k * P <= 16) {                                     // few: one after the other
    for (n = 0; n < k;) {
      hi = 0;
#pragma unroll
      for (int i = 0; i < P; ++i) hi = max(hi, v[i]);
      hi = __reduce_max_sync(0xffffffffu, hi);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const bool is = v[i] == hi;
        n += __popc(__ballot_sync(0xffffffffu, is));
        if (is) v[i] = 0;
      }
    }
    return hi;
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi) + 1;
  while (hi - lo > 1) {                                  // at least k reach lo, fewer than k reach hi
    const uint32_t mid = lo + (hi - lo) / 2;
    n = 0;
#pragma unroll
    for (int i = 0; i < P; ++i) n += v[i] >= mid;
    n = __reduce_add_sync(0xffffffffu, n);
    if (n < k) {
      hi = mid;
    } else {
      lo = mid;
      if (n <= k + k / 8) break;
    }
  }
  return lo;
}

// Puts the keys of the piece's k largest logits (all of them, if there are fewer) into ts.list and returns how many are
// there: at least min(k, logits), at most CANDIDATES.
//   The k-th largest of the 2 NT maxima of the threads' even and odd vectors, or a little less, is reached by at least k
//   logits, and of logits in no particular order by hardly more (k = 64 of 256: 74).  Only vectors under a maximum that
//   reaches it are read again, and only elements of those that do are compared.
//   Where more than CANDIDATES logits reach it (many equal ones, or large ones side by side), the bound is raised by halving
//   until they fit, or until it is the k-th largest value itself, of which those with the lowest ids are taken.
template <typename T, int NT, int B>
__device__ int top_candidates(const Piece<T, NT, B>& p, float edge, int k, int shift, TopSpace<NT>& ts) {
  constexpr int N = Vec<T>::N, AT_ONCE = 3;
  constexpr uint32_t NOTHING = 0x007fffffu;              // the order of -infinity; maxima of it may hide a NaN, which stands below
  const int t = threadIdx.x, per = 4 << shift, entries = (p.count + per * NT - 1) / (per * NT);
  auto vector = [&](int v) { return quad(*(const uint4*)(p.x + p.element(v))); };
  // The logits that reach b go to the list; returns how many there are, or some number above CANDIDATES if there are more.
  auto collect = [&](uint32_t b) {
    sync_block();
    if (t == 0) ts.count = ts.found = ts.queued = 0;
    sync_block();
    const float bound = b <= NOTHING ? -INFINITY : value_of(b);
    auto add = [&](float x, int j) {
      const uint32_t o = order_of(x);
      if (o < b) return;
      const int at = atomicAdd(&ts.count, 1);
      if (at < CANDIDATES) ts.list[at] = key_of(o, j);
    };
    for (int e = 0; e < entries; ++e)
      if (e * per * NT + t < p.count && (b <= NOTHING || ts.maxima[e][t] >= bound))
        ts.hits[atomicAdd(&ts.found, 1)] = (unsigned short)(e * NT + t);
    if (p.edge >= 0) add(edge, p.edge);
    sync_block();
    const int units = ts.found * per;
    for (int i0 = t; i0 < units; i0 += AT_ONCE * NT) {
      Quad a[AT_ONCE];
      int v[AT_ONCE];
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) {
        const int i = i0 + u * NT, h = i < units ? ts.hits[i >> (shift + 2)] : 0;
        v[u] = i < units ? ((h / NT << (shift + 2)) + (i & (per - 1))) * NT + h % NT : p.count;
        a[u] = v[u] < p.count ? vector(v[u]) : nothing<T>();
      }
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u)
        if (v[u] < p.count && (b == 0 || Vec<T>::value(Vec<T>::most(a[u])) >= bound)) {
          const int at = atomicAdd(&ts.queued, 1);
          if (at < CANDIDATES) ts.queue[at] = v[u];
        }
    }
    sync_block();
    if (ts.queued > CANDIDATES) return ts.queued;        // each has a logit that reaches it
    for (int i = t; i < ts.queued * N; i += NT) {
      const int j = p.element(ts.queue[i / N]) + i % N;
      add(to_f(p.x[j]), j);
    }
    sync_block();
    return ts.count;
  };
  if (t < 32) {
    const uint32_t b = bound_of<2 * NT>(ts.halves, k);
    if (t == 0) ts.bound = b;
  }
  sync_block();
  uint32_t lo = ts.bound;
  int n = collect(lo);
  if (n <= CANDIDATES) return n;
  uint32_t hi = 0xffffffffu, probe = lo + 1;             // often lo itself is the value
  while (hi - lo > 1) {
    n = collect(probe);
    if (n < k) hi = probe;
    else if (n <= CANDIDATES) return n;
    else lo = probe;
    probe = lo + (hi - lo) / 2;
  }
  n = collect(hi);                                       // fewer than k; the rest are equal to lo, their ids ascending
  if (t < 32) {                                          // one warp, from the row's first elements over its vectors to its last
    auto take = [&](unsigned same, int j) {              // bit i: element j + i is equal
      int before = __popc(same);
      const int own = before;
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, before, o);
        if (t >= o) before += y;
      }
      const int total = __shfl_sync(0xffffffffu, before, 31);
      for (int at = n + before - own; same && at < k; ++at) {
        const int i = __ffs(same) - 1;
        ts.list[at] = key_of(lo, j + i);
        same &= same - 1;
      }
      n += total;
    };
    const bool equal = p.edge >= 0 && order_of(edge) == lo;
    take(equal && p.edge < p.head, p.edge);
    for (int v0 = 0; v0 < p.count && n < k; v0 += 32) {
      const int v = v0 + t;
      unsigned same = 0;
      if (v < p.count) {
        const Quad a = vector(v);
#pragma unroll
        for (int l = 0; l < N; ++l) same |= (unsigned)(order_of(Vec<T>::get(a, l)) == lo) << l;
      }
      take(same, p.element(v));
    }
    if (n < k) take(equal && p.edge >= p.head, p.edge);
    if (t == 0) ts.bound = (uint32_t)min(n, k);
  }
  sync_block();
  return (int)ts.bound;
}

// A candidate's place is the number of larger ones.
template <int NT, typename Put>
__device__ __forceinline__ void rank_candidates(const u64* list, int found, int k, Put put) {
  for (int i = threadIdx.x; i < found; i += NT) {
    const u64 key = list[i];
    int at = 0;
#pragma unroll 4
    for (int j = 0; j < found / 2; ++j) {
      const ulonglong2 two = ((const ulonglong2*)list)[j];
      at += (two.x > key) + (two.y > key);
    }
    if (found & 1) at += list[found - 1] > key;
    if (at < k) put(at, key);
  }
}

// ---------------------------------------------------------------------------------------------- kernels
// A block (a cluster) takes every groups-th row.
struct Place {
  int rank, groups;                           // of the block in its cluster; clusters
  long long row;                              // the first
  template <bool CL> static __device__ __forceinline__ Place of(const Geometry& g) {
    return CL ? Place{(int)(blockIdx.x % g.cluster), (int)(gridDim.x / g.cluster), (long long)(blockIdx.x / g.cluster)}
              : Place{0, (int)gridDim.x, (long long)blockIdx.x};
  }
};

// What a thread leaves of a row for the search of its top alternatives.
template <typename T, int NT>
struct Leaves {
  typedef Vec<T> V;
  typename V::Most even = V::lowest(), odd = V::lowest(), m = V::lowest();
  __device__ __forceinline__ void group(TopSpace<NT>& ts, int q, typename V::Most e, typename V::Most o, int shift) {
    if (m_of != q >> shift) {
      m = V::lowest();
      m_of = q >> shift;
    }
    even = V::more(even, e);
    odd = V::more(odd, o);
    m = V::more(m, V::more(e, o));
    ts.maxima[q >> shift][threadIdx.x] = V::value(m);
  }
  int m_of = -1;                              // the entry that m belongs to
  __device__ __forceinline__ void end(TopSpace<NT>& ts, float edge) {
    const float a = V::value(even), b = fmaxf(V::value(odd), edge);
    ts.halves[threadIdx.x] = a > -INFINITY ? order_of(a) : 0u;         // what counts as -infinity may be a NaN, which stands below
    ts.halves[NT + threadIdx.x] = b > -INFINITY ? order_of(b) : 0u;
  }
};

constexpr int SLOTS = 2;                      // batches on their way

// Batches pass through a ring of SLOTS, each thread's by itself: copies run ahead of the sums by SLOTS batches, over the end of
// a row into the next ones, so that they go on while a row's sums are joined and handed out.
template <typename T, int NT, bool W, bool CL, bool TOP>
__global__ void __launch_bounds__(NT) logprobs_kernel(const __grid_constant__ LogprobsArgs a, const __grid_constant__ Geometry g) {
  constexpr int B = batch_of(NT, TOP);
  __shared__ Exchange<NT, CL> ex;
  cudaGridDependencySynchronize();
  cluster_start<CL>();
  const Place me = Place::of<CL>(g);
  const int rank = me.rank, tid = threadIdx.x, rows = a.in.rows;
  const bool speaks = rank == 0 && tid == 0;             // for the row
  Piece<T, NT, B> p(a.in, me.row, rank, g), ahead = p;
  long long ahead_row = me.row;
  int ahead_batch = 0, slot = 0;
  auto fetch = [&]() {
    if (ahead_row >= rows) return p.commit();
    ahead.fetch(dynamic + slot * B * NT + tid, ahead_batch);
    if (++ahead_batch == g.batches) {
      ahead_batch = 0;
      ahead_row += me.groups;
      if (ahead_row < rows) ahead = Piece<T, NT, B>(a.in, ahead_row, rank, g);
    }
  };
  static_assert(SLOTS == 2, "slots take turns");
  fetch();
  slot = 1;
  fetch();
  slot = 0;
  float edge = p.edge_value();
  int t = speaks && a.tokens ? token_of(a.tokens, me.row, a.in.vocab, a.in.out_of_range, true) : -1;
  float xt = t >= 0 ? to_f(p.x[t]) : 0.f;
  cluster_started<CL>();
  TopSpace<NT>& ts = *(TopSpace<NT>*)(dynamic + SLOTS * B * NT);
  int turn = 0;
  for (long long r = me.row; r < rows; r += me.groups, turn ^= 1) {
    const bool has_next = r + me.groups < rows;
    const Piece<T, NT, B> next(a.in, has_next ? r + me.groups : r, rank, g);
    const float next_edge = next.edge_value();
    const int next_t = speaks && a.tokens && has_next ? token_of(a.tokens, r + me.groups, a.in.vocab, a.in.out_of_range, true) : -1;
    Running<T, W> run(g);
    Leaves<T, NT> leaves;
    for (int b = 0; b < g.batches; ++b) {
      wait_groups(SLOTS - 1);
      run.batch(p, dynamic + slot * B * NT + tid, b, g, [&](int q, typename Vec<T>::Most e, typename Vec<T>::Most o) {
        if (TOP) leaves.group(ts, q, e, o, g.shift);
      });
      fetch();
      slot ^= 1;
    }
    if (TOP) leaves.end(ts, edge);
    Sums s = join<NT, W, CL, false>(run.end(edge, g), ex.part[turn][0], g, rank);
    const Ref ref(s.m, g);
    if (ref.far) s = join<NT, W, CL, true>(sweep_far<T, NT, B, W>(p, g, s.m, edge), ex.part[turn][1], g, rank);
    const float logs = logf(s.s);
    auto logp = [&](float v) { return s.s == 0.f ? -INFINITY : ref.nat(v) - logs; };
    const float next_xt = next_t >= 0 ? to_f(next.x[next_t]) : 0.f;
    if (speaks) {
      if (a.logp) a.logp[r] = t >= 0 ? logp(xt) : 0.f;
      if (W && a.entropy) a.entropy[r] = s.s == 0.f ? 0.f : fmaf(-LN2, s.w / s.s, logs);
      if (a.lse) a.lse[r] = s.s == 0.f ? -INFINITY : ref.far ? fmaf(s.m, g.inv_t, logs) : fmaf(ref.rho, LN2, logs);
    }
    if constexpr (TOP) {
      const int k = a.top_k;
      auto put = [&](int at, u64 key) {
        a.top_ids[r * k + at] = (int)~(uint32_t)key;
        a.top_logp[r * k + at] = logp(value_of((uint32_t)(key >> 32)));
      };
      const int found = top_candidates<T, NT, B>(p, edge, k, g.shift, ts);
      u64* sorted = CL ? cg::this_cluster().map_shared_rank(&ts.sorted[rank][0], 0) : nullptr;
      rank_candidates<NT>(ts.list, found, k, [&](int at, u64 key) {
        if (CL) sorted[at] = key;
        else put(at, key);
      });
      if constexpr (CL) {
        for (int i = found + tid; i < k; i += NT) sorted[i] = 0;   // fewer logits than k in this piece
        sync_row<true>();
        if (rank == 0)
          for (int i = tid; i < g.cluster * k; i += NT) {          // the place among all: the larger ones of every block's list
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
      // the lists are used again behind the barrier of the next row's sums
    }
    p = next;
    edge = next_edge;
    t = next_t;
    xt = next_xt;
  }
  wait_groups(0);
}

// The row's second pass: dst = 2^y (k0 + k1 y), a token's own term added; the next row takes the place.
template <typename T, int NT, int B, bool W>
__device__ __forceinline__ void gradient(const Piece<T, NT, B>& p, uint4* buf, float edge, const Geometry& g, const Ref& ref, float k0, float k1,
                                         int t, float at_t, T* dst, const Piece<T, NT, B>& next, bool fetch_next) {
  constexpr int N = Vec<T>::N;
  auto one = [&](float x, int j) {
    const float y = ref.y(W && !ref.far ? max_nan(x, g.lo) : x), e = ex2(y);
    return (W && e != 0.f ? e * fmaf(k1, y, k0) : e * k0) + (j == t ? at_t : 0.f);       // y may be infinite
  };
  if (p.edge >= 0) dst[p.edge] = from_f<T>(one(edge, p.edge));
  if (ref.far) {
    for (int v = threadIdx.x; v < p.count; v += NT) {
      const Quad x = quad(buf[v]);
      Quad o;
      const int j = p.element(v);
#pragma unroll
      for (int i = 0; i < N / 2; ++i)
        Vec<T>::set_pair(o, i, pack(one(Vec<T>::get(x, 2 * i), j + 2 * i), one(Vec<T>::get(x, 2 * i + 1), j + 2 * i + 1)));
      p.store(dst, v, o);
    }
    if (fetch_next) next.fetch_all(buf, g);
    return;
  }
  const u64 c2 = pack(g.c, g.c), nrho = pack(-ref.rho, -ref.rho), k02 = pack(k0, k0), k12 = pack(k1, k1);
  const bool aligned = ((uintptr_t)(dst + p.head) & 15) == 0;
  // the token's element, written again by the thread that writes its vector
  const int spot = t - p.head - p.first * N;
  const bool mine = t >= 0 && spot >= 0 && spot < p.count * N && spot / N % NT == threadIdx.x;
  const float at = mine ? one(to_f(((const T*)buf)[spot]), t) : 0.f;
  auto one_vector = [&](Quad a) {
    Quad o;
    if (W) Vec<T>::clamp(a, g.lo);
    u64 d[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const u64 y = fma2(Vec<T>::pair(a, i), c2, nrho), e = ex22(y);
      d[i] = mul2(e, W ? fma2(k12, y, k02) : k02);
    }
#pragma unroll
    for (int i = 0; i < N / 2; ++i) Vec<T>::set_pair(o, i, d[i]);
    return o;
  };
  for (int b = 0; b < g.batches; ++b) {
    const int v0 = B * b * NT + threadIdx.x;
    if (p.whole(b) && aligned) {
      uint4* d = (uint4*)(dst + p.element(v0));
#pragma unroll
      for (int u = 0; u < B; ++u) d[u * NT] = four(one_vector(quad(buf[v0 + u * NT])));
    } else {
      for (int v = v0; v < min(v0 + B * NT, p.count); v += NT) p.store(dst, v, one_vector(quad(buf[v])));
    }
    if (fetch_next) next.fetch(buf + v0, b);
  }
  if (mine) dst[t] = from_f<T>(at);
}

// The sums of a row whose batches all have their place: they stay, or as they are read make room for those of the next row.
template <typename T, int NT, int B, bool W, bool REFILL>
__device__ __forceinline__ Sums sweep(const Piece<T, NT, B>& p, uint4* buf, float edge, const Geometry& g, const Piece<T, NT, B>& next, bool has_next) {
  Running<T, W> run(g);
  for (int b = 0; b < g.batches; ++b) {
    wait_groups(REFILL ? g.batches - 1 : g.batches - 1 - b);
    run.batch(p, buf + B * b * NT + threadIdx.x, b, g, [](int, typename Vec<T>::Most, typename Vec<T>::Most) {});
    if (REFILL) {
      if (has_next) next.fetch(buf + B * b * NT + threadIdx.x, b);
      else p.commit();
    }
  }
  return run.end(edge, g);
}

template <typename T, int NT, bool W, bool CL>
__global__ void __launch_bounds__(NT, NT == STAY ? 4 : 1) logprobs_bwd_kernel(const __grid_constant__ LogprobsBwdArgs a, const __grid_constant__ Geometry g) {
  constexpr int B = batch_of(NT, false);
  __shared__ Exchange<NT, CL> ex;
  cudaGridDependencySynchronize();
  cluster_start<CL>();
  const Place me = Place::of<CL>(g);
  const int rank = me.rank, rows = a.in.rows;
  uint4* buf = dynamic;
  struct In {                                 // what comes into a row
    int t;
    float ga, gb, gl;
    __device__ __forceinline__ bool any() const { return !(ga == 0.f && gb == 0.f && gl == 0.f); }
  };
  auto incoming = [&](long long r) {
    In i{-1, 0.f, W ? a.dentropy[r] : 0.f, a.dlse ? a.dlse[r] : 0.f};
    if (a.dlogp) {
      i.t = token_of(a.tokens, r, a.in.vocab, a.in.out_of_range, rank == 0 && threadIdx.x == 0);
      i.ga = i.t >= 0 ? a.dlogp[r] : 0.f;
    }
    return i;
  };
  Piece<T, NT, B> p(a.in, me.row, rank, g);
  In in = incoming(me.row);
  if (in.any()) p.fetch_all(buf, g);
  float edge = p.edge_value();
  cluster_started<CL>();
  int turn = 0;
  for (long long r = me.row; r < rows; r += me.groups, turn ^= 1) {
    const long long rn = r + me.groups < rows ? r + me.groups : r;
    const Piece<T, NT, B> next(a.in, rn, rank, g);
    const In next_in = incoming(rn);
    const float next_edge = next.edge_value();
    T* dx = (T*)a.dx + r * a.ld_out;
    if (in.any()) {
      Sums s = join<NT, W, CL, false>(sweep<T, NT, B, W, false>(p, buf, edge, g, next, false), ex.part[turn][0], g, rank);
      const Ref ref(s.m, g);
      if (ref.far) s = join<NT, W, CL, true>(sweep_far<T, NT, B, W>(p, g, s.m, edge), ex.part[turn][1], g, rank);
      const bool more = rn != r && next_in.any();
      if (s.s == 0.f) {                                  // no token
        p.zeros(dx);
        if (more) next.fetch_all(buf, g);
      } else {
        const float k = g.inv_t / s.s;
        gradient<T, NT, B, W>(p, buf, edge, g, ref, W ? (in.gl - in.ga + in.gb * (LN2 * (s.w / s.s))) * k : (in.gl - in.ga) * k, -in.gb * LN2 * k, in.t,
                       in.ga * g.inv_t, dx, next, more);
      }
    } else {
      p.zeros(dx);
      if (rn != r && next_in.any()) next.fetch_all(buf, g);
    }
    p = next;
    in = next_in;
    edge = next_edge;
  }
  wait_groups(0);
}

// Distillation: warps that sweep over the logits, as above, and one for the teacher's row.  Four entries per lane; while the
// others sum a row it prepares the next one, and behind their sums it forms the loss and writes the listed tokens' gradient.
constexpr int PER_LANE = TOP_MAX / 32, CLAIMS = 512;

struct Lesson {                               // what the sums of a row are weighed with
  alignas(16) int id[TOP_MAX];                // tokens listed, -1: none; read four at a time
  float most, student;                        // largest logit of the listed tokens; their sum against it
  float Q, qr;                                // teacher's weight in all, and of what is not listed
  int any;                                    // there is weight
};
static_assert(offsetof(Lesson, id) % 16 == 0 && sizeof(Lesson) % 16 == 0, "four ids at a time");

// A row's sums weighed: S against the row's maximum, f the factor of the sums o to it, kappa of the gradient.
struct Weighed {
  Ref ro, ref;
  float f, S;
  __device__ __forceinline__ Weighed(const Sums& o, const Lesson& l, bool rest, const Geometry& g)
      : ro(o.m, g), ref(rest ? fmaxf(o.m, l.most) : o.m, g), f(1.f), S(o.s) {
    if (!rest) return;                                   // the sums are those of all tokens
    f = factor(ro);
    S = o.s * f + l.student * factor(Ref(l.most, g));
  }
  // b's reference above ref's, in powers of two: in 64 bits, as a far row's, its maximum times c, need be no number of 32 bits.
  __device__ __forceinline__ double apart(const Ref& b) const {
    return (b.far ? (double)b.m * b.c : (double)b.rho) - (ref.far ? (double)ref.m * ref.c : (double)ref.rho);
  }
  __device__ __forceinline__ float factor(const Ref& b) const {
    return b.m == -INFINITY ? 0.f : ex2(b.far || ref.far ? (float)apart(b) : b.rho - ref.rho);
  }
};

// Where the two meet; whoever has nothing to wait for arrives and goes on.
enum { LANDED = 1, PATCHED, LESSON, SUMMED, WRITTEN };
template <int NT>
__device__ __forceinline__ void arrive(int what) {
  __syncwarp();
  asm volatile("bar.arrive %0, %1;" ::"r"(what), "n"(NT + 32) : "memory");
}
template <int NT>
__device__ __forceinline__ void await(int what) {
  __syncwarp();
  asm volatile("bar.sync %0, %1;" ::"r"(what), "n"(NT + 32) : "memory");
}
// The sums of a row: the sweeping warps leave them when the row's lesson is there; the teacher's warp hands it over and goes
// on, and takes the sums up later.
template <int NT, bool CL>
__device__ __forceinline__ void hand_over() {
  __syncwarp();
  if (CL) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  else arrive<NT>(LESSON);
}
template <int NT, bool CL>
__device__ __forceinline__ void take_up() {
  __syncwarp();
  if (CL) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  else await<NT>(SUMMED);
}
template <int NT, bool CL>
__device__ __forceinline__ void summed() {
  if (CL) {
    sync_row<true>();
  } else {
    await<NT>(LESSON);
    arrive<NT>(SUMMED);
  }
}

template <typename T, int NT, bool CL>
__global__ void __launch_bounds__(NT + 32, NT == STAY ? 4 : 1) distill_kernel(const __grid_constant__ DistillArgs a, const __grid_constant__ Geometry g) {
  constexpr int N = Vec<T>::N, B = batch_of(NT, false);
  __shared__ Exchange<NT, CL> ex;
  __shared__ Lesson lessons[2];               // of two rows in turn
  __shared__ float edges[2 * N];
  __shared__ int claims[CLAIMS];              // the teacher's warp's
  cudaGridDependencySynchronize();
  cluster_start<CL>();
  const Place me = Place::of<CL>(g);
  const int rank = me.rank, lane = threadIdx.x & 31, rows = a.in.rows;
  uint4* buf = dynamic;
  Piece<T, NT, B> p(a.in, me.row, rank, g);
  int turn = 0;

  if (threadIdx.x < NT) {
    p.fetch_all(buf, g);
    float edge = p.edge_value();
    cluster_started<CL>();
    for (long long r = me.row; r < rows; r += me.groups, turn ^= 1) {
      const bool has_next = r + me.groups < rows;
      const Piece<T, NT, B> next(a.in, has_next ? r + me.groups : r, rank, g);
      const float next_edge = next.edge_value(), dl = a.dloss ? a.dloss[r] : 1.f;
      if (a.rest) {                                      // the listed tokens leave the row
        wait_groups(0);
        if (p.edge >= 0) edges[threadIdx.x] = edge;
        arrive<NT>(LANDED);
        await<NT>(PATCHED);
        if (p.edge >= 0) edge = edges[threadIdx.x];
      }
      leave_part<NT, false, CL>(a.dx ? sweep<T, NT, B, false, false>(p, buf, edge, g, next, false) : sweep<T, NT, B, false, true>(p, buf, edge, g, next, has_next),
                                ex.part[turn][0], g, rank);
      summed<NT, CL>();
      Sums o = take_parts<NT, false, CL, false>(ex.part[turn][0], g);
      const Lesson& l = lessons[turn];
      if (Ref(o.m, g).far) o = join<NT, false, CL, true>(sweep_far<T, NT, B, false>(p, g, o.m, edge, l.id, a.rest ? a.k : 0), ex.part[turn][1], g, rank);
      if (a.dx) {
        T* dx = (T*)a.dx + r * a.ld_out;
        if (!l.any || dl == 0.f) {
          p.zeros(dx);
          if (has_next) next.fetch_all(buf, g);
        } else {
          const Weighed s(o, l, a.rest, g);
          const float kappa = s.S != s.S ? s.S : o.s == 0.f ? 0.f : (l.Q * s.f / s.S - (l.qr > 0.f ? l.qr / o.s : 0.f)) * (dl * a.scale * g.inv_t);
          gradient<T, NT, B, false>(p, buf, edge, g, s.ro, kappa, 0.f, -1, 0.f, dx, next, has_next);
        }
        arrive<NT>(WRITTEN);                             // the listed tokens' gradient goes over it
      }
      p = next;
      edge = next_edge;
    }
    wait_groups(0);
    return;
  }

  struct Entries { int id[PER_LANE]; float t[PER_LANE], x[PER_LANE]; };       // token, teacher's value, student's logit
  struct Weights { float q[PER_LANE], lq[PER_LANE]; double mass; unsigned first; bool twins; };     // q = exp(lq) by mass, or in REST by 1
  const int used = (a.k + 31) / 32;                      // entries per lane
  auto read = [&](long long r, Entries& e) {
#pragma unroll
    for (int i = 0; i < PER_LANE; ++i) {
      const int j = lane + 32 * i;
      e.id[i] = -1;
      e.t[i] = -INFINITY;
      e.x[i] = -INFINITY;
      if (j < a.k && r < rows) {
        e.id[i] = a.ids[r * a.k + j];
        e.t[i] = a.teacher[r * a.k + j];
      }
    }
  };
  auto look = [&](const T* x, Entries& e) {              // up the student's logits
#pragma unroll
    for (int i = 0; i < PER_LANE; ++i) {
      if (i >= used) break;
      if (e.id[i] >= a.in.vocab && a.in.out_of_range) atomicOr(a.in.out_of_range, 1);
      if (e.id[i] < 0 || e.id[i] >= a.in.vocab) { e.id[i] = -1; e.t[i] = -INFINITY; }
      if (e.id[i] >= 0) e.x[i] = to_f(x[e.id[i]]);
    }
  };
  auto prepare = [&](const Entries& e, Weights& w, Lesson& l) {
    float mt = -INFINITY, most = -INFINITY;
    bool some = false;
#pragma unroll
    for (int i = 0; i < PER_LANE; ++i) {
      if (i >= used) break;
      l.id[lane + 32 * i] = e.id[i];
      mt = fmaxf(mt, e.t[i]);
      most = fmaxf(most, e.x[i]);
      some = some || !(e.t[i] == -INFINITY);
    }
    mt = a.rest ? 0.f : warp_most(mt);
    const float by = a.rest ? 1.f : g.inv_t;
    double mass = 0.0;                                   // of which the rest is what lacks of 1
    w.twins = false;
    w.first = 0;
    int claim[PER_LANE];
#pragma unroll
    for (int i = 0; i < PER_LANE; ++i) {
      claim[i] = -1;
      w.q[i] = 0.f;
      if (i >= used) continue;
      const double v = e.t[i] == -INFINITY ? 0.0 : a.rest ? exp((double)e.t[i]) : (double)expf((e.t[i] - mt) * by);
      w.q[i] = (float)v;
      mass += v;
      if (e.id[i] < 0) continue;
      // Does a token stand in two entries?  Each claims a place by its id.
      unsigned at = (unsigned)e.id[i] * 2654435761u >> 23;
      int had;
      while ((had = atomicCAS(&claims[at], 0, e.id[i] + 1)) != 0 && had != e.id[i] + 1) at = (at + 1) % CLAIMS;
      if (had == 0) claim[i] = (int)at;
      else w.twins = true;
      w.first |= 1u << i;
    }
    __syncwarp();                                        // the claims are made before any is cleared, l.id is written before it is searched
    for (int o = 16; o > 0; o >>= 1) mass += __shfl_xor_sync(0xffffffffu, mass, o);
    const float scale = a.rest ? 1.f : 1.f / (float)mass;
    w.mass = mass;
#pragma unroll
    for (int i = 0; i < PER_LANE; ++i) {
      if (i >= used) break;
      if (claim[i] >= 0) claims[claim[i]] = 0;
      w.q[i] *= scale;
      w.lq[i] = (e.t[i] - mt) * by;
    }
    w.twins = __any_sync(0xffffffffu, w.twins);          // then the first entry stands for the token
    if (w.twins)
      for (int j = 0; j < a.k; ++j)
#pragma unroll
        for (int i = 0; i < PER_LANE; ++i)
          if (j < lane + 32 * i && l.id[j] == e.id[i]) w.first &= ~(1u << i);
    float student = 0.f;
    if (a.rest) {
      most = warp_most(most);
      const Ref rl(most, g);
#pragma unroll
      for (int i = 0; i < PER_LANE; ++i) {
        if (i >= used) break;
        student += (w.first >> i & 1) && e.x[i] != -INFINITY ? ex2(rl.y(e.x[i])) : 0.f;
      }
      student = warp_sum(student);
    }
    some = __any_sync(0xffffffffu, some);
    if (lane == 0) {
      l.most = most;
      l.student = student;
      l.qr = a.rest && 1.0 - mass > SMALLEST_REST ? (float)(1.0 - mass) : 0.f;
      l.Q = a.rest ? (l.qr > 0.f ? 1.f : (float)mass) : mass == mass ? 1.f : (float)mass;
      l.any = some;
    }
    __syncwarp();
  };
  auto beyond = [&](const Piece<T, NT, B>& p) { return a.in.vocab - (a.in.vocab - p.head) % N; };   // from here on in no vector
  auto patch = [&](const Piece<T, NT, B>& p, const Entries& e) {
    await<NT>(LANDED);
    const int end = beyond(p);
#pragma unroll
    for (int i = 0; i < PER_LANE; ++i) {
      const int id = e.id[i], at = id - p.head - p.first * N;
      if (i >= used) break;
      if (id < 0) continue;
      if (at >= 0 && at < p.count * N) ((T*)buf)[at] = from_f<T>(-INFINITY);
      else if (rank == 0 && id < p.head) edges[id] = -INFINITY;
      else if (rank == 0 && id >= end) edges[p.head + id - end] = -INFINITY;
    }
    arrive<NT>(PATCHED);
  };

  Entries now, later;
  Weights w;
  for (int i = lane; i < CLAIMS; i += 32) claims[i] = 0;
#pragma unroll
  for (int i = 0; i < PER_LANE; ++i) lessons[0].id[lane + 32 * i] = lessons[1].id[lane + 32 * i] = -1;
  __syncwarp();
  read(me.row, now);
  look(p.x, now);
  read(me.row + me.groups, later);
  prepare(now, w, lessons[0]);
  cluster_started<CL>();
  if (a.rest) patch(p, now);
  for (long long r = me.row; r < rows; r += me.groups, turn ^= 1) {
    const Lesson& l = lessons[turn];
    const bool has_next = r + me.groups < rows;
    const Piece<T, NT, B> next(a.in, has_next ? r + me.groups : r, rank, g);
    const float dl = a.dloss ? a.dloss[r] : 1.f;
    Entries coming;
    Weights next_w;
    hand_over<NT, CL>();
    if (has_next) {                                      // while the others sum the row
      look(next.x, later);
      read(r + 2 * me.groups, coming);
      prepare(later, next_w, lessons[turn ^ 1]);
    }
    take_up<NT, CL>();
    Sums o = take_parts<NT, false, CL, false>(ex.part[turn][0], g);
    if (Ref(o.m, g).far) {
      sync_row<CL>();
      o = take_parts<NT, false, CL, true>(ex.part[turn][1], g);
    }
    if (!a.dx && a.rest && has_next) patch(next, later);
    const Weighed s(o, l, a.rest, g);
    if (a.loss && rank == 0) {
      // sum q ((lq - y ln 2) + (log S - log mass)): what the logarithms are large in they share with one another
      float part = 0.f;
#pragma unroll
      for (int i = 0; i < PER_LANE; ++i) {
        if (i >= used) break;
        if (now.id[i] >= 0 && !(w.q[i] == 0.f)) part += s.ref.above(w.q[i], w.lq[i], now.x[i]);
      }
      part = warp_sum(part);
      // A logarithm in 64 bits per lane, all at once: of S, of the others' sum, of the listed ones', of the rest, of the teacher's sum.
      const double LN2D = 0.693147180559945309417;
      const double mine = log(lane == 0 ? (double)s.S : lane == 1 ? (double)o.s : lane == 2 ? (double)l.student : lane == 3 ? (double)l.qr : w.mass);
      auto log_of = [&](int i) { return __shfl_sync(0xffffffffu, mine, i); };
      double logs = log_of(0), loss;
      if (a.rest) {
        const Ref rl(l.most, g);
        const double log_o = log_of(1), log_l = log_of(2), log_q = log_of(3);
        double logr;                                       // log p_r
        if (s.ref.far || s.ro.far || rl.far || o.s == 0.f || l.student == 0.f) {
          logr = o.s == 0.f ? -(double)INFINITY : s.apart(s.ro) * LN2D + log_o - logs;
        } else {
          // both from one ratio of the listed to the others, whose rounding they then share: it enters the loss by p_r - q_r only
          const float up = rl.rho - s.ro.rho;
          const float u = l.student / o.s * ex2(up), v = o.s / l.student * ex2(-up);
          const double lr = log_o + s.apart(s.ro) * LN2D;
          logs = u <= 1.f ? lr + (double)log1pf(u) : log_l + s.apart(rl) * LN2D + (double)log1pf(v);
          logr = u <= 1.f ? -(double)log1pf(u) : lr - logs;
        }
        loss = (double)part + w.mass * logs;
        if (l.qr > 0.f) loss += (double)l.qr * (log_q - logr);
      } else {
        loss = (double)part + (logs - log_of(4));
      }
      if (s.S == 0.f) loss = (double)INFINITY;
      if (lane == 0) a.loss[r] = l.any ? (float)((double)a.scale * loss) : 0.f;
    }
    if (a.dx) {
      await<NT>(WRITTEN);
      if (a.rest && has_next) patch(next, later);
      if (l.any && dl != 0.f) {
        T* dx = (T*)a.dx + r * a.ld_out;
        const float f = dl * a.scale * g.inv_t, share = l.Q / s.S;
        const int end = beyond(p);
#pragma unroll
        for (int i = 0; i < PER_LANE; ++i) {
          if (i >= used) break;
          const int id = now.id[i], at = id - p.head - p.first * N;
          float q = w.q[i];
          if (w.twins) {                                 // the sum over the entries of the token
            q = 0.f;
#pragma unroll
            for (int b = 0; b < PER_LANE; ++b)
              for (int j = 0; j < 32; ++j) {
                const float other = __shfl_sync(0xffffffffu, w.q[b], j);
                if (32 * b + j < a.k && l.id[32 * b + j] == id) q += other;
              }
          }
          const bool here = (at >= 0 && at < p.count * N) || (rank == 0 && (id < p.head || id >= end));
          if (!(w.first >> i & 1) || !here) continue;
          const float e = now.x[i] == -INFINITY ? 0.f : ex2(s.ref.y(now.x[i]));
          dx[id] = from_f<T>(s.S == 0.f ? 0.f : fmaf(e, share, -q) * f);
        }
      }
    }
    p = next;
    now = later;
    later = coming;
    w = next_w;
  }
}

// ---------------------------------------------------------------------------------------------- launches
// Vectors of a staying piece at most: 65 KB, so that three blocks share an SM.  Pieces to 4400 would fit three times too: with that limit
// bf16 rows of 34000 take 101 us instead of 111 (gradient) and 119 instead of 142 (distillation), but those of 100300 110 instead of
// 105 and fp32 rows of 16700 211 instead of 191.
constexpr int PIECE = 4160;
constexpr int SMS = 148;                      // of a B200, and not asked of the device: a row's cut, and with it its bits, goes by sizes alone

struct Plan {
  Geometry g;
  int rows, threads;
  size_t smem;
};
// Blocks of `threads` (and more_threads); stay: rows stay in shared memory as a whole, otherwise it takes `smem` bytes.
Plan plan_rows(const LogitsIn& in, int elem_bytes, int threads, int batch, bool stay, bool top, size_t smem, size_t smem_cluster, int more_threads = 0) {
  Plan p{};
  const int N = 16 / elem_bytes, all = std::max(1, in.vocab / N);
  int c = stay ? std::min(MAX_CLUSTER, (all + PIECE - 1) / PIECE) : 1;
  // More blocks for rows too few for the device, where a piece is still worth the exchange: four to an SM of pieces of 64 KB,
  // one to an SM of 16 KB where no alternatives have to be joined.
  auto split = [&](int blocks, int vectors) {
    while (threads > FEW && 2 * c <= MAX_CLUSTER && (long long)in.rows * c < blocks && all / (2 * c) >= vectors) c *= 2;
  };
  split(4 * SMS, 4096);
  if (!top) split(SMS, 1024);
  const int per = (all + c - 1) / c;
  p.rows = in.rows;
  p.threads = threads + more_threads;
  p.smem = (stay ? (size_t)per * 16 : smem) + (c > 1 ? smem_cluster : 0);
  const double cc = 1.4426950408889634 / (double)in.temperature;
  p.g = Geometry{(float)cc, (float)(1.0 / (double)in.temperature), (float)(LOWEST / cc), (float)(SLACK / cc), c, per,
                 (per + batch * threads - 1) / (batch * threads), 0};
  while (batch / 4 * p.g.batches > ENTRIES << p.g.shift) ++p.g.shift;
  return p;
}

// What a kernel needs to know of the device, asked for once: the limit of its shared memory, and how many clusters run at
// a time (blocks beyond would start on their rows when the others are through), for the last size of each cluster.
struct Residency {
  SmemLimit limit;
  std::atomic<unsigned long long> seen[MAX_CLUSTER + 1];
  template <typename... KArgs>
  cudaError_t of(void (*kernel)(KArgs...), const Plan& p, int* clusters) {
    cudaError_t e = limit.raise((const void*)kernel, 160 * 1024);
    if (e != cudaSuccess) return e;
    int dev = 0;
    if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
    const unsigned long long key = ((unsigned long long)(dev + 1) << 40 | p.smem << 16) & ~0xffffull;
    const unsigned long long had = seen[p.g.cluster].load(std::memory_order_relaxed);
    if ((had & ~0xffffull) == key) {
      *clusters = (int)(had & 0xffff);
      return cudaSuccess;
    }
    int n = 0;
    if (p.g.cluster > 1) {
      cudaLaunchConfig_t cfg{};
      cudaLaunchAttribute at{};
      at.id = cudaLaunchAttributeClusterDimension;
      at.val.clusterDim.x = (unsigned)p.g.cluster;
      at.val.clusterDim.y = at.val.clusterDim.z = 1;
      cfg.gridDim = dim3((unsigned)p.g.cluster);
      cfg.blockDim = dim3((unsigned)p.threads);
      cfg.dynamicSmemBytes = p.smem;
      cfg.attrs = &at;
      cfg.numAttrs = 1;
      if ((e = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg)) != cudaSuccess) return e;
    } else {
      int sms = 0;
      if ((e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, p.threads, p.smem)) != cudaSuccess) return e;
      if ((e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
      n *= sms;
    }
    n = std::min(std::max(n, 1), 0xffff);
    seen[p.g.cluster].store(key | (unsigned)n, std::memory_order_relaxed);
    *clusters = n;
    return cudaSuccess;
  }
};

// Rows of at most `limit` bytes, enough of them to give every warp of the device one.
bool short_rows(const LogitsIn& in, size_t elem_bytes, size_t limit) { return in.vocab * elem_bytes <= limit && in.rows >= SMS * 8; }

template <typename... KArgs, typename A>
cudaError_t run(void (*kernel)(KArgs...), Residency& residency, const Plan& p, cudaStream_t s, const A& a) {
  int clusters = 0;
  const cudaError_t e = residency.of(kernel, p, &clusters);
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)(std::min(p.rows, clusters) * p.g.cluster));
  return launch_cluster_after(kernel, p.g.cluster, grid, p.threads, p.smem, s, a, p.g);
}

template <typename T, int NT, bool W, bool CL, bool TOP>
cudaError_t run_logprobs(const LogprobsArgs& a, const Plan& p, cudaStream_t s) {
  static Residency residency;
  return run(logprobs_kernel<T, NT, W, CL, TOP>, residency, p, s, a);
}
template <typename T, int NT, bool W, bool TOP>
cudaError_t run_logprobs(const LogprobsArgs& a, cudaStream_t s) {
  typedef TopSpace<NT> Top;
  constexpr int B = batch_of(NT, TOP);
  const size_t ring = SLOTS * B * NT * 16, desk = offsetof(Top, sorted);
  const Plan p = TOP ? plan_rows(a.in, sizeof(T), NT, B, false, true, ring + desk, sizeof(Top) - desk) : plan_rows(a.in, sizeof(T), NT, B, false, false, ring, 0);
  if constexpr (NT == STREAM)
    if (p.g.cluster > 1) return run_logprobs<T, NT, W, true, TOP>(a, p, s);
  return run_logprobs<T, NT, W, false, TOP>(a, p, s);
}
// A warp leaves 64 maxima to find a bound for its alternatives with, which is close for up to half as many: 32 of 2048 bf16 logits in
// 16384 rows take 61 us against 104 with four warps per row, 64 of them 354 against 128.
constexpr int TOP_OF_A_WARP = 32;
template <typename T, bool W>
cudaError_t run_logprobs(const LogprobsArgs& a, cudaStream_t s) {
  if (short_rows(a.in, sizeof(T), 16384) && a.top_k <= TOP_OF_A_WARP) return a.top_k > 0 ? run_logprobs<T, FEW, W, true>(a, s) : run_logprobs<T, FEW, W, false>(a, s);
  return a.top_k > 0 ? run_logprobs<T, STREAM, W, true>(a, s) : run_logprobs<T, STREAM, W, false>(a, s);
}
template <typename T, int NT, bool W, bool CL>
cudaError_t run_bwd(const LogprobsBwdArgs& a, const Plan& p, cudaStream_t s) {
  static Residency residency;
  return run(logprobs_bwd_kernel<T, NT, W, CL>, residency, p, s, a);
}
template <typename T, bool W>
cudaError_t run_bwd(const LogprobsBwdArgs& a, cudaStream_t s) {
  if (short_rows(a.in, sizeof(T), 16384)) return run_bwd<T, FEW, W, false>(a, plan_rows(a.in, sizeof(T), FEW, batch_of(FEW, false), true, false, 0, 0), s);
  const Plan p = plan_rows(a.in, sizeof(T), STAY, batch_of(STAY, false), true, false, 0, 0);
  return p.g.cluster > 1 ? run_bwd<T, STAY, W, true>(a, p, s) : run_bwd<T, STAY, W, false>(a, p, s);
}

template <typename T, int NT, bool CL>
cudaError_t run_distill(const DistillArgs& a, const Plan& p, cudaStream_t s) {
  static Residency residency;
  return run(distill_kernel<T, NT, CL>, residency, p, s, a);
}
template <typename T>
cudaError_t run_distill(const DistillArgs& a, cudaStream_t s) {
  if (short_rows(a.in, sizeof(T), 8192)) return run_distill<T, FEW, false>(a, plan_rows(a.in, sizeof(T), FEW, batch_of(FEW, false), true, false, 0, 0, 32), s);
  const Plan p = plan_rows(a.in, sizeof(T), STAY, batch_of(STAY, false), true, false, 0, 0, 32);
  return p.g.cluster > 1 ? run_distill<T, STAY, true>(a, p, s) : run_distill<T, STAY, false>(a, p, s);
}

}  // namespace

cudaError_t launch_logprobs(const LogprobsArgs& a, bool is_bf16, cudaStream_t s) {
  if (is_bf16) return a.entropy ? run_logprobs<bf16, true>(a, s) : run_logprobs<bf16, false>(a, s);
  return a.entropy ? run_logprobs<float, true>(a, s) : run_logprobs<float, false>(a, s);
}

cudaError_t launch_logprobs_bwd(const LogprobsBwdArgs& a, bool is_bf16, cudaStream_t s) {
  if (is_bf16) return a.dentropy ? run_bwd<bf16, true>(a, s) : run_bwd<bf16, false>(a, s);
  return a.dentropy ? run_bwd<float, true>(a, s) : run_bwd<float, false>(a, s);
}

cudaError_t launch_distill(const DistillArgs& a, bool is_bf16, cudaStream_t s) {
  return is_bf16 ? run_distill<bf16>(a, s) : run_distill<float>(a, s);
}

}  // namespace lp
