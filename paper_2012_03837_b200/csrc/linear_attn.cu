// Linear attention with a decay for each head, heads of 64, bf16 operands, fp32 sums and states.
//
//   S_t = l S_{t-1} + k_t v_t^T   (64 x 64, l = exp(log_decay[head])),   o_t = scale * q_t S_t
//
// Chunked form (prompts, training).  Inside a chunk of 64 tokens with S the state before it,
//   o_i = scale * ( l^(i+1) q_i S + sum_{j<=i} l^(i-j) (q_i . k_j) v_j ),    S' = l^n S + sum_j l^(n-1-j) k_j v_j^T
// so a chunk is four 64 x 64 x 64 products (two of them triangular).  The gradients are the same operator:
//   dq = it on (do, v, k);  with R_s = sum_{t>=s} l^(t-s) scale q_t do_t^T, running backwards in time,
//   dk_s = R_s v_s,  dv_s = R_s^T k_s:  both from one state.
// All powers l^n come from a table that is formed in 64 bits once per block; none is ever divided by, so strong decays
// neither overflow nor lose anything.
//
// Rounding: the operands are bf16; scores, sums and states are fp32.  Where a product needs an fp32 value as an operand
// it is rounded to bf16: the decayed scores, the state as operand of q S, the decayed k.  Each of these errors (2^-9
// relative per term, at random) is of the size of the output's own rounding.  A state that is handed out in fp32 must
// not carry them: there the decayed k is split into two bf16 terms (2^-17) and the state is never rounded itself.
#include "common.cuh"
#include "launch.cuh"

namespace lp {
namespace {

constexpr int C = 64;                            // tokens of a chunk = width of a head
constexpr int THREADS = 128;                     // four warps, 16 rows of the chunk each
constexpr int TILE = C * C;                      // elements of a bf16 tile (8 KB, rows of 128 bytes, 16-byte units swizzled)

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t unit(uint32_t tile, int row, int u) { return tile + row * 128 + ((u ^ (row & 7)) << 4); }
__device__ __forceinline__ void ldsm(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *(uint32_t*)&v;
}
__device__ __forceinline__ float lo_f(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float hi_f(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }

// Fragments of a swizzled tile.  a_frag: rows r0..r0+15, k-step ks.  b_frag: operand B(k, n) = tile[n][k], columns
// n0..n0+15 (two 8-column tiles: r[0..1], r[2..3]).  b_frag_t: B(k, n) = tile[k][n].  a_frag_t: A(m, k) = tile[k][m].
__device__ __forceinline__ void a_frag(uint32_t (&r)[4], uint32_t t, int r0, int ks, int lane) { ldsm(r, unit(t, r0 + (lane & 15), ks * 2 + (lane >> 4))); }
__device__ __forceinline__ void b_frag(uint32_t (&r)[4], uint32_t t, int n0, int ks, int lane) {
  ldsm(r, unit(t, n0 + (lane & 7) + ((lane >> 4) << 3), ks * 2 + ((lane >> 3) & 1)));
}
__device__ __forceinline__ void b_frag_t(uint32_t (&r)[4], uint32_t t, int k0, int np, int lane) {
  ldsm_t(r, unit(t, k0 + (lane & 7) + (((lane >> 3) & 1) << 3), np * 2 + (lane >> 4)));
}
__device__ __forceinline__ void a_frag_t(uint32_t (&r)[4], uint32_t t, int k0, int mu, int lane) {
  ldsm_t(r, unit(t, k0 + (lane & 7) + ((lane >> 4) << 3), mu * 2 + ((lane >> 3) & 1)));
}

__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// 64 token rows of one head into a swizzled tile; rows at or behind n read as zero (nothing is fetched for them).
__device__ __forceinline__ void load_tile(uint32_t tile, const bf16* src, long long ts, int n) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int x = threadIdx.x + i * THREADS, row = x >> 3, u = x & 7;
    const bf16* g = src + (row < n ? (long long)row * ts : 0) + u * 8;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(unit(tile, row, u)), "l"(g), "r"(row < n ? 16 : 0) : "memory");
  }
}

// Powers l^0 .. l^64; l^0 = 1 also for l = 0.
__device__ __forceinline__ void decay_table(float* pw, float log_decay) {
  if (threadIdx.x <= C) pw[threadIdx.x] = threadIdx.x == 0 ? 1.f : (float)exp((double)threadIdx.x * (double)log_decay);
}
__device__ __forceinline__ float decay_pow(float log_decay, long long n) { return n == 0 ? 1.f : (float)exp((double)n * (double)log_decay); }

// The state of a warp: rows 16 w + g (+8), columns 8 j + 2 t (+1), g = lane / 4, t = lane % 4.
__device__ __forceinline__ void state_load(float (&s)[8][4], const float* src, bool transposed, int w, int lane) {
  const int g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 16 * w + g + (e >> 1) * 8, c = 8 * j + 2 * t + (e & 1);
      s[j][e] = src ? src[transposed ? c * C + r : r * C + c] : 0.f;
    }
}
__device__ __forceinline__ void state_store(float* dst, const float (&s)[8][4], int w, int lane) {
  const int g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    *(float2*)(dst + (16 * w + g) * C + 8 * j + 2 * t) = make_float2(s[j][0], s[j][1]);
    *(float2*)(dst + (16 * w + g + 8) * C + 8 * j + 2 * t) = make_float2(s[j][2], s[j][3]);
  }
}
// ... and its bf16 copy, the operand of the next chunk's products.
__device__ __forceinline__ void state_publish(uint32_t tile, const float (&s)[8][4], int w, int lane) {
  const int g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    asm volatile("st.shared.b32 [%0], %1;" ::"r"(unit(tile, 16 * w + g, j) + 4 * t), "r"(pack(s[j][0], s[j][1])) : "memory");
    asm volatile("st.shared.b32 [%0], %1;" ::"r"(unit(tile, 16 * w + g + 8, j) + 4 * t), "r"(pack(s[j][2], s[j][3])) : "memory");
  }
}

// s += (weights . B)^T C over the 16 tokens of step kk: `bt` is the fragment of B^T, cf the fragments of C.
template <bool TWO>
__device__ __forceinline__ void state_mma(float (&s)[8][4], const uint32_t (&bt)[4], const uint32_t (&cf)[4][4], const float (&wt)[4]) {
  uint32_t hi[4], lo[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {                  // registers 0, 1: tokens 2t, 2t+1; registers 2, 3: tokens 2t+8, 2t+9
    const float x0 = lo_f(bt[e]) * wt[(e >> 1) * 2], x1 = hi_f(bt[e]) * wt[(e >> 1) * 2 + 1];
    hi[e] = pack(x0, x1);
    if (TWO) lo[e] = pack(x0 - lo_f(hi[e]), x1 - hi_f(hi[e]));
  }
#pragma unroll
  for (int np = 0; np < 4; ++np) {
    mma(s[2 * np], hi, cf[np][0], cf[np][1]);
    mma(s[2 * np + 1], hi, cf[np][2], cf[np][3]);
    if (TWO) {
      mma(s[2 * np], lo, cf[np][0], cf[np][1]);
      mma(s[2 * np + 1], lo, cf[np][2], cf[np][3]);
    }
  }
}

// A warp's 16 output rows through its own rows of a shared tile (only this warp reads or wrote them), then 16 bytes
// per thread to memory.
__device__ __forceinline__ void store_rows(uint32_t tile, const float (&acc)[8][4], bf16* dst, long long ts, int n, int w, int lane) {
  const int g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    asm volatile("st.shared.b32 [%0], %1;" ::"r"(unit(tile, 16 * w + g, j) + 4 * t), "r"(pack(acc[j][0], acc[j][1])) : "memory");
    asm volatile("st.shared.b32 [%0], %1;" ::"r"(unit(tile, 16 * w + g + 8, j) + 4 * t), "r"(pack(acc[j][2], acc[j][3])) : "memory");
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int x = lane + 32 * i, row = 16 * w + (x >> 3), u = x & 7;
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(unit(tile, row, u)) : "memory");
    if (row < n) *(uint4*)(dst + (long long)row * ts + u * 8) = v;
  }
  __syncwarp();
}

// Tokens [t0, t1) of sequence (b, h) that this block covers; n_tok is the sequence's length.
struct Span { int b, h, seg, t0, t1; };
__device__ __forceinline__ Span span_of(const LinAttnArgs& a, int item) {
  Span s;
  s.seg = item % a.n_seg;
  const int bh = item / a.n_seg;
  s.h = bh % a.H;
  s.b = bh / a.H;
  int len = a.lengths ? min(max(a.lengths[s.b], 0), a.T) : a.T;
  s.t0 = min((long long)s.seg * a.seg_len, (long long)len);
  s.t1 = min((long long)s.t0 + a.seg_len, (long long)len);
  return s;
}
__device__ __forceinline__ const bf16* at(const LinAttnTok& x, const Span& s, long long t) { return x.p + s.b * x.bs + t * x.ts + s.h * C; }
__device__ __forceinline__ bf16* at_w(const LinAttnTok& x, const Span& s, long long t) { return const_cast<bf16*>(at(x, s, t)); }
__device__ __forceinline__ size_t state_at(const Span& s, int H) { return ((size_t)s.b * H + s.h) * TILE; }

// Forward in time: y_i = out_scale ( l^(i+1) a_i S + sum_{j<=i} l^(i-j) (a_i . b_j) c_j ),  S += decayed b c^T.
// With a = q, b = k, c = v the output; with a = do, b = v, c = k (and S transposed) the gradient of q.
template <bool TWO>
__device__ __forceinline__ void scan_forward(const LinAttnArgs& p, const Span& sp, const LinAttnTok& A, const LinAttnTok& B, const LinAttnTok& Cc,
                                             const LinAttnTok& Y, const float* s_in, bool transposed, float* s_out, char* smem) {
  float* pw = (float*)smem;
  const uint32_t tiles = smem_addr(smem + 512), st = tiles + 6 * TILE * 2;   // [2][A, B, C], [2] states
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  decay_table(pw, p.log_decay[sp.h]);
  float s[8][4];
  state_load(s, s_in, transposed, w, lane);
  const int n_chunks = (sp.t1 - sp.t0 + C - 1) / C;
  auto fetch = [&](int ch) {
    const long long tb = sp.t0 + (long long)ch * C;
    const int n = min(C, (int)(sp.t1 - tb));
    const uint32_t buf = tiles + (ch & 1) * 3 * TILE * 2;
    load_tile(buf, at(A, sp, tb), A.ts, n);
    load_tile(buf + TILE * 2, at(B, sp, tb), B.ts, n);
    load_tile(buf + 2 * TILE * 2, at(Cc, sp, tb), Cc.ts, n);
  };
  if (n_chunks > 0) fetch(0);
  cp_commit();
  state_publish(st, s, w, lane);
  for (int ch = 0; ch < n_chunks; ++ch) {
    cp_wait<0>();
    __syncthreads();                             // this chunk's tiles and state are in place; the other buffers are free
    if (ch + 1 < n_chunks) fetch(ch + 1);
    cp_commit();
    const long long tb = sp.t0 + (long long)ch * C;
    const int n = min(C, (int)(sp.t1 - tb));
    const uint32_t ta = tiles + (ch & 1) * 3 * TILE * 2, tbb = ta + TILE * 2, tc = tbb + TILE * 2, ss = st + (ch & 1) * TILE * 2;
    uint32_t af[4][4];
    float acc[8][4] = {};
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      a_frag(af[ks], ta, 16 * w, ks, lane);
#pragma unroll
      for (int np = 0; np < 4; ++np) {
        uint32_t b[4];
        b_frag_t(b, ss, 16 * ks, np, lane);
        mma(acc[2 * np], af[ks], b[0], b[1]);
        mma(acc[2 * np + 1], af[ks], b[2], b[3]);
      }
    }
    const float w0 = pw[16 * w + g + 1] * p.scale, w1 = pw[16 * w + g + 9] * p.scale, ln = pw[n];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      acc[j][0] *= w0; acc[j][1] *= w0; acc[j][2] *= w1; acc[j][3] *= w1;
#pragma unroll
      for (int e = 0; e < 4; ++e) s[j][e] *= ln;
    }
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      uint32_t cf[4][4];
#pragma unroll
      for (int np = 0; np < 4; ++np) b_frag_t(cf[np], tc, 16 * kk, np, lane);
      if (kk <= w) {
        float sc[2][4] = {};
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          uint32_t b[4];
          b_frag(b, tbb, 16 * kk, ks, lane);
          mma(sc[0], af[ks], b[0], b[1]);
          mma(sc[1], af[ks], b[2], b[3]);
        }
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int age = 16 * w + g + (e >> 1) * 8 - (16 * kk + 8 * x + 2 * t + (e & 1));
            sc[x][e] = age >= 0 ? sc[x][e] * (pw[max(age, 0)] * p.scale) : 0.f;
          }
        const uint32_t pf[4] = {pack(sc[0][0], sc[0][1]), pack(sc[0][2], sc[0][3]), pack(sc[1][0], sc[1][1]), pack(sc[1][2], sc[1][3])};
#pragma unroll
        for (int np = 0; np < 4; ++np) {
          mma(acc[2 * np], pf, cf[np][0], cf[np][1]);
          mma(acc[2 * np + 1], pf, cf[np][2], cf[np][3]);
        }
      }
      uint32_t bt[4];
      a_frag_t(bt, tbb, 16 * kk, w, lane);
      float wt[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) wt[e] = pw[max(n - 1 - (16 * kk + 2 * t + (e & 1) + (e >> 1) * 8), 0)];   // rows behind n are zero
      state_mma<TWO>(s, bt, cf, wt);
    }
    state_publish(st + ((ch + 1) & 1) * TILE * 2, s, w, lane);
    store_rows(ta, acc, at_w(Y, sp, tb), Y.ts, n, w, lane);
  }
  if (s_out) state_store(s_out, s, w, lane);
}

// Backwards in time: dk and dv from the state R (rows: k index, columns: v index).
template <bool TWO>
__device__ __forceinline__ void scan_backward(const LinAttnArgs& p, const Span& sp, const float* r_in, float* r_out, char* smem) {
  float* pw = (float*)smem;
  const uint32_t tiles = smem_addr(smem + 512), st = tiles + 8 * TILE * 2;   // [2][q, k, v, do], [2] states
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  decay_table(pw, p.log_decay[sp.h]);
  float s[8][4];
  state_load(s, r_in, false, w, lane);
  const int n_chunks = (sp.t1 - sp.t0 + C - 1) / C;
  auto fetch = [&](int it) {
    const long long tb = sp.t0 + (long long)(n_chunks - 1 - it) * C;
    const int n = min(C, (int)(sp.t1 - tb));
    const uint32_t buf = tiles + (it & 1) * 4 * TILE * 2;
    load_tile(buf, at(p.q, sp, tb), p.q.ts, n);
    load_tile(buf + TILE * 2, at(p.k, sp, tb), p.k.ts, n);
    load_tile(buf + 2 * TILE * 2, at(p.v, sp, tb), p.v.ts, n);
    load_tile(buf + 3 * TILE * 2, at(p.dout, sp, tb), p.dout.ts, n);
  };
  if (n_chunks > 0) fetch(0);
  cp_commit();
  state_publish(st, s, w, lane);
  for (int it = 0; it < n_chunks; ++it) {
    cp_wait<0>();
    __syncthreads();
    if (it + 1 < n_chunks) fetch(it + 1);
    cp_commit();
    const long long tb = sp.t0 + (long long)(n_chunks - 1 - it) * C;
    const int n = min(C, (int)(sp.t1 - tb));
    const uint32_t tq = tiles + (it & 1) * 4 * TILE * 2, tk = tq + TILE * 2, tv = tk + TILE * 2, td = tv + TILE * 2,
                   ss = st + (it & 1) * TILE * 2;
    uint32_t kf[4][4], vf[4][4];
    float dv[8][4] = {}, dk[8][4] = {};
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      a_frag(kf[ks], tk, 16 * w, ks, lane);
      a_frag(vf[ks], tv, 16 * w, ks, lane);
#pragma unroll
      for (int np = 0; np < 4; ++np) {
        uint32_t b[4];
        b_frag_t(b, ss, 16 * ks, np, lane);      // dv: k R
        mma(dv[2 * np], kf[ks], b[0], b[1]);
        mma(dv[2 * np + 1], kf[ks], b[2], b[3]);
        b_frag(b, ss, 16 * np, ks, lane);        // dk: v R^T
        mma(dk[2 * np], vf[ks], b[0], b[1]);
        mma(dk[2 * np + 1], vf[ks], b[2], b[3]);
      }
    }
    const float w0 = pw[max(n - 1 - (16 * w + g), 0)], w1 = pw[max(n - 1 - (16 * w + g + 8), 0)], ln = pw[n];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      dv[j][0] *= w0; dv[j][1] *= w0; dv[j][2] *= w1; dv[j][3] *= w1;
      dk[j][0] *= w0; dk[j][1] *= w0; dk[j][2] *= w1; dk[j][3] *= w1;
#pragma unroll
      for (int e = 0; e < 4; ++e) s[j][e] *= ln;
    }
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      uint32_t df[4][4];
#pragma unroll
      for (int np = 0; np < 4; ++np) b_frag_t(df[np], td, 16 * kk, np, lane);
      if (kk >= w) {
        float s1[2][4] = {}, s2[2][4] = {};
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          uint32_t b[4];
          b_frag(b, tq, 16 * kk, ks, lane);      // k . q
          mma(s1[0], kf[ks], b[0], b[1]);
          mma(s1[1], kf[ks], b[2], b[3]);
          b_frag(b, td, 16 * kk, ks, lane);      // v . do
          mma(s2[0], vf[ks], b[0], b[1]);
          mma(s2[1], vf[ks], b[2], b[3]);
        }
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int age = 16 * kk + 8 * x + 2 * t + (e & 1) - (16 * w + g + (e >> 1) * 8);
            const float f = pw[max(age, 0)] * p.scale;
            s1[x][e] = age >= 0 ? s1[x][e] * f : 0.f;
            s2[x][e] = age >= 0 ? s2[x][e] * f : 0.f;
          }
        const uint32_t p1[4] = {pack(s1[0][0], s1[0][1]), pack(s1[0][2], s1[0][3]), pack(s1[1][0], s1[1][1]), pack(s1[1][2], s1[1][3])};
        const uint32_t p2[4] = {pack(s2[0][0], s2[0][1]), pack(s2[0][2], s2[0][3]), pack(s2[1][0], s2[1][1]), pack(s2[1][2], s2[1][3])};
#pragma unroll
        for (int np = 0; np < 4; ++np) {
          mma(dv[2 * np], p1, df[np][0], df[np][1]);
          mma(dv[2 * np + 1], p1, df[np][2], df[np][3]);
          uint32_t qf[4];
          b_frag_t(qf, tq, 16 * kk, np, lane);
          mma(dk[2 * np], p2, qf[0], qf[1]);
          mma(dk[2 * np + 1], p2, qf[2], qf[3]);
        }
      }
      uint32_t qt[4];
      a_frag_t(qt, tq, 16 * kk, w, lane);
      float wt[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) wt[e] = pw[16 * kk + 2 * t + (e & 1) + (e >> 1) * 8 + 1] * p.scale;   // rows behind n are zero
      state_mma<TWO>(s, qt, df, wt);
    }
    state_publish(st + ((it + 1) & 1) * TILE * 2, s, w, lane);
    store_rows(tk, dk, at_w(p.dk, sp, tb), p.dk.ts, n, w, lane);
    store_rows(tv, dv, at_w(p.dv, sp, tb), p.dv.ts, n, w, lane);
  }
  if (r_out) state_store(r_out, s, w, lane);
}

constexpr int FWD_SMEM = 512 + 8 * TILE * 2;
constexpr int BWD_SMEM = 512 + 10 * TILE * 2;

// TWO: the state leaves the operator in fp32.  With segments the entry states come from the workspace.
template <bool TWO>
__global__ void __launch_bounds__(THREADS) la_forward_kernel(LinAttnArgs p) {
  extern __shared__ __align__(128) char smem[];
  const Span sp = span_of(p, blockIdx.x);
  const size_t so = state_at(sp, p.H);
  const float* in = p.n_seg > 1 ? p.seg_states + ((size_t)blockIdx.x) * TILE : p.state_in ? p.state_in + so : nullptr;
  float* out = p.n_seg > 1 || !p.state_out ? nullptr : p.state_out + so;
  scan_forward<TWO>(p, sp, p.q, p.k, p.v, p.o, in, false, out, smem);
}

// Even blocks: dq, forward in time; odd blocks: dk and dv, backwards in time.
template <bool TWO>
__global__ void __launch_bounds__(THREADS) la_backward_kernel(LinAttnArgs p) {
  extern __shared__ __align__(128) char smem[];
  const int item = blockIdx.x >> 1;
  const Span sp = span_of(p, item);
  const size_t so = state_at(sp, p.H);
  if (blockIdx.x & 1) {
    const float* in = p.n_seg > 1 ? p.seg_grads + (size_t)item * TILE : p.dstate_out ? p.dstate_out + so : nullptr;
    float* out = p.n_seg > 1 || !p.dstate_in ? nullptr : p.dstate_in + so;
    scan_backward<TWO>(p, sp, in, out, smem);
  } else {
    const float* in = p.n_seg > 1 ? p.seg_states + (size_t)item * TILE : p.state_in ? p.state_in + so : nullptr;
    scan_forward<false>(p, sp, p.dout, p.v, p.k, p.dq, in, true, nullptr, smem);
  }
}

// The state a segment leaves when it starts from zero: sum_j l^(end-1-j) b_j c_j^T, or backwards in time
// sum_j l^(j+1) scale b_j c_j^T (reverse).
template <bool TWO>
__device__ __forceinline__ void segment_state(const LinAttnArgs& p, const Span& sp, const LinAttnTok& B, const LinAttnTok& Cc, bool reverse,
                                              float* out, char* smem) {
  float* pw = (float*)smem;
  const uint32_t tiles = smem_addr(smem + 512);
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, t = lane & 3;
  decay_table(pw, p.log_decay[sp.h]);
  float s[8][4] = {};
  const int n_chunks = (sp.t1 - sp.t0 + C - 1) / C;
  auto fetch = [&](int it) {
    const long long tb = sp.t0 + (long long)(reverse ? n_chunks - 1 - it : it) * C;
    const int n = min(C, (int)(sp.t1 - tb));
    const uint32_t buf = tiles + (it % 3) * 2 * TILE * 2;
    load_tile(buf, at(B, sp, tb), B.ts, n);
    load_tile(buf + TILE * 2, at(Cc, sp, tb), Cc.ts, n);
  };
  if (n_chunks > 0) fetch(0);
  cp_commit();
  if (n_chunks > 1) fetch(1);
  cp_commit();
  for (int it = 0; it < n_chunks; ++it) {
    cp_wait<1>();
    __syncthreads();
    if (it + 2 < n_chunks) fetch(it + 2);
    cp_commit();
    const long long tb = sp.t0 + (long long)(reverse ? n_chunks - 1 - it : it) * C;
    const int n = min(C, (int)(sp.t1 - tb));
    const uint32_t tbb = tiles + (it % 3) * 2 * TILE * 2, tc = tbb + TILE * 2;
    const float ln = pw[n], f = reverse ? p.scale : 1.f;
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[j][e] *= ln;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      uint32_t cf[4][4], bt[4];
#pragma unroll
      for (int np = 0; np < 4; ++np) b_frag_t(cf[np], tc, 16 * kk, np, lane);
      a_frag_t(bt, tbb, 16 * kk, w, lane);
      float wt[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = 16 * kk + 2 * t + (e & 1) + (e >> 1) * 8;
        wt[e] = pw[reverse ? j + 1 : max(n - 1 - j, 0)] * f;
      }
      state_mma<TWO>(s, bt, cf, wt);
    }
  }
  state_store(out, s, w, lane);
}
constexpr int SEG_SMEM = 512 + 6 * TILE * 2;

// blockIdx.y 0: states of k v^T; 1: gradients' states of q do^T.
template <bool TWO>
__global__ void __launch_bounds__(THREADS) la_segment_kernel(LinAttnArgs p) {
  extern __shared__ __align__(128) char smem[];
  const Span sp = span_of(p, blockIdx.x);
  if (blockIdx.y == 0) segment_state<TWO>(p, sp, p.k, p.v, false, p.seg_states + (size_t)blockIdx.x * TILE, smem);
  else segment_state<TWO>(p, sp, p.q, p.dout, true, p.seg_grads + (size_t)blockIdx.x * TILE, smem);
}

// Turns every segment's own state into the state at its entry, and forms the last state.
__global__ void __launch_bounds__(256) la_join_kernel(LinAttnArgs p) {
  const bool reverse = blockIdx.y != 0;
  const int bh = blockIdx.x, h = bh % p.H, b = bh / p.H, len = p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T;
  float* seg = (reverse ? p.seg_grads : p.seg_states) + (size_t)bh * p.n_seg * TILE;
  const float* in = reverse ? p.dstate_out : p.state_in;
  float* out = reverse ? p.dstate_in : p.state_out;
  const float lg = p.log_decay[h];
  const int e = (blockIdx.z * blockDim.x + threadIdx.x) * 4;
  float4 run = in ? *(const float4*)(in + (size_t)bh * TILE + e) : make_float4(0.f, 0.f, 0.f, 0.f);
  const float lfull = decay_pow(lg, p.seg_len);
  for (int i = 0; i < p.n_seg; ++i) {
    const int sidx = reverse ? p.n_seg - 1 - i : i;
    const int n = (int)min(max((long long)len - (long long)sidx * p.seg_len, 0LL), (long long)p.seg_len);
    const float l = n == p.seg_len ? lfull : decay_pow(lg, n);
    float4* at = (float4*)(seg + (size_t)sidx * TILE + e);
    const float4 own = *at;
    *at = run;
    run.x = fmaf(l, run.x, own.x); run.y = fmaf(l, run.y, own.y); run.z = fmaf(l, run.z, own.z); run.w = fmaf(l, run.w, own.w);
  }
  if (out) *(float4*)(out + (size_t)bh * TILE + e) = run;
}

// One token: a block per sequence and head.  The state is read and written once (32 KB), all in fp32.
__global__ void __launch_bounds__(256) la_step_kernel(LinAttnArgs p) {
  const int h = blockIdx.x % p.H, b = blockIdx.x / p.H, tid = threadIdx.x;
  const float* in = p.state_in ? p.state_in + (size_t)blockIdx.x * TILE : nullptr;
  float* out = p.state_out ? p.state_out + (size_t)blockIdx.x * TILE : nullptr;
  const bool live = !p.lengths || p.lengths[b] > 0;
  const int c4 = (tid & 15) * 4, r0 = tid >> 4;
  float4 s[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) s[i] = in ? *(const float4*)(in + (r0 + 16 * i) * C + c4) : make_float4(0.f, 0.f, 0.f, 0.f);
  if (!live) {
    if (out && out != in)
#pragma unroll
      for (int i = 0; i < 4; ++i) *(float4*)(out + (r0 + 16 * i) * C + c4) = s[i];
    return;
  }
  const bf16* q = p.q.p + b * p.q.bs + h * C;
  const bf16* k = p.k.p + b * p.k.bs + h * C;
  const uint2 vv = *(const uint2*)(p.v.p + b * p.v.bs + h * C + c4);
  const float l = decay_pow(p.log_decay[h], 1);
  const float4 v = make_float4(lo_f(vv.x), hi_f(vv.x), lo_f(vv.y), hi_f(vv.y));
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float kr = to_f(k[r0 + 16 * i]), qr = to_f(q[r0 + 16 * i]);
    s[i].x = fmaf(l, s[i].x, kr * v.x); s[i].y = fmaf(l, s[i].y, kr * v.y); s[i].z = fmaf(l, s[i].z, kr * v.z); s[i].w = fmaf(l, s[i].w, kr * v.w);
    if (out) *(float4*)(out + (r0 + 16 * i) * C + c4) = s[i];
    o.x = fmaf(qr, s[i].x, o.x); o.y = fmaf(qr, s[i].y, o.y); o.z = fmaf(qr, s[i].z, o.z); o.w = fmaf(qr, s[i].w, o.w);
  }
  __shared__ float4 red[8][16];
  o.x += __shfl_xor_sync(0xffffffffu, o.x, 16); o.y += __shfl_xor_sync(0xffffffffu, o.y, 16);
  o.z += __shfl_xor_sync(0xffffffffu, o.z, 16); o.w += __shfl_xor_sync(0xffffffffu, o.w, 16);
  if ((tid & 31) < 16) red[tid >> 5][tid & 15] = o;
  __syncthreads();
  if (tid < 16) {
    float4 a = red[0][tid];
#pragma unroll
    for (int i = 1; i < 8; ++i) { a.x += red[i][tid].x; a.y += red[i][tid].y; a.z += red[i][tid].z; a.w += red[i][tid].w; }
    *(uint2*)(const_cast<bf16*>(p.o.p) + b * p.o.bs + h * C + c4) =
        make_uint2(pack(a.x * p.scale, a.y * p.scale), pack(a.z * p.scale, a.w * p.scale));
  }
}

// Segments per sequence: enough blocks to fill the GPU (148 SMs), none shorter than four chunks.
void choose_segments(long long bh, int T, int* n_seg, int* seg_len) {
  const int chunks = (T + C - 1) / C;
  long long want = bh >= 296 ? 1 : (444 + bh - 1) / bh;
  want = std::min<long long>(want, std::max(1, chunks / 4));
  const int per = (int)((chunks + want - 1) / want);
  *n_seg = (chunks + per - 1) / per;
  *seg_len = per * C;
}

}  // namespace

size_t linattn_workspace(bool backward, int B, int T, int H) {
  int ns, sl;
  choose_segments((long long)B * H, T, &ns, &sl);
  return ns > 1 ? (size_t)B * H * ns * TILE * sizeof(float) * (backward ? 2 : 1) : 0;
}

cudaError_t launch_linattn_step(const LinAttnArgs& a, cudaStream_t s) {
  return launch_kernel(la_step_kernel, dim3((unsigned)(a.B * a.H)), 256, 0, s, a);
}

cudaError_t launch_linattn(LinAttnArgs a, bool backward, void* workspace, cudaStream_t s) {
  const int bh = a.B * a.H;
  choose_segments(bh, a.T, &a.n_seg, &a.seg_len);
  cudaError_t e;
  const bool two = backward ? a.dstate_in != nullptr : a.state_out != nullptr;
  if (a.n_seg > 1) {
    a.seg_states = (float*)workspace;
    a.seg_grads = a.seg_states + (size_t)bh * a.n_seg * TILE;
    static SmemLimit l1, l2;
    auto seg = two ? la_segment_kernel<true> : la_segment_kernel<false>;
    if ((e = (two ? l1 : l2).raise((const void*)seg, SEG_SMEM)) != cudaSuccess) return e;
    if ((e = launch_kernel(seg, dim3((unsigned)(bh * a.n_seg), backward ? 2 : 1), THREADS, SEG_SMEM, s, a)) != cudaSuccess) return e;
    if ((e = launch_kernel(la_join_kernel, dim3((unsigned)bh, backward ? 2 : 1, 4), 256, 0, s, a)) != cudaSuccess) return e;
  }
  const bool two_main = two && a.n_seg == 1;
  if (backward) {
    static SmemLimit l1, l2;
    auto k = two_main ? la_backward_kernel<true> : la_backward_kernel<false>;
    if ((e = (two_main ? l1 : l2).raise((const void*)k, BWD_SMEM)) != cudaSuccess) return e;
    return launch_kernel(k, dim3((unsigned)(2 * bh * a.n_seg)), THREADS, BWD_SMEM, s, a);
  }
  static SmemLimit l1, l2;
  auto k = two_main ? la_forward_kernel<true> : la_forward_kernel<false>;
  if ((e = (two_main ? l1 : l2).raise((const void*)k, FWD_SMEM)) != cudaSuccess) return e;
  return launch_kernel(k, dim3((unsigned)(bh * a.n_seg)), THREADS, FWD_SMEM, s, a);
}

}  // namespace lp
