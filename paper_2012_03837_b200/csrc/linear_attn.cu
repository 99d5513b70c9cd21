// Linear attention with a decay for each head, heads of 64, bf16 operands, fp32 sums and states.
//
//   S_t = l S_{t-1} + k_t v_t^T   (64 x 64, l = exp(log_decay[head])),   o_t = scale * q_t S_t
//
// Chunked form (prompts, training).  Inside a chunk of 64 tokens with S the state before it,
//   o_i = scale * ( l^(i+1) q_i S + sum_{j<=i} l^(i-j) (q_i . k_j) v_j ),    S' = l^n S + sum_j l^(n-1-j) k_j v_j^T
// so a chunk is four 64 x 64 x 64 products (two of them triangular).  One scan over time does all of it:
//   y_i = decayed a_i S + sum_j l^|i-j| (a_i . b_j) c_j,   S += decayed b_j c_j^T
//   output    forward   a, b, c = q, k, v     S = state              dk   backwards   v, do, q    S = R^T
//   dq        forward             do, v, k    S = state^T            dv   backwards   k, q, do    S = R
// with R_s = sum_{t>=s} l^(t-s) scale q_t do_t^T (+ the gradient of the last state).
// All powers l^n come from a table formed once per block; none is ever divided by, so strong decays neither overflow nor
// lose anything.
//
// Rounding: the operands are bf16; scores, sums and states are fp32.  Where a product needs an fp32 value as an operand:
// the decayed b is split into two bf16 terms (what is left is 2^-17 of a term); the decayed scores and the state as
// operand of a S are rounded once (2^-8 of a term, of the size of the output's own rounding, and at random; in
// sequences of one chunk, where few terms average out, the scores too are split).  A state that is handed out in fp32
// is formed from three terms and summed chunk by chunk in fp32, as exact as fp32 products would be.
//
// What bounds it: per token and head 512 bytes (forward) stand against 4.25 products of 64 x 64 (the triangles, and the two
// terms of b), so the memory's time (82 us for [128, 512, 16 heads]) lies above that of the products on mma.sync (74 us at
// 8 cycles per m16n8k16, measured) only by a little, and neither alone is met: 122 us forward, 0.36 of the memory's rate
// backward ([64, 512, 16]: 178 us; the scans of dq, dk and dv each read three tensors).  Half of the tensor pipe's time is
// used, with three blocks of four warps per SM; the rest are the waits of the chains ldmatrix, mma, scaling, mma.  Four
// blocks (one buffer of tiles, 128 registers) were no faster, eight warps with half of the columns each slower (14.4
// against 12.0 us on [32, 256, 8]).
// The scans of dk and dv in one, for the state they share (five tiles, two blocks per SM, 240 registers): 50 against 52 us on
// [16, 512, 16] and 168 against 177 on [64, 512, 16], but 45 against 40 on [12, 512, 16] and 71 against 51 on [3, 2048, 16].
// On tcgen05 (chunks of 128, accumulators in tensor memory, TMA, eight row warps and two issuing ones, two blocks per
// SM) the same scan was right and slower: 154 / 243 us on the two cases above.  Every chunk is a chain of four short
// products with row work between them; a product of N = 64 and K = 128 took its issuing thread 2000 to 2600 clocks with
// two blocks on the SM, and the tensor pipe was busy for a sixth of the time.
#include <algorithm>

#include "common.cuh"
#include "launch.cuh"

namespace lp {
namespace {

// l^n for n >= 0, l = exp(lg), l^0 = 1 also for l = 0.  n lg is formed as a product and its rounding error, so that
// the error of the result stays that of one expf.  A power of 0 takes no correction: of an n lg beyond fp32's range the
// rounding error is infinite, of lg = -infinity it is no number.
__device__ __forceinline__ float decay_pow(float lg, float n) {
  if (n == 0.f) return 1.f;
  const float x = n * lg, r = fmaf(n, lg, -x), e = expf(x);
  return e > 0.f ? fmaf(e, r, e) : e;
}

// Tokens [t0, t1) of sequence (b, h) that a block covers.
struct Span { int b, h, t0, t1; };
__device__ __forceinline__ Span span_of(const LinAttnArgs& a, int item) {
  Span s;
  const int seg = item % a.n_seg, bh = item / a.n_seg;
  s.h = bh % a.H;
  s.b = bh / a.H;
  const int len = a.lengths ? min(max(a.lengths[s.b], 0), a.T) : a.T;
  s.t0 = (int)min((long long)seg * a.seg_len, (long long)len);
  s.t1 = (int)min((long long)s.t0 + a.seg_len, (long long)len);
  return s;
}
__device__ __forceinline__ const bf16* at(const LinAttnTok& x, const Span& s, long long t) { return x.p + s.b * x.bs + t * x.ts + s.h * 64; }

__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *(uint32_t*)&v;
}
__device__ __forceinline__ float lo_f(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float hi_f(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
constexpr int C = 64;                            // tokens of a chunk = width of a head
constexpr int TILE = C * C;                      // elements of a state
// Tiles in shared memory are 64 rows of 64 bf16, 144 bytes apart: the 16-byte units of eight consecutive rows lie in eight
// different groups of banks, and every address of a fragment is one register plus a constant.
constexpr int PITCH = 144;
constexpr int TILE_B = C * PITCH;
constexpr int TAB = 1280;                        // bytes of the tables of powers

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void ldsm(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void stsm(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// The same with zeros in place of the accumulator.
__device__ __forceinline__ void mma0(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
// Two products (or sums) at a time.
__device__ __forceinline__ void mul2(float& x, float& y, float a, float b) {
  asm("{\n\t.reg .b64 u, v;\n\tmov.b64 u, {%0, %1};\n\tmov.b64 v, {%2, %3};\n\tmul.rn.f32x2 u, u, v;\n\tmov.b64 {%0, %1}, u;\n\t}"
      : "+f"(x), "+f"(y) : "f"(a), "f"(b));
}
__device__ __forceinline__ void sub2(float& x, float& y, float a, float b) {
  asm("{\n\t.reg .b64 u, v, m;\n\tmov.b64 u, {%0, %1};\n\tmov.b64 v, {%2, %3};\n\tmov.b64 m, {%4, %4};\n\tfma.rn.f32x2 u, v, m, u;\n\tmov.b64 {%0, %1}, u;\n\t}"
      : "+f"(x), "+f"(y) : "f"(a), "f"(b), "f"(-1.f));
}
// The bf16 pair nearest to (x, y); x and y become what is left.
__device__ __forceinline__ uint32_t split(float& x, float& y) {
  const uint32_t h = pack(x, y);
  sub2(x, y, lo_f(h), hi_f(h));
  return h;
}

// What a lane adds to a tile's address.  lane_rows: rows lane % 16, unit lane / 16 -- ldsm gives the A fragment of 16 rows
// and 16 columns, ldsm_t the B fragments B(k, n) = tile[k][n] of 16 k and 16 n.  lane_cols: rows and units the other way
// round -- ldsm gives B(k, n) = tile[n][k], ldsm_t the A fragment A(m, k) = tile[k][m].
__device__ __forceinline__ uint32_t lane_rows(int lane) { return (lane & 15) * PITCH + (lane >> 4) * 16; }
__device__ __forceinline__ uint32_t lane_cols(int lane) { return ((lane & 7) + ((lane >> 4) << 3)) * PITCH + ((lane >> 3) & 1) * 16; }
// A warp's 16 x 64 accumulators as bf16 rows of a tile; at: address of the first row plus lane_rows.
__device__ __forceinline__ void put_rows(uint32_t at, const float (&x)[8][4]) {
#pragma unroll
  for (int j = 0; j < 8; j += 2)
    stsm(at + j * 16, pack(x[j][0], x[j][1]), pack(x[j][2], x[j][3]), pack(x[j + 1][0], x[j + 1][1]), pack(x[j + 1][2], x[j + 1][3]));
}

__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// 64 token rows into a tile, by 128 threads; rows at or behind n read as zero (nothing is fetched for them).
__device__ __forceinline__ void load_tile(uint32_t tile, const bf16* src, long long ts, int n) {
  constexpr int STEP = 16;                       // rows of one round
  const int row = threadIdx.x >> 3, u = threadIdx.x & 7;
  const uint32_t d = tile + row * PITCH + u * 16;
  const bf16* g = src + row * ts + u * 8;
  if (n == C) {
#pragma unroll
    for (int i = 0; i < C / STEP; ++i)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d + i * STEP * PITCH), "l"(g + i * STEP * ts) : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < C / STEP; ++i) {
      const bool in = row + i * STEP < n;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d + i * STEP * PITCH), "l"(in ? g + i * STEP * ts : src), "r"(in ? 16 : 0) : "memory");
    }
  }
}

// pw[n] = l^n and sc[n] = scale * l^n for 0 <= n <= 64; 0 for -64 <= n < 0 (tokens that do not exist, or are not seen)
__device__ __forceinline__ void decay_tables(float* pw, float* sc, float lg, float scale) {
  const int x = threadIdx.x;
  if (x < C) pw[x - C] = sc[x - C] = 0.f;
  if (x <= C) {
    const float p = decay_pow(lg, (float)x);
    pw[x] = p;
    sc[x] = p * scale;
  }
}

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

// d += (weights . B)^T C over the 16 tokens of a step: `bt` is the fragment of B^T, cf the fragments of C.  The decayed
// b goes in as TERMS bf16 terms, the smallest first.
template <int TERMS>
__device__ __forceinline__ void state_mma(float (&d)[8][4], const uint32_t (&bt)[4], const uint32_t (&cf)[4][4], const float (&wt)[4]) {
  uint32_t term[TERMS][4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {                  // registers 0, 1: tokens 2t, 2t+1; registers 2, 3: tokens 2t+8, 2t+9
    float x = lo_f(bt[e]), y = hi_f(bt[e]);
    mul2(x, y, wt[(e >> 1) * 2], wt[(e >> 1) * 2 + 1]);
#pragma unroll
    for (int k = 0; k + 1 < TERMS; ++k) term[k][e] = split(x, y);
    term[TERMS - 1][e] = pack(x, y);
  }
#pragma unroll
  for (int k = TERMS - 1; k >= 0; --k)
#pragma unroll
    for (int np = 0; np < 4; ++np) {
      mma(d[2 * np], term[k], cf[np][0], cf[np][1]);
      mma(d[2 * np + 1], term[k], cf[np][2], cf[np][3]);
    }
}

// The scan of a sequence of at most one chunk (see the head of the file): four warps, 16 rows of y and of the state each.
// TERMS: bf16 terms of the decayed b.
template <int TERMS, bool REV>
__device__ __forceinline__ void scan_short(const LinAttnArgs& p, const Span& sp, const LinAttnTok& A, const LinAttnTok& B, const LinAttnTok& Cc,
                                           const LinAttnTok& Y, const float* s_in, bool transposed, float* s_out, char* smem) {
  float *pw = (float*)smem + 64, *sc = (float*)smem + 193;
  const uint32_t tiles = smem_addr(smem + TAB);  // a, b, c, the state
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, t = lane & 3, n = sp.t1 - sp.t0;
  // Blocks of 16 tokens that exist; the work of others is left out (backward of 38 sequences x 15 heads, 9 tokens 16.7 -> 10.4
  // us, 20 tokens 16.6 -> 13.4, 60 tokens 17.0 -> 18; in the scan of longer sequences it cost 1 to 2 %).
  const int steps = (n + 15) >> 4;
  load_tile(tiles, at(A, sp, sp.t0), A.ts, n);
  load_tile(tiles + TILE_B, at(B, sp, sp.t0), B.ts, n);
  load_tile(tiles + 2 * TILE_B, at(Cc, sp, sp.t0), Cc.ts, n);
  cp_commit();
  decay_tables(pw, sc, p.log_decay[sp.h], p.scale);
  float s[8][4];
  state_load(s, s_in, transposed, w, lane);
  const uint32_t rows = lane_rows(lane), own = rows + w * 16 * PITCH, cols = lane_cols(lane);
  put_rows(tiles + 3 * TILE_B + own, s);
  cp_wait<0>();
  __syncthreads();
  // ages of the pair (row g of this warp, first column of a step): rows lie 8 apart, columns 8 and 1 apart
  const float* wp = REV ? sc - 16 * w - g + 2 * t : sc + 16 * w + g - 2 * t;
  const uint32_t ba = tiles + own, bb = tiles + TILE_B + cols, bt_at = bb + w * 32, bc = tiles + 2 * TILE_B + rows, bs = bc + TILE_B;
  uint32_t af[4][4];
  float acc[8][4] = {};
  if (w < steps) {
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      ldsm(af[ks], ba + ks * 32);
#pragma unroll
      for (int np = 0; np < 4; ++np) {
        uint32_t b[4];
        ldsm_t(b, bs + ks * 16 * PITCH + np * 32);
        mma(acc[2 * np], af[ks], b[0], b[1]);
        mma(acc[2 * np + 1], af[ks], b[2], b[3]);
      }
    }
  }
  // distance of the rows from the incoming state; backwards in time it is the state right behind the chunk
  const int r0 = 16 * w + g;
  const float w0 = REV ? pw[n - 1 - r0] : sc[r0 + 1], w1 = REV ? pw[n - 9 - r0] : sc[r0 + 9], ln = pw[n];
  const float* wj = REV ? sc + 1 + 2 * t : pw + n - 1 - 2 * t;   // weights of the tokens in the state
  float d[8][4] = {};
#pragma unroll
  for (int j = 0; j < 8; ++j) { acc[j][0] *= w0; acc[j][1] *= w0; acc[j][2] *= w1; acc[j][3] *= w1; }
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) {
    if (kk >= steps) break;
    uint32_t cf[4][4];
#pragma unroll
    for (int np = 0; np < 4; ++np) ldsm_t(cf[np], bc + kk * 16 * PITCH + np * 32);
    if (w < steps && (REV ? kk >= w : kk <= w)) {
      float x[2][4] = {};
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        uint32_t b[4];
        ldsm(b, bb + kk * 16 * PITCH + ks * 32);
        mma(x[0], af[ks], b[0], b[1]);
        mma(x[1], af[ks], b[2], b[3]);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[h][e] *= REV ? wp[16 * kk + 8 * h + (e & 1) - (e >> 1) * 8] : wp[(e >> 1) * 8 - (16 * kk + 8 * h + (e & 1))];
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float u = x[e >> 1][(e & 1) * 2], v = x[e >> 1][(e & 1) * 2 + 1];
        hi[e] = split(u, v);
        lo[e] = pack(u, v);
      }
#pragma unroll
      for (int np = 0; np < 4; ++np) {
        mma(acc[2 * np], lo, cf[np][0], cf[np][1]);
        mma(acc[2 * np + 1], lo, cf[np][2], cf[np][3]);
        mma(acc[2 * np], hi, cf[np][0], cf[np][1]);
        mma(acc[2 * np + 1], hi, cf[np][2], cf[np][3]);
      }
    }
    if (s_out) {
      uint32_t bt[4];
      ldsm_t(bt, bt_at + kk * 16 * PITCH);
      float wt[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = 16 * kk + (e & 1) + (e >> 1) * 8;
        wt[e] = REV ? wj[j] : wj[-j];
      }
      state_mma<TERMS>(d, bt, cf, wt);
    }
  }
  if (s_out) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[j][e] = fmaf(ln, s[j][e], d[j][e]);
    state_store(s_out, s, w, lane);
  }
  if (w >= steps) return;
  __syncwarp();
  put_rows(ba, acc);                         // y leaves through this warp's own rows of a: no other warp reads them
  __syncwarp();
  bf16* y = const_cast<bf16*>(at(Y, sp, sp.t0));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = lane + 32 * i, row = 16 * w + (e >> 3), u = e & 7;
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(tiles + row * PITCH + u * 16) : "memory");
    if (row < n) *(uint4*)(y + (long long)row * Y.ts + u * 8) = v;
  }
}
constexpr int SHORT_SMEM = TAB + 4 * TILE_B;

__global__ void __launch_bounds__(128) la_forward_short_kernel(LinAttnArgs p) {
  extern __shared__ __align__(128) char smem[];
  cudaGridDependencySynchronize();
  const Span sp = span_of(p, blockIdx.x);
  const size_t so = (size_t)blockIdx.x * TILE;
  scan_short<3, false>(p, sp, p.q, p.k, p.v, p.o, p.state_in ? p.state_in + so : nullptr, false, p.state_out ? p.state_out + so : nullptr, smem);
}

// Scans of every sequence and head: dq, dk, dv (0, 1, 2), `scans` of them from `first` on.  dk's and dv's both begin with
// dstate_out, each in a block of its own, and dv's ends with dstate_in: where that is the same memory, dv's scans have to
// be a launch behind the other two (run_backward below).
__global__ void __launch_bounds__(128) la_backward_short_kernel(LinAttnArgs p, int first, int scans) {
  extern __shared__ __align__(128) char smem[];
  cudaGridDependencySynchronize();
  const int which = first + blockIdx.x % scans, item = blockIdx.x / scans;
  const Span sp = span_of(p, item);
  const size_t so = (size_t)item * TILE;
  const float* r_in = p.dstate_out ? p.dstate_out + so : nullptr;
  if (which == 0) scan_short<1, false>(p, sp, p.dout, p.v, p.k, p.dq, p.state_in ? p.state_in + so : nullptr, true, nullptr, smem);
  else if (which == 1) scan_short<1, true>(p, sp, p.v, p.dout, p.q, p.dk, r_in, true, nullptr, smem);
  else scan_short<3, true>(p, sp, p.k, p.q, p.dout, p.dv, r_in, false, p.dstate_in ? p.dstate_in + so : nullptr, smem);
}

// Tokens in the order of a scan: the first one, and the distance to the next (negative backwards in time).
struct Run { const bf16* p; long long ts; };
__device__ __forceinline__ Run run_of(const LinAttnTok& x, const Span& sp, bool rev) {
  return rev ? Run{at(x, sp, sp.t1 - 1), -x.ts} : Run{at(x, sp, sp.t0), x.ts};
}

// Fetches a run's tokens tile by tile, in order; 128 threads.  Rows behind the end read as zero.
struct Loader {
  const bf16* g;                                 // this thread's unit of the next tile
  long long step;                                // 16 rows on
  const bf16* any;                               // an address that may be named where nothing is fetched
  int left;                                      // rows from this thread's first one to the end
  __device__ __forceinline__ Loader(const Run& r, int len)
      : g(r.p + (threadIdx.x >> 3) * r.ts + (threadIdx.x & 7) * 8), step(16 * r.ts), any(r.p), left(len - (int)(threadIdx.x >> 3)) {}
  __device__ __forceinline__ void next(uint32_t tile) {
    const uint32_t d = tile + (threadIdx.x >> 3) * PITCH + (threadIdx.x & 7) * 16;
    if (left > 48) {                             // all four rows of this thread
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d + i * 16 * PITCH), "l"(g) : "memory");
        g += step;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool in = 16 * i < left;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d + i * 16 * PITCH), "l"(in ? g : any), "r"(in ? 16 : 0) : "memory");
        g += step;
      }
    }
    left -= C;
  }
};

// The scan of a span (see the head of the file): four warps, 16 rows of y and of the state each.  TERMS: bf16 terms of the
// decayed b.  Backwards in time the tokens are taken in reversed order, so that both directions are one and the same
// code (three copies of it, one per gradient, kept the warps waiting for instructions for a quarter of their time); the
// state is then the one right at the first token, not a step before it, and carries the scale.
template <int TERMS>
__device__ __forceinline__ void scan(int len, const Run A, const Run B, const Run Cc, const Run Y, bool rev, float lg, float scale, const float* s_in,
                                     bool transposed, float* s_out, char* smem) {
  constexpr int BUF = 4 * TILE_B;                // two buffers of a, b, c and the state
  float *pw = (float*)smem + 64, *sc = (float*)smem + 193;
  const uint32_t tiles = smem_addr(smem + TAB);
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int n_chunks = (len + C - 1) / C;
  Loader la(A, len), lb(B, len), lc(Cc, len);
  auto fetch = [&](uint32_t buf) {
    la.next(buf);
    lb.next(buf + TILE_B);
    lc.next(buf + 2 * TILE_B);
  };
  if (n_chunks > 0) fetch(tiles);
  cp_commit();
  decay_tables(pw, sc, lg, scale);
  float s[8][4];
  state_load(s, s_in, transposed, w, lane);
  const uint32_t rows = lane_rows(lane), own = rows + w * 16 * PITCH, cols = lane_cols(lane);
  put_rows(tiles + 3 * TILE_B + own, s);
  const float* from_state = (rev ? pw : sc + 1) + 16 * w + g;            // weights of the rows' products with the state
  bf16* y = const_cast<bf16*>(Y.p) + (16 * w + (lane >> 3)) * Y.ts + (lane & 7) * 8;
  const uint32_t y_at = (16 * w + (lane >> 3)) * PITCH + (lane & 7) * 16;
  for (int it = 0; it < n_chunks; ++it) {
    const uint32_t buf = tiles + (it & 1) * BUF, other = tiles + ((it & 1) ^ 1) * BUF;
    cp_wait<0>();
    __syncthreads();                             // this chunk's tiles and state are in place; the other buffer is free
    if (it + 1 < n_chunks) fetch(other);
    cp_commit();
    const int n = min(C, len - it * C);
    const uint32_t ba = buf + own, bs = buf + 3 * TILE_B + rows;
    uint32_t af[4][4];
    float acc[8][4];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      ldsm(af[ks], ba + ks * 32);
#pragma unroll
      for (int np = 0; np < 4; ++np) {
        uint32_t b[4];
        ldsm_t(b, bs + ks * 16 * PITCH + np * 32);
        if (ks == 0) {
          mma0(acc[2 * np], af[ks], b[0], b[1]);
          mma0(acc[2 * np + 1], af[ks], b[2], b[3]);
        } else {
          mma(acc[2 * np], af[ks], b[0], b[1]);
          mma(acc[2 * np + 1], af[ks], b[2], b[3]);
        }
      }
    }
    const float w0 = from_state[0], w1 = from_state[8], ln = pw[n];
    float d[TERMS == 3 ? 8 : 1][4] = {};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      mul2(acc[j][0], acc[j][1], w0, w0);
      mul2(acc[j][2], acc[j][3], w1, w1);
      if (TERMS < 3) {
        mul2(s[j][0], s[j][1], ln, ln);
        mul2(s[j][2], s[j][3], ln, ln);
      }
    }
    uint32_t bb = buf + TILE_B + cols, bc = buf + 2 * TILE_B + rows;
    const float* wp = sc + 16 * w + g - 2 * t;   // ages of the pair (row g of this warp, column 2t of a step): rows lie 8 apart
    const float* wj = (rev ? sc + n : pw + n - 1) - 2 * t;               // weights of the tokens in the state
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      uint32_t cf[4][4], bt[4];
      ldsm_t(bt, bb + w * 32);
#pragma unroll
      for (int np = 0; np < 4; ++np) ldsm_t(cf[np], bc + np * 32);
      const float wt[4] = {wj[0], wj[-1], wj[-8], wj[-9]};
      // The state's products stand in both branches: beside the scores' they fill the waits of that chain.
      if (kk <= w) {
        float x[2][4];
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          uint32_t b[4];
          ldsm(b, bb + ks * 32);
          if (ks == 0) {
            mma0(x[0], af[ks], b[0], b[1]);
            mma0(x[1], af[ks], b[2], b[3]);
          } else {
            mma(x[0], af[ks], b[0], b[1]);
            mma(x[1], af[ks], b[2], b[3]);
          }
        }
        if constexpr (TERMS == 3) state_mma<TERMS>(d, bt, cf, wt);
        else state_mma<TERMS>(s, bt, cf, wt);
        uint32_t pf[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int up = (e & 1) * 8, left = (e >> 1) * 8;
          float u = x[e >> 1][(e & 1) * 2], v = x[e >> 1][(e & 1) * 2 + 1];
          mul2(u, v, wp[up - left], wp[up - left - 1]);
          pf[e] = pack(u, v);
        }
#pragma unroll
        for (int np = 0; np < 4; ++np) {
          mma(acc[2 * np], pf, cf[np][0], cf[np][1]);
          mma(acc[2 * np + 1], pf, cf[np][2], cf[np][3]);
        }
      } else {
        if constexpr (TERMS == 3) state_mma<TERMS>(d, bt, cf, wt);
        else state_mma<TERMS>(s, bt, cf, wt);
      }
      bb += 16 * PITCH;
      bc += 16 * PITCH;
      wp -= 16;
      wj -= 16;
    }
    if constexpr (TERMS == 3) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[j][e] = fmaf(ln, s[j][e], d[j][e]);
    }
    put_rows(other + 3 * TILE_B + own, s);
    // y leaves through this warp's own rows of a: no other warp reads them
    __syncwarp();
    put_rows(ba, acc);
    __syncwarp();
    const int left = n - 16 * w - (lane >> 3);   // rows 4 i of this warp with 4 i < left exist
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint4 v;
      asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(buf + y_at + i * 4 * PITCH) : "memory");
      if (4 * i < left) *(uint4*)(y + i * 4 * Y.ts) = v;
    }
    y += C * Y.ts;
  }
  if (s_out) state_store(s_out, s, w, lane);
}

// Entry states: from the workspace where segments were formed, else from the caller.
template <int TERMS>
__global__ void __launch_bounds__(128, TERMS == 3 ? 2 : 3) la_forward_kernel(LinAttnArgs p) {
  extern __shared__ __align__(128) char smem[];
  cudaGridDependencySynchronize();
  const Span sp = span_of(p, blockIdx.x);
  const size_t so = ((size_t)sp.b * p.H + sp.h) * TILE;
  const float* in = p.seg_states ? p.seg_states + (size_t)blockIdx.x * TILE : p.state_in ? p.state_in + so : nullptr;
  scan<TERMS>(sp.t1 - sp.t0, run_of(p.q, sp, false), run_of(p.k, sp, false), run_of(p.v, sp, false), run_of(p.o, sp, false), false, p.log_decay[sp.h],
              p.scale, in, false, p.seg_states || !p.state_out ? nullptr : p.state_out + so, smem);
}
// Scans of every segment: dq, dk, dv, as in la_backward_short_kernel.
template <int TERMS>
__global__ void __launch_bounds__(128, TERMS == 3 ? 2 : 3) la_backward_kernel(LinAttnArgs p, int first, int scans) {
  extern __shared__ __align__(128) char smem[];
  cudaGridDependencySynchronize();
  const int which = first + blockIdx.x % scans, item = blockIdx.x / scans;
  const Span sp = span_of(p, item);
  const size_t so = ((size_t)sp.b * p.H + sp.h) * TILE;
  const float* s_in = p.seg_states ? p.seg_states + (size_t)item * TILE : p.state_in ? p.state_in + so : nullptr;
  const float* r_in = p.seg_states ? p.seg_grads + (size_t)item * TILE : p.dstate_out ? p.dstate_out + so : nullptr;
  const LinAttnTok &a = which == 0 ? p.dout : which == 1 ? p.v : p.k, &b = which == 0 ? p.v : which == 1 ? p.dout : p.q,
                   &c = which == 0 ? p.k : which == 1 ? p.q : p.dout, &y = which == 0 ? p.dq : which == 1 ? p.dk : p.dv;
  const bool rev = which != 0;
  scan<TERMS>(sp.t1 - sp.t0, run_of(a, sp, rev), run_of(b, sp, rev), run_of(c, sp, rev), run_of(y, sp, rev), rev, p.log_decay[sp.h], p.scale,
              rev ? r_in : s_in, which != 2, which != 2 || p.seg_states || !p.dstate_in ? nullptr : p.dstate_in + so, smem);
}
constexpr int SCAN_SMEM = TAB + 8 * TILE_B;

// The state a run of tokens leaves when it starts from zero: sum_j l^(n-1-j) b_j c_j^T, or backwards in time
// sum_j l^(n-j) scale b_j c_j^T.
template <int TERMS>
__device__ __forceinline__ void run_state(int len, const Run B, const Run Cc, bool rev, float lg, float scale, float* out, char* smem) {
  float *pw = (float*)smem + 64, *sc = (float*)smem + 193;
  const uint32_t tiles = smem_addr(smem + TAB);
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, t = lane & 3;
  float s[8][4] = {};
  const int n_chunks = (len + C - 1) / C;
  Loader lb(B, len), lc(Cc, len);
  auto fetch = [&](int it) {
    const uint32_t buf = tiles + (it % 3) * 2 * TILE_B;
    lb.next(buf);
    lc.next(buf + TILE_B);
  };
  if (n_chunks > 0) fetch(0);
  cp_commit();
  if (n_chunks > 1) fetch(1);
  cp_commit();
  decay_tables(pw, sc, lg, scale);
  for (int it = 0; it < n_chunks; ++it) {
    cp_wait<1>();
    __syncthreads();
    if (it + 2 < n_chunks) fetch(it + 2);
    cp_commit();
    const int n = min(C, len - it * C);
    const uint32_t buf = tiles + (it % 3) * 2 * TILE_B;
    uint32_t bt_at = buf + lane_cols(lane) + w * 32, bc = buf + TILE_B + lane_rows(lane);
    const float ln = pw[n];
    const float* wj = (rev ? sc + n : pw + n - 1) - 2 * t;
    float d[8][4] = {};
#pragma unroll 1
    for (int kk = 0; kk < 4; ++kk) {
      uint32_t cf[4][4], bt[4];
#pragma unroll
      for (int np = 0; np < 4; ++np) ldsm_t(cf[np], bc + np * 32);
      ldsm_t(bt, bt_at);
      const float wt[4] = {wj[0], wj[-1], wj[-8], wj[-9]};
      state_mma<TERMS>(d, bt, cf, wt);
      bt_at += 16 * PITCH;
      bc += 16 * PITCH;
      wj -= 16;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[j][e] = fmaf(ln, s[j][e], d[j][e]);
  }
  state_store(out, s, w, lane);
}
constexpr int SEG_SMEM = TAB + 6 * TILE_B;

// blockIdx.y 0: states of k v^T; 1: gradients' states of q do^T.
template <int TERMS>
__global__ void __launch_bounds__(128, 4) la_segment_kernel(LinAttnArgs p) {
  extern __shared__ __align__(128) char smem[];
  cudaGridDependencySynchronize();
  const Span sp = span_of(p, blockIdx.x);
  const bool rev = blockIdx.y != 0;
  const LinAttnTok &b = rev ? p.q : p.k, &c = rev ? p.dout : p.v;
  run_state<TERMS>(sp.t1 - sp.t0, run_of(b, sp, rev), run_of(c, sp, rev), rev, p.log_decay[sp.h], p.scale,
                   (rev ? p.seg_grads : p.seg_states) + (size_t)blockIdx.x * TILE, smem);
}

// Turns every segment's own state into the state at its entry, and forms the last state.  A thread per element, sixteen
// segments in flight.
__global__ void __launch_bounds__(256) la_join_kernel(LinAttnArgs p) {
  cudaGridDependencySynchronize();
  const bool reverse = blockIdx.y != 0;
  const int bh = blockIdx.x, h = bh % p.H, b = bh / p.H, len = p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T;
  const int e = blockIdx.z * blockDim.x + threadIdx.x;
  float* seg = (reverse ? p.seg_grads : p.seg_states) + (size_t)bh * p.n_seg * TILE + e;
  const float* in = reverse ? p.dstate_out : p.state_in;
  float* out = reverse ? p.dstate_in : p.state_out;
  const float lg = p.log_decay[h], lfull = decay_pow(lg, (float)p.seg_len);
  float run = in ? in[(size_t)bh * TILE + e] : 0.f;
  constexpr int BATCH = 16;
  for (int i0 = 0; i0 < p.n_seg; i0 += BATCH) {
    float own[BATCH];
#pragma unroll
    for (int u = 0; u < BATCH; ++u)
      if (i0 + u < p.n_seg) own[u] = seg[(size_t)(reverse ? p.n_seg - 1 - i0 - u : i0 + u) * TILE];
#pragma unroll
    for (int u = 0; u < BATCH; ++u) {
      if (i0 + u >= p.n_seg) break;
      const int sidx = reverse ? p.n_seg - 1 - i0 - u : i0 + u;
      const int n = (int)min(max((long long)len - (long long)sidx * p.seg_len, 0LL), (long long)p.seg_len);
      seg[(size_t)sidx * TILE] = run;
      run = fmaf(n == p.seg_len ? lfull : decay_pow(lg, (float)n), run, own[u]);
    }
  }
  if (out) out[(size_t)bh * TILE + e] = run;
}

// One token: a block per sequence and head.  The state is read and written once (32 KB), all in fp32.
__global__ void __launch_bounds__(256) la_step_kernel(LinAttnArgs p) {
  cudaGridDependencySynchronize();
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
  const float l = expf(p.log_decay[h]);
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

// Whether sequences are cut into segments whose entry states are formed ahead of the scans (k, v -- and q, do -- are then
// read twice, in two more launches).  One block alone takes 1.7 us a chunk, three on an SM 3.4, so cutting pays where there
// are fewer scans than SMs, and more segments than would fill the GPU even out its last wave.  Measured, whole / cut:
// forward of 16 sequences and heads x 8192 tokens 209 / 38 us, 96 x 8192 212 / 165, 128 x 8192 212 / 200, 192 x 2048
// 79 / 94; backward of 16 x 8192 212 / 80, 48 x 2048 56 / 64, 96 x 8192 308 / 383; of 16 x 512 either way 16 / 17.
// scans: how many scans of every sequence run in the launch (1, or 3 in the backward pass).
struct Layout { int n_seg, seg_len; };
Layout choose_layout(long long bh, int T, int scans) {
  const int chunks = (T + C - 1) / C;
  const long long want = bh * scans < 112 && chunks >= 16 ? std::min<long long>((1024 + bh - 1) / bh, chunks / 4) : 1;
  const int per = (int)((chunks + want - 1) / want);
  return Layout{(chunks + per - 1) / per, per * C};
}

}  // namespace

size_t linattn_workspace(bool backward, int B, int T, int H) {
  const Layout l = choose_layout((long long)B * H, T, backward ? 3 : 1);
  return l.n_seg > 1 ? (size_t)B * H * l.n_seg * TILE * sizeof(float) * (backward ? 2 : 1) : 0;
}

cudaError_t launch_linattn_step(const LinAttnArgs& a, cudaStream_t s) {
  return launch_after(la_step_kernel, dim3((unsigned)(a.B * a.H)), 256, 0, s, a);
}

cudaError_t launch_linattn(LinAttnArgs a, bool backward, void* workspace, cudaStream_t s) {
  const int bh = a.B * a.H;
  // The backward pass of `items` spans.  Without segments the gradient of the incoming state is written by dv's scans while dk's
  // may still have to read the outgoing one: two launches where the caller gave one buffer for both (with segments the
  // join has read and written it before, and the scans begin with the workspace).  One buffer against two: [16, 512, 16] 75 / 72
  // us, [64, 512, 16] 246 / 240, 38 x 15 sequences of 9 tokens 20.6 / 16.6.
  auto run_backward = [&](void (*kernel)(LinAttnArgs, int, int), int items, size_t smem) {
    const bool one_launch = a.n_seg > 1 || !a.dstate_in || a.dstate_in != a.dstate_out;
    if (one_launch) return launch_after(kernel, dim3((unsigned)(3 * items)), 128, smem, s, a, 0, 3);
    const cudaError_t e = launch_after(kernel, dim3((unsigned)(2 * items)), 128, smem, s, a, 0, 2);
    return e != cudaSuccess ? e : launch_after(kernel, dim3((unsigned)items), 128, smem, s, a, 2, 1);
  };
  if (a.T <= C) {
    a.n_seg = 1;
    a.seg_len = C;
    return backward ? run_backward(la_backward_short_kernel, bh, SHORT_SMEM) : launch_after(la_forward_short_kernel, dim3((unsigned)bh), 128, SHORT_SMEM, s, a);
  }
  const Layout l = choose_layout(bh, a.T, backward ? 3 : 1);
  a.n_seg = l.n_seg;
  a.seg_len = l.seg_len;
  const bool leaves = backward ? a.dstate_in != nullptr : a.state_out != nullptr;
  cudaError_t e;
  if (a.n_seg > 1) {
    a.seg_states = (float*)workspace;
    a.seg_grads = a.seg_states + (size_t)bh * a.n_seg * TILE;
    static SmemLimit limit[2];
    auto seg = leaves ? la_segment_kernel<3> : la_segment_kernel<2>;
    e = limit[leaves].raise((const void*)seg, SEG_SMEM);
    if (e == cudaSuccess) e = launch_after(seg, dim3((unsigned)(bh * a.n_seg), backward ? 2 : 1), 128, SEG_SMEM, s, a);
    if (e == cudaSuccess) e = launch_after(la_join_kernel, dim3((unsigned)bh, backward ? 2 : 1, TILE / 256), 256, 0, s, a);
    if (e != cudaSuccess) return e;
  }
  // Three terms for the state that leaves, unless it comes from the segments.  In the backward pass that is one instance for all
  // three scans, though only dv's hands a state out: [16, 512, 16] 72 us with dstate_in, 57 without, [64, 512, 16] 240 and 187.
  const bool three = leaves && a.n_seg == 1;
  static SmemLimit limit[4];
  SmemLimit& lim = limit[backward * 2 + three];
  if (backward) {
    auto kernel = three ? la_backward_kernel<3> : la_backward_kernel<2>;
    e = lim.raise((const void*)kernel, SCAN_SMEM);
    return e != cudaSuccess ? e : run_backward(kernel, bh * a.n_seg, SCAN_SMEM);
  }
  auto kernel = three ? la_forward_kernel<3> : la_forward_kernel<2>;
  e = lim.raise((const void*)kernel, SCAN_SMEM);
  return e != cudaSuccess ? e : launch_after(kernel, dim3((unsigned)(bh * a.n_seg)), 128, SCAN_SMEM, s, a);
}

}  // namespace lp
