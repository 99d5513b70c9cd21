// The scan of linear attention (formulas: linear_attn.cu) on the 5th-generation tensor cores, chunks of 128 tokens.
//
//   y_i = w_i (a_i S) + sum_j l^|i-j| scale (a_i . b_j) c_j,     S <- l^n S + sum_j v_j b_j c_j^T
//
// per chunk, with accumulators in tensor memory (256 columns of a block):
//   SC = A B^T           128 x 128, K = 64     thread i (= lane i of tensor memory) scales its row by the decays and
//   INT = A (S1 + S2)    128 x 64,  K = 2 x 64 writes it back as bf16: P, the A operand of the next product
//   Y = P C              128 x 64,  K = 128
//   DS = [B1 | B2]^T C   128 x 64,  K = 128    b_j v_j as two bf16 terms: rows 0-63 their first, rows 64-127 their second
// The state is kept as two fp32 matrices in registers, one row per thread: threads 0-63 what the first terms add up
// to, threads 64-127 the second; S1 and S2 are their bf16 copies.
//
// mma.sync did the same with 16 rows per warp, re-reading the state and the tiles of b and c from shared memory for each
// of them: 0.8 of its time went on shared-memory reads and their latency (1.15 us per 64 tokens and SM; 24 backward
// scans' worth of a [16, 512, 16 heads] pass took 61 us).  Here an operand is read once per product and no fragment passes
// through registers.  A tcgen05.mma costs its issuing thread about a hundred clocks, so two control warps issue: one SC and
// Y, the other INT and DS.  Two blocks share an SM: one's products run under the other's row work.
// Tiles come in by cp.async (rows behind the end of a sequence as zeros); a and b of the next chunk are fetched as soon as
// this chunk's first products have read them, c behind the second.
// Every wait is bounded (tc::mbar_wait); one that gives up raises the TIMEOUT bit of a.status (if given), and the block
// runs to its end without waiting.
#include "linear_attn.cuh"
#include "tc_prims.cuh"

namespace lp {
namespace {
using namespace tc;

constexpr int C = 128;                           // tokens of a chunk
constexpr int ROWS = 128, THREADS = ROWS + 64;   // four row warps, two control warps
constexpr int T16 = C * 128;                     // bytes of a tile of 128 tokens
constexpr int O_A = 0, O_B = T16, O_C = 2 * T16, O_HL = 3 * T16, O_S = 5 * T16, O_END = O_S + 2 * 8192;
constexpr uint32_t COL_SC = 0, COL_P = 0, COL_Y = 64, COL_INT = 128, COL_DS = 192, COLS = 256;

struct __align__(16) Shared {
  uint64_t sc, in, y, ds;
  uint32_t tmem;
  int abort_flag, no_status;
  float pw[C + 1];                               // l^n
  float diag[64];                                // [32 + n] = scale l^n, 0 for n < 0
  float unit[32];                                // scale l^(distance to the block's edge): forward [x] = 31 - x, backwards [x] = x
};
constexpr int SMEM = 1024 + O_END + (int)sizeof(Shared);

// 16-byte unit u of row r of a 128-byte-swizzled tile.
__device__ __forceinline__ uint32_t unit_at(uint32_t tile, int r, int u) { return tile + r * 128 + ((u ^ (r & 7)) << 4); }
__device__ __forceinline__ void sts(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ uint4 lds(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }

// 128 token rows into a tile by the row threads; rows at or behind n become zero.
__device__ __forceinline__ void load_tile(uint32_t tile, const bf16* src, long long ts, int n) {
  const int row = threadIdx.x >> 3, u = threadIdx.x & 7;
  const uint32_t d = unit_at(tile, row, u);      // (row + 16 i) & 7 does not depend on i
  const bf16* g = src + row * ts + u * 8;
  if (n == C) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d + i * 2048), "l"(g + i * 16 * ts) : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool in = row + i * 16 < n;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d + i * 2048), "l"(in ? g + i * 16 * ts : src), "r"(in ? 16 : 0) : "memory");
    }
  }
}

// One poller per warp; afterwards the whole warp may read what the barrier's products have written.
__device__ __forceinline__ void warp_wait(uint64_t* bar, uint32_t parity, Shared* sh, int* status, int lane) {
  if (lane == 0) mbar_wait(bar, parity, &sh->abort_flag, status);
  __syncwarp();
  tc_fence_after();
}

template <bool REV>
__device__ __forceinline__ void scan(const LinAttnArgs& p, const LaSpan& sp, const LinAttnTok& A, const LinAttnTok& B, const LinAttnTok& Cc,
                                     const LinAttnTok& Y, const float* s_in, bool transposed) {
  extern __shared__ uint8_t raw[];
  uint8_t* base = (uint8_t*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
  Shared* sh = (Shared*)(base + O_END);
  const uint32_t sm = smem_u32(base);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n_chunks = (sp.t1 - sp.t0 + C - 1) / C;
  if (n_chunks == 0) return;
  int* status = p.status ? p.status : &sh->no_status;
  const float lg = p.log_decay[sp.h];
  auto begin = [&](int it) { return sp.t0 + (long long)(REV ? n_chunks - 1 - it : it) * C; };
  auto valid = [&](int it) { return min(C, (int)(sp.t1 - begin(it))); };
  if (tid < ROWS) {
    load_tile(sm + O_A, la_at(A, sp, begin(0)), A.ts, valid(0));
    load_tile(sm + O_B, la_at(B, sp, begin(0)), B.ts, valid(0));
    cp_commit();
    load_tile(sm + O_C, la_at(Cc, sp, begin(0)), Cc.ts, valid(0));
    cp_commit();
  }
  if (tid == 0) {
    mbar_init(&sh->sc, 1); mbar_init(&sh->in, 1); mbar_init(&sh->y, 1); mbar_init(&sh->ds, 1);
    sh->abort_flag = 0;
    sh->no_status = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid < 64) sh->diag[tid] = tid < 32 ? 0.f : decay_pow(lg, (float)(tid - 32)) * p.scale;
  else if (tid < 96) sh->unit[tid - 64] = decay_pow(lg, (float)(REV ? tid - 64 : 95 - tid)) * p.scale;
  if (tid <= C) sh->pw[tid] = decay_pow(lg, (float)tid);
  if (warp == 4) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem)), "r"(COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // state: row tid of the first terms (tid < 64) or row tid - 64 of the second
  float st[64];
  const int srow = tid & 63;
  auto publish = [&]() {
    const uint32_t tile = sm + O_S + (tid >> 6) * 8192;
#pragma unroll
    for (int u = 0; u < 8; ++u)
      sts(unit_at(tile, srow, u), la_pack(st[8 * u], st[8 * u + 1]), la_pack(st[8 * u + 2], st[8 * u + 3]), la_pack(st[8 * u + 4], st[8 * u + 5]),
          la_pack(st[8 * u + 6], st[8 * u + 7]));
  };
  if (tid < ROWS) {
#pragma unroll
    for (int c = 0; c < 64; ++c) st[c] = tid < 64 && s_in ? s_in[transposed ? c * 64 + srow : srow * 64 + c] : 0.f;
    publish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *(volatile uint32_t*)&sh->tmem, mine = tmem + ((uint32_t)((warp & 3) * 32) << 16);

  if (warp >= 4) {
    // ---------------------------------------------------------------- control: SC and Y (warp 4), INT and DS (warp 5)
    const uint32_t i_sc = make_idesc(128, 128, false, false), i_n64 = make_idesc(128, 64, false, true), i_ds = make_idesc(128, 64, true, true);
    const uint64_t da = make_desc(sm + O_A, false, 0), db = make_desc(sm + O_B, false, 0), dc = make_desc(sm + O_C, true, T16),
                   dhl = make_desc(sm + O_HL, true, T16), dst = make_desc(sm + O_S, true, 8192);
    for (int it = 0; it < n_chunks; ++it) {
      __syncthreads();                           // a, b and the state are in place, the last chunk's accumulators have been read
      tc_fence_after();
      if (lane == 0) {
        if (warp == 4) {
#pragma unroll
          for (int k = 0; k < 4; ++k) tc_mma(tmem + COL_SC, da + (uint64_t)(k * 2), db + (uint64_t)(k * 2), i_sc, k != 0);
          tc_commit(&sh->sc);
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k)            // k-steps 4-7: the same columns of a against the second state
            tc_mma(tmem + COL_INT, da + (uint64_t)((k & 3) * 2), dst + (uint64_t)(k * 128), i_n64, k != 0);
          tc_commit(&sh->in);
        }
      }
      __syncwarp();
      __syncthreads();                           // P, the decayed b and c are in place
      tc_fence_after();
      if (lane == 0) {
        if (warp == 4) {
#pragma unroll
          for (int k = 0; k < 8; ++k) tc_mma_ts(tmem + COL_Y, tmem + COL_P + k * 8, dc + (uint64_t)(k * 128), i_n64, k != 0);
          tc_commit(&sh->y);
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) tc_mma(tmem + COL_DS, dhl + (uint64_t)(k * 128), dc + (uint64_t)(k * 128), i_ds, k != 0);
          tc_commit(&sh->ds);
        }
      }
      __syncwarp();
    }
  } else {
    // ---------------------------------------------------------------- row threads
    for (int it = 0; it < n_chunks; ++it) {
      const int n = valid(it), ph = it & 1;
      cp_wait<1>();                              // a and b; c may still be under way
      proxy_fence();
      __syncthreads();
      // b_tid times its weight in the state, as two terms.  Rows behind n are zero.
      const float wt = REV ? sh->pw[tid + 1] * p.scale : sh->pw[max(n - 1 - tid, 0)];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const uint4 v = lds(unit_at(sm + O_B, tid, u));
        const uint32_t x[4] = {v.x, v.y, v.z, v.w};
        uint32_t h[4], l[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float f0 = la_lo(x[e]) * wt, f1 = la_hi(x[e]) * wt;
          h[e] = la_take(f0, f1);
          l[e] = la_pack(f0, f1);
        }
        sts(unit_at(sm + O_HL, tid, u), h[0], h[1], h[2], h[3]);
        sts(unit_at(sm + O_HL + T16, tid, u), l[0], l[1], l[2], l[3]);
      }
      warp_wait(&sh->sc, ph, sh, status, lane);
      // row tid of P: pieces of 32 columns; the warp's own piece crosses the diagonal, those beyond it are not seen
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t pk[16];
        if (REV ? q < warp : q > warp) {
#pragma unroll
          for (int i = 0; i < 16; ++i) pk[i] = 0u;
        } else {
          uint32_t v[32];
          tc_ld32(mine + COL_SC + 32 * q, v);
          tc_wait_ld();
          if (q == warp) {
            const float* dg = sh->diag + 32 + (REV ? -lane : lane);
#pragma unroll
            for (int i = 0; i < 32; i += 2)
              pk[i >> 1] = la_pack(__uint_as_float(v[i]) * dg[REV ? i : -i], __uint_as_float(v[i + 1]) * dg[REV ? i + 1 : -i - 1]);
          } else {
            const float f = REV ? sh->pw[32 * (q - warp) - lane] : sh->pw[32 * (warp - q) + lane - 31];
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
              const float4 u = *(const float4*)(sh->unit + i);
              pk[i >> 1] = la_pack(__uint_as_float(v[i]) * (u.x * f), __uint_as_float(v[i + 1]) * (u.y * f));
              pk[(i >> 1) + 1] = la_pack(__uint_as_float(v[i + 2]) * (u.z * f), __uint_as_float(v[i + 3]) * (u.w * f));
            }
          }
        }
        tc_st16(mine + COL_P + 16 * q, pk);      // columns of SC that this row has read already
      }
      tc_wait_st();
      warp_wait(&sh->in, ph, sh, status, lane);  // a has been read for the last time
      cp_wait<0>();                              // c
      proxy_fence();
      tc_fence_before();
      __syncthreads();
      if (it + 1 < n_chunks) {
        load_tile(sm + O_A, la_at(A, sp, begin(it + 1)), A.ts, valid(it + 1));
        load_tile(sm + O_B, la_at(B, sp, begin(it + 1)), B.ts, valid(it + 1));
      }
      cp_commit();
      uint32_t v[64];
      warp_wait(&sh->ds, ph, sh, status, lane);
      tc_ld32(mine + COL_DS, v);
      tc_ld32(mine + COL_DS + 32, v + 32);
      tc_wait_ld();
      const float ln = sh->pw[n];
#pragma unroll
      for (int c = 0; c < 64; ++c) st[c] = fmaf(ln, st[c], __uint_as_float(v[c]));
      publish();
      warp_wait(&sh->y, ph, sh, status, lane);
      if (it + 1 < n_chunks) load_tile(sm + O_C, la_at(Cc, sp, begin(it + 1)), Cc.ts, valid(it + 1));
      cp_commit();
      const float wi = REV ? sh->pw[max(n - 1 - tid, 0)] : sh->pw[tid + 1] * p.scale;
      bf16* dst = const_cast<bf16*>(la_at(Y, sp, begin(it))) + tid * Y.ts;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        uint32_t iv[32];
        tc_ld32(mine + COL_Y + 32 * half, v);
        tc_ld32(mine + COL_INT + 32 * half, iv);
        tc_wait_ld();
        if (tid < n) {
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            uint32_t o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int c = 8 * u + 2 * e;
              o[e] = la_pack(fmaf(wi, __uint_as_float(iv[c]), __uint_as_float(v[c])), fmaf(wi, __uint_as_float(iv[c + 1]), __uint_as_float(v[c + 1])));
            }
            *(uint4*)(dst + 32 * half + 8 * u) = make_uint4(o[0], o[1], o[2], o[3]);
          }
        }
      }
      tc_fence_before();
    }
  }
  __syncthreads();
  if (warp == 4) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(COLS) : "memory");
  }
}

// Entry states: from the workspace where they were formed ahead of the scans (state_out may then be state_in), else state_in.
__global__ void __launch_bounds__(THREADS, 2) la_forward_tc_kernel(LinAttnArgs p) {
  const LaSpan sp = la_span(p, blockIdx.x);
  const float* in = p.seg_states ? p.seg_states + (size_t)blockIdx.x * LA_STATE : p.state_in ? p.state_in + ((size_t)sp.b * p.H + sp.h) * LA_STATE : nullptr;
  scan<false>(p, sp, p.q, p.k, p.v, p.o, in, false);
}

// Three scans of every segment: dq, dk, dv.
__global__ void __launch_bounds__(THREADS, 2) la_backward_tc_kernel(LinAttnArgs p) {
  const int which = blockIdx.x % 3, item = blockIdx.x / 3;
  const LaSpan sp = la_span(p, item);
  const size_t so = ((size_t)sp.b * p.H + sp.h) * LA_STATE;
  const float* s_in = p.seg_states ? p.seg_states + (size_t)item * LA_STATE : p.state_in ? p.state_in + so : nullptr;
  const float* r_in = p.seg_states ? p.seg_grads + (size_t)item * LA_STATE : p.dstate_out ? p.dstate_out + so : nullptr;
  if (which == 0) scan<false>(p, sp, p.dout, p.v, p.k, p.dq, s_in, true);
  else if (which == 1) scan<true>(p, sp, p.v, p.dout, p.q, p.dk, r_in, true);
  else scan<true>(p, sp, p.k, p.q, p.dout, p.dv, r_in, false);
}

}  // namespace

cudaError_t launch_linattn_scan_tc(const LinAttnArgs& a, bool backward, cudaStream_t s) {
  static SmemLimit limit[2];
  auto kernel = backward ? la_backward_tc_kernel : la_forward_tc_kernel;
  const cudaError_t e = limit[backward].raise((const void*)kernel, SMEM);
  const long long blocks = (long long)a.B * a.H * a.n_seg * (backward ? 3 : 1);
  return e != cudaSuccess ? e : launch_kernel(kernel, dim3((unsigned)blocks), THREADS, (size_t)SMEM, s, a);
}

}  // namespace lp
