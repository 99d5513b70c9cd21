// Token and position embedding (chunk 0 of a language model), and its gradient by sorted tokens.
//
//   h[r]      = scale * table[ids[r]] + pos[r mod T]
//   dtable[v] = scale * sum of dh[r] over the rows r with ids[r] = v, in increasing r;  rows of unused tokens are 0
//   dpos[t]   = sum of dh[r] over the rows r with r mod T = t
//
// The gradient is bound by memory: dh is read once, the whole table's gradient is written once.  No floating-point
// atomics: every sum has a fixed order.
//   sort    : a stable counting sort of the rows by token in ONE launch without communication between blocks.  The
//             tokens are dealt out to n blocks (token mod n: frequent tokens tend to have neighbouring ids); every
//             block reads all ids, counts those of its tokens per warp (each warp has its own stretch of rows) and
//             the ids that belong to blocks before it, which gives its place in the order.  A second sweep places
//             the rows.  The ids are small (32 KB for 8192 rows), so reading them n times costs less than the
//             launches and grid-wide exchanges of a radix sort.
//   sum     : the sorted rows are cut into stretches of P; a worker sums the tokens that start in its stretch, reading
//             whole rows of dh.  A token with more than 4 P rows is cut into pieces of 4 P, one per worker, whose fp32
//             sums go to the workspace.  Further blocks of the launch write the zero rows and the position gradient.
//   combine : adds the pieces of every such token in order (a launch of its own, only if more than 4 P rows exist).
// Measured: 8192 rows of 512 into 8192 tokens 14 us (sort 5, sums 6, pieces 2: launches that follow one another); 65536 rows
// of 1024 into 32768 tokens of natural text 87 us: sort 16, the position gradient's read of dh 24, of which it hides
// a third, sums 46 (134 MB read and 134 written, of which 62 are still in the L2 cache when it ends: memory at 54 %), pieces
// 6.  The floor of the latter, dh read once and both gradients written, is 41 us.  fp32: 16.5 and 136 us.  The lookup of 8192
// rows of 1024 with positions takes 5.2 us with all of it in the L2 cache, as in a replayed graph, and 10.7 from memory.
// More than 131072 tokens are sorted by more than 128 blocks, one on an SM at a time, which compare the ids one by one:
// 65536 rows of 64 into 131072 tokens 28.8 us, 131073 39.0, 262144 51, 2^20 156 (floors 6.4, 6.4, 12, 42); rows of 512 80, 90,
// 146, 535 (51, 51, 92, 338).  From there on the sort costs rows * vocab / 1024 reads of ids.
#include <algorithm>
#include <climits>

#include "common.cuh"
#include "launch.cuh"

namespace lp {
namespace {

constexpr int SORT_WARPS = 32;
constexpr int SORT_MAX_LOCAL = 1024;             // tokens of one sorting block (ten bits of a list entry): (32 + 2) * 1024 counters and the lists fit its shared memory
constexpr int SORT_LIST = 512;                   // rows of this block that a warp remembers
constexpr int SORT_IDS = 8;                       // ids of a lane at a time
constexpr int SUM_THREADS = 128;
constexpr int PIECES = 4;                        // rows of a piece of a long token, in stretches
constexpr int ZERO_ROWS = 16;                    // table rows a zero-filling block looks at
constexpr int POS_THREADS = 256;                 // of a block that sums positions beside the sort
constexpr int POS_PIECE = 64;                    // rows one position worker sums
constexpr uint32_t HEAVY = 0x80000000u;

template <typename T, int VEC> struct Pack;      // VEC elements as loaded (load_l2: past the SM's own cache); get(i) converts
template <> struct Pack<float, 1> {
  float x;
  __device__ void load(const float* p) { x = *p; }
  __device__ void load_l2(const float* p) { x = __ldcg(p); }
  __device__ float get(int) const { return x; }
};
template <> struct Pack<bf16, 1> {
  bf16 x;
  __device__ void load(const bf16* p) { x = *p; }
  __device__ void load_l2(const bf16* p) { x = __ldcg(p); }
  __device__ float get(int) const { return to_f(x); }
};
template <> struct Pack<float, 4> {
  float x[4];
  __device__ void load(const float* p) { *(float4*)x = *(const float4*)p; }
  __device__ void load_l2(const float* p) { *(float4*)x = __ldcg((const float4*)p); }
  __device__ float get(int i) const { return x[i]; }
};
template <> struct Pack<bf16, 8> {
  uint32_t x[4];
  __device__ void load(const bf16* p) { *(uint4*)x = *(const uint4*)p; }
  __device__ void load_l2(const bf16* p) { *(uint4*)x = __ldcg((const uint4*)p); }
  __device__ float get(int i) const { return __uint_as_float(i & 1 ? x[i >> 1] & 0xffff0000u : x[i >> 1] << 16); }
};
template <typename T> __device__ __forceinline__ void store_vec(T* p, const float (&v)[1]) { *p = from_f<T>(v[0]); }
// The gradients leave past the caches' resident set: dh, which several blocks read, is to stay there.
__device__ __forceinline__ void stream_vec(float* p, const float (&v)[1]) { __stcs(p, v[0]); }
__device__ __forceinline__ void stream_vec(float* p, const float (&v)[4]) { __stcs((float4*)p, make_float4(v[0], v[1], v[2], v[3])); }
__device__ __forceinline__ void stream_vec(float* p, const float (&v)[8]) {
  __stcs((float4*)p, make_float4(v[0], v[1], v[2], v[3]));
  __stcs((float4*)(p + 4), make_float4(v[4], v[5], v[6], v[7]));
}
__device__ __forceinline__ void store_vec(float* p, const float (&v)[4]) { *(float4*)p = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void store_vec(float* p, const float (&v)[8]) {
  *(float4*)p = make_float4(v[0], v[1], v[2], v[3]);
  *(float4*)(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store_vec(bf16* p, const float (&v)[8]) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    u[i] = *(uint32_t*)&b;
  }
  *(uint4*)p = make_uint4(u[0], u[1], u[2], u[3]);
}

// ids outside [0, vocab) are flagged and clamped.
__device__ __forceinline__ int clamp_id(int id, int vocab) { return min(max(id, 0), vocab - 1); }

// `lanes` threads (a power of two) per row, VEC elements each.
template <typename T, int VEC>
__global__ void __launch_bounds__(128) embed_fwd_kernel(EmbedProb p, int lanes_log2, int* status) {
  cudaGridDependencySynchronize();
  const long long gt = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  const long long row = gt >> lanes_log2;
  const int lane = (int)(gt & ((1 << lanes_log2) - 1));
  if (row >= p.rows) return;
  int id = p.ids[row];
  if (id < 0 || id >= p.vocab) {
    if (lane == 0 && status) atomicOr(status, ST_LABEL_RANGE);
    id = clamp_id(id, p.vocab);
  }
  const T* tok = (const T*)p.tok + (size_t)id * p.d;
  const T* pos = p.pos ? (const T*)p.pos + (size_t)(row % p.T) * p.d : nullptr;
  T* h = (T*)p.h + (size_t)row * p.d;
#pragma unroll 4
  for (int c = lane * VEC; c < p.d; c += VEC << lanes_log2) {
    Pack<T, VEC> a, b;
    float v[VEC];
    a.load(tok + c);
    if (pos) {
      b.load(pos + c);
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[i] = fmaf(p.scale, a.get(i), b.get(i));
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[i] = p.scale * a.get(i);
    }
    store_vec(h + c, v);
  }
}

// Position gradient: 2^split_log2 groups of 2^lanes_log2 threads sum one piece of one position's rows together; the first
// of them adds their sums in order.  buf: a float per thread and element.
template <typename T, int VEC>
__device__ void pos_sums(const EmbedBwdProb& p, int lanes_log2, int split_log2, int block, int pos_pieces, float* buf) {
  const int lanes = 1 << lanes_log2, lane = threadIdx.x & (lanes - 1), split = 1 << split_log2, sub = (threadIdx.x >> lanes_log2) & (split - 1);
  const long long wk = ((long long)block * blockDim.x + threadIdx.x) >> (lanes_log2 + split_log2);
  const bool real = wk < (long long)p.T * pos_pieces;
  const int t = real ? (int)(wk / pos_pieces) : 0, piece = real ? (int)(wk % pos_pieces) : 0;
  const long long step = p.T, i0 = (long long)piece * POS_PIECE;
  const long long rows = real && t < p.rows ? (p.rows - 1 - t) / step + 1 : 0;          // of this position
  const long long n = max(0LL, pos_pieces == 1 ? rows : min(rows - i0, (long long)POS_PIECE));
  const long long per = (n + split - 1) >> split_log2, k0 = min(n, sub * per), k1 = min(n, k0 + per);
  float* out = pos_pieces == 1 ? p.dpos + (size_t)t * p.d : p.pos_part + (size_t)wk * p.d;
  constexpr int U = 4;                           // rows in flight
  for (int c0 = 0; c0 < p.d; c0 += lanes * VEC) {
    const int c = c0 + lane * VEC;
    const T* dh = (const T*)p.dh + (size_t)(t + i0 * step) * p.d + c;
    float acc[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[i] = 0.f;
    if (c < p.d)
      for (long long k = k0; k < k1; k += U) {
        Pack<T, VEC> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) if (k + u < k1) x[u].load_l2(dh + (size_t)((k + u) * step) * p.d);
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (k + u < k1) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) acc[i] += x[u].get(i);
          }
      }
    if (split > 1) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < VEC; ++i) buf[threadIdx.x + i * blockDim.x] = acc[i];
      __syncthreads();
      if (sub == 0)
        for (int k = 1; k < split; ++k)
#pragma unroll
          for (int i = 0; i < VEC; ++i) acc[i] += buf[threadIdx.x + k * lanes + i * blockDim.x];
    }
    if (real && sub == 0 && c < p.d) store_vec(out + c, acc);
  }
}

// The position gradient beside the sort, whose blocks let this launch start once they know that all work before them is
// complete.  It ends no earlier than the sort, so that what follows it finds both.
template <typename T, int VEC>
__global__ void __launch_bounds__(POS_THREADS) embed_pos_kernel(EmbedBwdProb p, int lanes_log2, int split_log2, int pos_pieces) {
  __shared__ float buf[POS_THREADS * VEC];
  pos_sums<T, VEC>(p, lanes_log2, split_log2, blockIdx.x, pos_pieces, buf);
  cudaGridDependencySynchronize();
}

// Rows by token.  Block j owns the tokens t with t mod n = j (n a power of two), local index t div n.
// sorted[p] = {row, token | HEAVY if the token has more than `piece` rows}; seg[t] = {first p, number of rows}.
// First sweep: every warp counts its stretch's rows per token and lists those of this block, a lane taking eight ids at a
// time and comparing their blocks as bytes (65536 rows: 13 thousand clocks; one id per lane at a time 15, and with the next
// ones fetched ahead 17; the ids read once per cluster of four blocks, with lists passed through distributed shared memory,
// gave 85 instead of 87 us for the whole gradient and 16 instead of 14 for 8192 rows).  Second sweep: over the list
// (or over the stretch again, if the list overflowed).  let_next: the next launch may start beside this one.
__global__ void __launch_bounds__(SORT_WARPS * 32, 1) embed_sort_kernel(EmbedBwdProb p, int n_log2, int local, int piece, int* status, bool let_next) {
  extern __shared__ int sm[];
  cudaGridDependencySynchronize();
  if (let_next) cudaTriggerProgrammaticLaunchCompletion();
  const int pitch = local | 1;
  int* cnt = sm;                                 // [SORT_WARPS][pitch]
  int* start = cnt + SORT_WARPS * pitch;         // [local]
  int* total = start + local;                    // [local]
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, j = blockIdx.x, mask = (1 << n_log2) - 1;
  uint32_t* list = (uint32_t*)(total + local) + w * SORT_LIST;           // [SORT_LIST] row in the stretch * 1024 + local index
  __shared__ int less_sum, carry_of[SORT_WARPS];
  for (int i = tid; i < SORT_WARPS * pitch; i += blockDim.x) cnt[i] = 0;
  if (tid == 0) {
    less_sum = 0;
    if (j == 0) *p.n_long = 0;
  }
  __syncthreads();
  const int stretch = ((p.rows + SORT_WARPS * 32 - 1) / (SORT_WARPS * 32)) * 32;
  const long long lo = (long long)w * stretch;
  const int r0 = (int)min(lo, (long long)p.rows), r1 = (int)min(lo + stretch, (long long)p.rows);
  int* mine = cnt + w * pitch;
  const unsigned below = (1u << lane) - 1;
  int less = 0, listed = 0;
  uint32_t most = 0;                             // of all ids as unsigned numbers: at least vocab if one is out of range
  const bool wide = ((uintptr_t)p.ids & 15) == 0;
  const uint32_t jj = (uint32_t)j * 0x01010101u;
  for (int rb = r0; rb < r1; rb += 32 * SORT_IDS) {                      // a lane looks at SORT_IDS consecutive ids
    const int first = rb + lane * SORT_IDS;
    const bool whole = rb + 32 * SORT_IDS <= r1;
    int id[SORT_IDS];
    if (whole && wide) {
      *(int4*)id = *(const int4*)(p.ids + first);
      *(int4*)(id + 4) = *(const int4*)(p.ids + first + 4);
    } else {
#pragma unroll
      for (int u = 0; u < SORT_IDS; ++u) id[u] = first + u < r1 ? p.ids[first + u] : 0;
    }
    uint32_t here = 0;
#pragma unroll
    for (int u = 0; u < SORT_IDS; ++u) here = max(here, (uint32_t)id[u]);
    most = max(most, here);
    if (__any_sync(0xffffffffu, here >= (uint32_t)p.vocab)) {
#pragma unroll
      for (int u = 0; u < SORT_IDS; ++u) id[u] = clamp_id(id[u], p.vocab);
    }
    uint32_t m = 0;                              // which of them are this block's
    if (whole && n_log2 <= 7) {                  // blocks of four tokens as bytes of at most 127: compared all at once
      uint32_t in[2], geq[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t c = __byte_perm(__byte_perm(id[4 * k], id[4 * k + 1], 0x0040), __byte_perm(id[4 * k + 2], id[4 * k + 3], 0x0040), 0x5410) &
                           (uint32_t)mask * 0x01010101u;
        geq[k] = ((c | 0x80808080u) - jj) & 0x80808080u;
        in[k] = (0x80808080u - (c ^ jj)) & 0x80808080u;
      }
      less += SORT_IDS - __popc(geq[0] | geq[1] >> 1);
      m = ((in[0] >> 7) * 0x10204080u) >> 28 | ((in[1] >> 7) * 0x10204080u) >> 28 << 4;    // bits 7, 15, 23, 31 side by side
    } else {
#pragma unroll
      for (int u = 0; u < SORT_IDS; ++u) {
        const int cls = first + u < r1 ? id[u] & mask : INT_MAX;
        less += cls < j;
        m |= (uint32_t)(cls == j) << u;
      }
    }
    if (__any_sync(0xffffffffu, m)) {
      const int n = __popc(m);
      int at = listed;
#pragma unroll
      for (int k = 0; k < 4; ++k) {              // n <= 8 summed over the lanes, bit by bit
        const unsigned v = __ballot_sync(0xffffffffu, n >> k & 1);
        at += __popc(v & below) << k;
        listed += __popc(v) << k;
      }
#pragma unroll
      for (int u = 0; u < SORT_IDS; ++u)
        if (m >> u & 1) {
          const int lt = id[u] >> n_log2;
          atomicAdd(&mine[lt], 1);
          if (at < SORT_LIST) list[at] = (uint32_t)(first + u - r0) << 10 | (uint32_t)lt;
          ++at;
        }
    }
  }
  less = __reduce_add_sync(0xffffffffu, less);
  if (lane == 0 && less) atomicAdd(&less_sum, less);
  if (most >= (uint32_t)p.vocab && status && j == 0) atomicOr(status, ST_LABEL_RANGE);
  __syncthreads();
  // per token: where each warp's rows begin; over the tokens: where each token's rows begin
  int carry = less_sum;
  for (int l0 = 0; l0 < local; l0 += blockDim.x) {
    const int lt = l0 + tid;
    int sum = 0;
    if (lt < local)
      for (int k0 = 0; k0 < SORT_WARPS; k0 += 16) {
        int c[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) c[k] = cnt[(k0 + k) * pitch + lt];
#pragma unroll
        for (int k = 0; k < 16; ++k) { cnt[(k0 + k) * pitch + lt] = sum; sum += c[k]; }
      }
    int s = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int u = __shfl_up_sync(0xffffffffu, s, o); if (lane >= o) s += u; }
    if (lane == 31) carry_of[w] = s;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int k = 0; k < SORT_WARPS; ++k) { const int c = carry_of[k]; before += k < w ? c : 0; all += c; }
    if (lt < local) {
      const int at = carry + before + s - sum;
      start[lt] = at;
      total[lt] = sum;
      const long long t = ((long long)lt << n_log2) | j;
      if (t < p.vocab) p.seg[t] = make_int2(at, sum);
    }
    carry += all;
    __syncthreads();
  }
  const bool fits = listed <= SORT_LIST && stretch <= 1 << 22;
  const int steps = fits ? listed : r1 - r0;
  for (int b = 0; b < steps; b += 32) {
    const int i = b + lane;
    int r = r0, t = 0;
    bool in = i < steps;
    if (in && fits) {
      r += (int)(list[i] >> 10);
      t = (int)(list[i] & 1023) << n_log2 | j;
    } else if (in) {
      r += i;
      t = clamp_id(p.ids[r], p.vocab);
      in = (t & mask) == j;
    }
    if (__ballot_sync(0xffffffffu, in) == 0) continue;
    const int lt = in ? t >> n_log2 : ~lane;
    const unsigned peers = __match_any_sync(0xffffffffu, lt);
    if (in) p.sorted[start[lt] + mine[lt] + __popc(peers & below)] = make_int2(r, (int)((uint32_t)t | (total[lt] > piece ? HEAVY : 0u)));
    __syncwarp();
    if (in && (peers & below) == 0) mine[lt] += __popc(peers);
    __syncwarp();
  }
}

// First sorted position that stretch c owns: the first start of a token, or of a piece of a long one, at or behind
// c * P.  (A token of at most PIECES * P rows is summed whole by the stretch it starts in; a longer one is cut into pieces
// of that length, of which at most one that is not the token's first starts in a stretch.)
__device__ __forceinline__ int stretch_begin(const EmbedBwdProb& p, long long c, int P) {
  if (c * P >= p.rows) return p.rows;
  const int q = (int)(c * P);
  const int2 e = p.sorted[q];
  const int2 sg = p.seg[(uint32_t)e.y & ~HEAVY];
  const int off = q - sg.x;
  if (off == 0) return q;
  if (!((uint32_t)e.y & HEAVY)) return sg.x + sg.y;
  const int piece = PIECES * P, up = (piece - off % piece) % piece;
  return min(q + up, sg.x + sg.y);
}

template <typename T, int VEC>
__global__ void __launch_bounds__(SUM_THREADS) embed_sum_kernel(EmbedBwdProb p, int lanes_log2, int P, int sum_blocks, int pos_blocks,
                                                                int pos_pieces) {
  cudaGridDependencySynchronize();
  const int lanes = 1 << lanes_log2, per_block = SUM_THREADS >> lanes_log2;
  const int grp = threadIdx.x >> lanes_log2, lane = threadIdx.x & (lanes - 1);
  if ((int)blockIdx.x >= sum_blocks && (int)blockIdx.x < sum_blocks + pos_blocks) {
    if (blockIdx.y == 0) pos_sums<T, VEC>(p, lanes_log2, 0, (int)blockIdx.x - sum_blocks, pos_pieces, nullptr);
    return;
  }
  const int c = (blockIdx.y * lanes + lane) * VEC;
  if (c >= p.d) return;
  const T* dh = (const T*)p.dh + c;
  if ((int)blockIdx.x < sum_blocks) {
    const long long ch = (long long)blockIdx.x * per_block + grp;
    const int b0 = stretch_begin(p, ch, P), b1 = stretch_begin(p, ch + 1, P);
    if (b0 >= b1) return;
    uint32_t cur = (uint32_t)p.sorted[b0].y;
    bool first = b0 == 0 || (uint32_t)p.sorted[b0 - 1].y != cur;
    float acc[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[i] = 0.f;
    auto flush = [&]() {
      if (cur & HEAVY) {
        if (first && lane == 0 && blockIdx.y == 0) p.long_list[atomicAdd(p.n_long, 1)] = make_int2((int)ch, (int)(cur & ~HEAVY));
        store_vec(p.part + (size_t)(2 * ch + (first ? 1 : 0)) * p.d + c, acc);
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] *= p.scale;
        stream_vec(p.dtok + (size_t)cur * p.d + c, acc);
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i) acc[i] = 0.f;
    };
    constexpr int U = VEC == 1 ? 4 : 8;          // rows in flight, whatever tokens they belong to
    int2 e[U], next[U];
#pragma unroll
    for (int u = 0; u < U; ++u) next[u] = b0 + u < b1 ? p.sorted[b0 + u] : make_int2(0, 0);
    for (int q = b0; q < b1; q += U) {
      Pack<T, VEC> x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        e[u] = next[u];
        if (q + u < b1) x[u].load(dh + (size_t)e[u].x * p.d);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) if (q + U + u < b1) next[u] = p.sorted[q + U + u];   // the next rows' numbers meanwhile
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (q + u >= b1) break;
        if ((uint32_t)e[u].y != cur) { flush(); cur = (uint32_t)e[u].y; first = true; }
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] += x[u].get(i);
      }
    }
    flush();
  } else {
    const long long t0 = (long long)(blockIdx.x - sum_blocks - pos_blocks) * ZERO_ROWS;
    float z[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) z[i] = 0.f;
    for (int i = grp; i < ZERO_ROWS; i += per_block)
      if (t0 + i < p.vocab && p.seg[t0 + i].y == 0) stream_vec(p.dtok + (size_t)(t0 + i) * p.d + c, z);
  }
}

// Adds `pieces` rows of d floats (piece 0 at base + first, piece i > 0 at base + i * stride) and stores the sum times
// scale.  A block has 256 columns: eight warps per 128 of them, each with every eighth piece, whose sums are added in
// order.  (One block for all columns of the commonest token of natural text read its pieces at 44 GB/s: 17 us.)
constexpr int COMBINE_COLS = 256, SLICES = 8, COMBINE_WARPS = SLICES * COMBINE_COLS / 128;
__device__ __forceinline__ void add_pieces(const float* base, long long first, long long stride, int pieces, int d, float* out, float scale,
                                           float (*red)[128]) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, tile = w / SLICES, slice = w % SLICES, c0 = blockIdx.y * COMBINE_COLS + tile * 128 + lane;
  int col[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) col[u] = min(c0 + 32 * u, d - 1);
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  constexpr int BATCH = 8;                       // pieces in flight
  for (int i0 = slice; i0 < pieces; i0 += SLICES * BATCH) {
    float x[BATCH][4];
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const int i = min(i0 + k * SLICES, pieces - 1);
      const float* src = base + (i == 0 ? first : (long long)i * stride);
#pragma unroll
      for (int u = 0; u < 4; ++u) x[k][u] = src[col[u]];
    }
#pragma unroll
    for (int k = 0; k < BATCH; ++k)
      if (i0 + k * SLICES < pieces) {
#pragma unroll
        for (int u = 0; u < 4; ++u) acc[u] += x[k][u];
      }
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < 4; ++u) red[w][lane + 32 * u] = acc[u];
  __syncthreads();
  if (slice == 0) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      float s = acc[u];
#pragma unroll
      for (int i = 1; i < SLICES; ++i) s += red[w + i][lane + 32 * u];
      if (c0 + 32 * u < d) out[c0 + 32 * u] = s * scale;
    }
  }
}
// The long tokens of the list, then the positions with several pieces, dealt out to the blocks.
__global__ void __launch_bounds__(COMBINE_WARPS * 32) embed_combine_kernel(EmbedBwdProb p, int P, int positions, int pos_pieces) {
  __shared__ float red[COMBINE_WARPS][128];
  cudaGridDependencySynchronize();
  const int n_long = *p.n_long;
  for (int i = blockIdx.x; i < n_long + positions; i += gridDim.x) {
    if (i < n_long) {
      const int2 e = p.long_list[i];             // stretch of the first piece, token
      const int rows = p.seg[e.y].y;
      add_pieces(p.part + (size_t)(2 * (long long)e.x) * p.d, p.d, 2LL * PIECES * p.d, (rows + PIECES * P - 1) / (PIECES * P), p.d,
                 p.dtok + (size_t)e.y * p.d, p.scale, red);
    } else {
      const int t = i - n_long;
      const long long per = (long long)POS_PIECE * p.T;
      add_pieces(p.pos_part + (size_t)t * pos_pieces * p.d, 0, p.d, (int)(((long long)p.rows - t + per - 1) / per), p.d, p.dpos + (size_t)t * p.d, 1.f, red);
    }
  }
}

int lanes_log2_for(int vecs, int max_log2) {
  int l = 0;
  while (l < max_log2 && (1 << l) < vecs) ++l;
  return l;
}
bool aligned16(const void* a, const void* b, const void* c) { return (((uintptr_t)a | (uintptr_t)b | (uintptr_t)c) & 15) == 0; }

// Rows of a stretch.  Few rows: short stretches, so that there are enough workers; many: long ones, so that the
// pieces of frequent tokens stay few.
// Narrow rows keep few threads busy, each of which then waits for one batch of rows after the other: stretches are
// halved until the sums have 256 threads for every SM (8 elements each).  17837 rows of 24 into 10790 tokens 31.2 -> 17.6 us,
// 1089 of 272 into 8 16.3 -> 11.6; with 512 threads for every SM 65536 rows of 64 take 43 us instead of 35.
int piece_rows(int rows, int d) {
  int P = rows <= 16384 ? 16 : rows <= 131072 ? 32 : 64;
  while (P > 4 && (long long)rows * d / (8 * P) < 148 * 256) P /= 2;
  return P;
}
// Pieces of a position's rows: only where the positions alone would not give every SM two workers.
int pos_pieces_for(int rows, int T) { return T >= 296 ? 1 : (int)(((rows + T - 1) / T + POS_PIECE - 1) / POS_PIECE); }
bool pos_beside_sort(const EmbedBwdProb& p, size_t elem) { return p.dpos && (size_t)p.rows * p.d * elem > ((size_t)64 << 20); }
// What the last launch has to do at most: tokens of several pieces, positions of several pieces.
struct Joins { int tokens, positions; };
Joins joins_of(const EmbedBwdProb& p) {
  return Joins{p.rows / (PIECES * piece_rows(p.rows, p.d) + 1), p.dpos && pos_pieces_for(p.rows, p.T) > 1 ? p.T : 0};
}
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

template <typename T, int VEC>
cudaError_t run_sort_and_sum(const EmbedBwdProb& p, int P, int chunks, int pos_pieces, int* d_status, cudaStream_t s) {
  const int vecs = (p.d + VEC - 1) / VEC, ll = lanes_log2_for(vecs, 7), per_block = SUM_THREADS >> ll;
  int n_log2 = 0;
  while (n_log2 < 7 && (1 << n_log2) < p.vocab) ++n_log2;
  while ((((long long)p.vocab + (1 << n_log2) - 1) >> n_log2) > SORT_MAX_LOCAL) ++n_log2;
  const int local = (int)(((long long)p.vocab + (1 << n_log2) - 1) >> n_log2);
  const size_t smem = ((size_t)SORT_WARPS * (local | 1) + 2 * (size_t)local + SORT_WARPS * SORT_LIST) * sizeof(int);
  static SmemLimit limit;
  cudaError_t e = limit.raise((const void*)embed_sort_kernel,
                              (SORT_WARPS * (SORT_MAX_LOCAL | 1) + 2 * SORT_MAX_LOCAL + SORT_WARPS * SORT_LIST) * (int)sizeof(int));
  if (e != cudaSuccess) return e;
  // The position gradient reads dh a second time.  While dh stays in the L2 cache (126 MB) that is cheap, and it rides with
  // the sums; a larger one is read beside the sort, which leaves the memory idle: on the SMs that have no sorting block, and
  // on the others as those end.  ([65536, 1024]: 91 us in the sort's own launch, 88 in one beside it; with few enough registers to
  // share the SMs with it 93 to 99, since the sort then waits for its ids.)  With the sums / beside the sort, bf16, natural text:
  // rows of 1024 into 32768 tokens, 512 positions, 8 MiB 43.2 / 43.8 us, 16 43.2 / 44.1, 32 49.5 / 50.5, 48 55.5 / 63, 64 65.1 / 68.8, 96
  // 79.0 / 76.2, 128 93.1 / 88.6; rows of 512 into 8192, 256 positions, 8 MiB 18.5 / 22.2, 32 39.0 / 41.0, 64 51.4 / 55.4, 96 74.3 /
  // 80.1, 128 94.2 / 98.3: beyond 64 MiB the wide rows gain, these lose 4 to 8 %.
  const long long pos_work = p.dpos ? (long long)p.T * pos_pieces : 0;
  const bool early = pos_beside_sort(p, sizeof(T));
  e = launch_after(embed_sort_kernel, dim3(1u << n_log2), SORT_WARPS * 32, smem, s, p, n_log2, local, PIECES * P, d_status, early);
  if (e != cudaSuccess) return e;
  if (early) {
    const int groups_log2 = 8 - ll;              // of a block
    int split = 0;                               // groups per sum: until every SM has four blocks
    while (split < groups_log2 && (pos_work << split >> groups_log2) < 4 * 148) ++split;
    const long long blocks = ((pos_work << split) + (1 << groups_log2) - 1) >> groups_log2;
    e = launch_after(embed_pos_kernel<T, VEC>, dim3((unsigned)blocks), POS_THREADS, 0, s, p, ll, split, pos_pieces);
    if (e != cudaSuccess) return e;
  }
  const long long pos_late = early ? 0 : (pos_work + per_block - 1) / per_block;
  const int sum_blocks = (chunks + per_block - 1) / per_block;
  const long long zero_blocks = ((long long)p.vocab + ZERO_ROWS - 1) / ZERO_ROWS;
  const dim3 grid((unsigned)(sum_blocks + pos_late + zero_blocks), (unsigned)((vecs + (1 << ll) - 1) >> ll));
  return launch_after(embed_sum_kernel<T, VEC>, grid, SUM_THREADS, 0, s, p, ll, P, sum_blocks, (int)pos_late, pos_pieces);
}

}  // namespace

cudaError_t launch_embed_fwd(const EmbedProb& p, int* d_status, bool is_bf16, cudaStream_t s) {
  const int full = is_bf16 ? 8 : 4;
  const int vec = p.d % full == 0 && aligned16(p.tok, p.pos, p.h) ? full : 1;
  const int ll = lanes_log2_for((p.d + vec - 1) / vec, 5);
  const dim3 grid((unsigned)((((long long)p.rows << ll) + 127) / 128));
  if (is_bf16)
    return vec == 8 ? launch_after(embed_fwd_kernel<bf16, 8>, grid, 128, 0, s, p, ll, d_status)
                    : launch_after(embed_fwd_kernel<bf16, 1>, grid, 128, 0, s, p, ll, d_status);
  return vec == 4 ? launch_after(embed_fwd_kernel<float, 4>, grid, 128, 0, s, p, ll, d_status)
                  : launch_after(embed_fwd_kernel<float, 1>, grid, 128, 0, s, p, ll, d_status);
}

// Workspace: sorted rows, token segments, pieces of long tokens, pieces of the position sums, the list of long
// tokens.  Pieces of positions are
// stored only if a position has more than POS_PIECE rows; then T < rows / POS_PIECE and T * pieces(T) < 3 rows / POS_PIECE.
size_t embed_bwd_workspace(int rows, int vocab, int d) {
  const size_t chunks = ((size_t)rows + piece_rows(rows, d) - 1) / piece_rows(rows, d);
  const size_t pos_rows = 3 * ((size_t)rows / POS_PIECE) + 3;
  return up256((size_t)rows * sizeof(int2)) + up256((size_t)vocab * sizeof(int2)) + up256(2 * chunks * d * sizeof(float)) +
         up256(pos_rows * d * sizeof(float)) + 256 + up256(chunks * sizeof(int2));
}

int embed_bwd_launches(const EmbedBwdProb& p, bool is_bf16) {
  const Joins joins = joins_of(p);
  return 2 + (pos_beside_sort(p, is_bf16 ? 2 : 4) ? 1 : 0) + (joins.tokens + joins.positions > 0 ? 1 : 0);
}

cudaError_t launch_embed_bwd(EmbedBwdProb p, void* workspace, int* d_status, bool is_bf16, cudaStream_t s) {
  const int P = piece_rows(p.rows, p.d), chunks = (int)(((long long)p.rows + P - 1) / P), pos_pieces = p.dpos ? pos_pieces_for(p.rows, p.T) : 0;
  char* w = (char*)workspace;
  p.sorted = (int2*)w;  w += up256((size_t)p.rows * sizeof(int2));
  p.seg = (int2*)w;     w += up256((size_t)p.vocab * sizeof(int2));
  p.part = (float*)w;   w += up256(2 * (size_t)chunks * p.d * sizeof(float));
  p.pos_part = (float*)w;
  w = (char*)workspace + embed_bwd_workspace(p.rows, p.vocab, p.d) - up256((size_t)chunks * sizeof(int2)) - 256;
  p.n_long = (int*)w;   w += 256;
  p.long_list = (int2*)w;
  const int full = is_bf16 ? 8 : 4;
  const bool vec = p.d % full == 0 && aligned16(p.dh, p.dtok, p.dpos);
  cudaError_t e;
  if (is_bf16) e = vec ? run_sort_and_sum<bf16, 8>(p, P, chunks, pos_pieces, d_status, s) : run_sort_and_sum<bf16, 1>(p, P, chunks, pos_pieces, d_status, s);
  else e = vec ? run_sort_and_sum<float, 4>(p, P, chunks, pos_pieces, d_status, s) : run_sort_and_sum<float, 1>(p, P, chunks, pos_pieces, d_status, s);
  if (e != cudaSuccess) return e;
  const Joins joins = joins_of(p);
  if (joins.tokens + joins.positions == 0) return cudaSuccess;
  return launch_after(embed_combine_kernel, dim3((unsigned)std::min(joins.tokens + joins.positions, 148), (unsigned)((p.d + COMBINE_COLS - 1) / COMBINE_COLS)),
                      COMBINE_WARPS * 32, 0, s, p, P, joins.positions, pos_pieces);
}

}  // namespace lp
