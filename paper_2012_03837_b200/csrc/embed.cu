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
//             whole rows of dh.  A token with more than P rows is cut into pieces of P, one per worker, whose fp32
//             sums go to the workspace.  Further blocks of the launch write the zero rows and the position gradient.
//   combine : adds the pieces of every such token in order (a launch of its own, only if more than P rows exist).
#include <algorithm>

#include "common.cuh"
#include "launch.cuh"

namespace lp {
namespace {

constexpr int SORT_WARPS = 32;
constexpr int SORT_MAX_LOCAL = 1536;             // tokens of one sorting block: (32 + 2) * 1536 counters fit its shared memory
constexpr int SUM_THREADS = 128;
constexpr int ZERO_ROWS = 16;                    // table rows a zero-filling block looks at
constexpr int POS_PIECE = 64;                    // rows one position worker sums
constexpr uint32_t HEAVY = 0x80000000u;

template <typename T, int VEC> struct Pack;
template <> struct Pack<float, 1> { float v[1]; __device__ void load(const float* p) { v[0] = *p; } };
template <> struct Pack<bf16, 1> { float v[1]; __device__ void load(const bf16* p) { v[0] = to_f(*p); } };
template <> struct Pack<float, 4> {
  float v[4];
  __device__ void load(const float* p) { const float4 x = *(const float4*)p; v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; }
};
template <> struct Pack<bf16, 8> {
  float v[8];
  __device__ void load(const bf16* p) {
    const uint4 x = *(const uint4*)p;
    const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(u[i] << 16); v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
  }
};
template <typename T> __device__ __forceinline__ void store_vec(T* p, const float (&v)[1]) { *p = from_f<T>(v[0]); }
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
    a.load(tok + c);
    if (pos) {
      b.load(pos + c);
#pragma unroll
      for (int i = 0; i < VEC; ++i) a.v[i] = fmaf(p.scale, a.v[i], b.v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) a.v[i] *= p.scale;
    }
    store_vec(h + c, a.v);
  }
}

// Rows by token.  Block j owns the tokens t with t mod n = j (n a power of two), local index t div n.
// sorted[p] = {row, token | HEAVY if the token has more than `piece` rows}; seg[t] = {first p, number of rows}.
__global__ void __launch_bounds__(SORT_WARPS * 32) embed_sort_kernel(EmbedBwdProb p, int n_log2, int local, int piece, int* status) {
  extern __shared__ int sm[];
  const int pitch = local | 1;                   // odd: a warp that reads one token's 32 counters meets 32 banks
  int* cnt = sm;                                 // [SORT_WARPS][pitch]
  int* start = cnt + SORT_WARPS * pitch;         // [local]
  int* total = start + local;                    // [local]
  __shared__ int less_sum;
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, j = blockIdx.x, mask = (1 << n_log2) - 1;
  for (int i = tid; i < SORT_WARPS * pitch; i += blockDim.x) cnt[i] = 0;
  if (tid == 0) less_sum = 0;
  __syncthreads();
  const int stretch = ((p.rows + SORT_WARPS * 32 - 1) / (SORT_WARPS * 32)) * 32;
  const long long lo = (long long)w * stretch;
  const int r0 = (int)min(lo, (long long)p.rows), r1 = (int)min(lo + stretch, (long long)p.rows);
  int less = 0;
  bool bad = false;
#pragma unroll 4
  for (int r = r0 + lane; r < r1; r += 32) {
    const int id = p.ids[r], t = clamp_id(id, p.vocab);
    bad |= id != t;
    less += (t & mask) < j;
    if ((t & mask) == j) atomicAdd(&cnt[w * pitch + (t >> n_log2)], 1);
  }
  less = __reduce_add_sync(0xffffffffu, less);
  if (lane == 0 && less) atomicAdd(&less_sum, less);
  if (bad && status && j == 0) atomicOr(status, ST_LABEL_RANGE);
  __syncthreads();
  for (int lt = w; lt < local; lt += SORT_WARPS) {        // per token: where each warp's rows begin
    const int c = cnt[lane * pitch + lt];
    int s = c;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int u = __shfl_up_sync(0xffffffffu, s, o); if (lane >= o) s += u; }
    cnt[lane * pitch + lt] = s - c;
    if (lane == 31) total[lt] = s;
  }
  __syncthreads();
  if (w == 0) {
    int carry = less_sum;
    for (int i0 = 0; i0 < local; i0 += 32) {
      const int lt = i0 + lane, c = lt < local ? total[lt] : 0;
      int s = c;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const int u = __shfl_up_sync(0xffffffffu, s, o); if (lane >= o) s += u; }
      if (lt < local) {
        start[lt] = carry + s - c;
        const long long t = ((long long)lt << n_log2) | j;
        if (t < p.vocab) p.seg[t] = make_int2(carry + s - c, c);
      }
      carry += __shfl_sync(0xffffffffu, s, 31);
    }
  }
  __syncthreads();
  for (int rb = r0; rb < r1; rb += 32) {
    const int r = rb + lane;
    const int t = r < r1 ? clamp_id(p.ids[r], p.vocab) : 0;
    const bool in = r < r1 && (t & mask) == j;
    if (__ballot_sync(0xffffffffu, in) == 0) continue;
    const int lt = in ? t >> n_log2 : 0;
    const unsigned peers = __match_any_sync(0xffffffffu, in ? lt : ~lane);
    if (in) {
      const int at = start[lt] + cnt[w * pitch + lt] + __popc(peers & ((1u << lane) - 1));
      p.sorted[at] = make_int2(r, (int)((uint32_t)t | (total[lt] > piece ? HEAVY : 0u)));
    }
    __syncwarp();
    if (in && (peers & ((1u << lane) - 1)) == 0) cnt[w * pitch + lt] += __popc(peers);
    __syncwarp();
  }
}

// First sorted position that stretch c owns: the first start of a token, or of a piece of a long one, at or behind
// c * P.  (A token of at most P rows is summed whole by the stretch it starts in.)
__device__ __forceinline__ int stretch_begin(const EmbedBwdProb& p, long long c, int P) {
  if (c * P >= p.rows) return p.rows;
  const int q = (int)(c * P);
  const int2 e = p.sorted[q];
  const int2 sg = p.seg[(uint32_t)e.y & ~HEAVY];
  const int off = q - sg.x;
  if (off == 0) return q;
  if (!((uint32_t)e.y & HEAVY)) return sg.x + sg.y;
  const int up = (P - off % P) % P;
  return min(q + up, sg.x + sg.y);
}

template <typename T, int VEC>
__global__ void __launch_bounds__(SUM_THREADS) embed_sum_kernel(EmbedBwdProb p, int lanes_log2, int P, int sum_blocks, int pos_blocks,
                                                                int pos_pieces) {
  const int lanes = 1 << lanes_log2, per_block = SUM_THREADS >> lanes_log2;
  const int grp = threadIdx.x >> lanes_log2, lane = threadIdx.x & (lanes - 1);
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
        store_vec(p.part + (size_t)(2 * ch + (first ? 1 : 0)) * p.d + c, acc);
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] *= p.scale;
        store_vec(p.dtok + (size_t)cur * p.d + c, acc);
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i) acc[i] = 0.f;
    };
    for (int q = b0; q < b1; q += 4) {           // four rows in flight, whatever tokens they belong to
      int2 e[4];
      Pack<T, VEC> x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) if (q + u < b1) e[u] = p.sorted[q + u];
#pragma unroll
      for (int u = 0; u < 4; ++u) if (q + u < b1) x[u].load(dh + (size_t)e[u].x * p.d);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (q + u >= b1) break;
        if ((uint32_t)e[u].y != cur) { flush(); cur = (uint32_t)e[u].y; first = true; }
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] += x[u].v[i];
      }
    }
    flush();
  } else if ((int)blockIdx.x < sum_blocks + pos_blocks) {
    const long long wk = (long long)(blockIdx.x - sum_blocks) * per_block + grp;
    if (wk >= (long long)p.T * pos_pieces) return;
    const int t = (int)(wk / pos_pieces), piece = (int)(wk % pos_pieces);
    long long r = t + (long long)piece * POS_PIECE * p.T;
    float acc[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[i] = 0.f;
    for (int k = 0; k < POS_PIECE; k += 4, r += 4LL * p.T) {
      if (r >= p.rows) break;
      Pack<T, VEC> x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) if (r + (long long)u * p.T < p.rows) x[u].load(dh + (size_t)(r + (long long)u * p.T) * p.d);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (r + (long long)u * p.T < p.rows) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) acc[i] += x[u].v[i];
        }
    }
    store_vec((pos_pieces == 1 ? p.dpos + (size_t)t * p.d : p.pos_part + (size_t)wk * p.d) + c, acc);
  } else {
    const long long t0 = (long long)(blockIdx.x - sum_blocks - pos_blocks) * ZERO_ROWS;
    float z[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) z[i] = 0.f;
    for (int i = grp; i < ZERO_ROWS; i += per_block)
      if (t0 + i < p.vocab && p.seg[t0 + i].y == 0) store_vec(p.dtok + (size_t)(t0 + i) * p.d + c, z);
  }
}

// Pieces of long tokens (and of positions with many rows): eight warps take every eighth piece of 128 columns, the
// eight sums are added in order.
__global__ void __launch_bounds__(256) embed_combine_kernel(EmbedBwdProb p, int P, int chunks, int pos_pieces) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const float* base;
  float* out;
  float scale = 1.f;
  int pieces;
  long long stride;                              // floats between consecutive pieces behind the first
  long long first;                               // offset of piece 0 relative to `base`; piece i > 0 at i * stride
  if ((int)blockIdx.x < chunks) {
    const long long c = blockIdx.x;
    const int last = (int)min((c + 1) * P, (long long)p.rows) - 1;
    const uint32_t e = (uint32_t)p.sorted[last].y;
    if (!(e & HEAVY)) return;
    const int2 sg = p.seg[e & ~HEAVY];
    if (sg.x < c * P) return;                    // that token started in an earlier stretch
    pieces = (sg.y + P - 1) / P;
    base = p.part + (size_t)(2 * c) * p.d;
    first = p.d;
    stride = 2LL * p.d;
    out = p.dtok + (size_t)(e & ~HEAVY) * p.d;
    scale = p.scale;
  } else {
    const int t = (int)blockIdx.x - chunks;
    pieces = (int)(((long long)p.rows - t + (long long)POS_PIECE * p.T - 1) / ((long long)POS_PIECE * p.T));
    if (p.rows <= t) pieces = 0;
    base = p.pos_part + (size_t)t * pos_pieces * p.d;
    first = 0;
    stride = p.d;
    out = p.dpos + (size_t)t * p.d;
  }
  const int c0 = blockIdx.y * 128 + lane;
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = w; i < pieces; i += 8) {
    const float* src = base + (i == 0 ? first : (long long)i * stride);
#pragma unroll
    for (int u = 0; u < 4; ++u) if (c0 + 32 * u < p.d) acc[u] += src[c0 + 32 * u];
  }
  __shared__ float red[8][128];
#pragma unroll
  for (int u = 0; u < 4; ++u) red[w][lane + 32 * u] = acc[u];
  __syncthreads();
  if (threadIdx.x < 128) {
    const int cc = blockIdx.y * 128 + threadIdx.x;
    if (cc < p.d) {
      float s = red[0][threadIdx.x];
#pragma unroll
      for (int i = 1; i < 8; ++i) s += red[i][threadIdx.x];
      out[cc] = s * scale;
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
int piece_rows(int rows) { return rows <= 32768 ? 16 : 64; }
int pos_pieces_for(int rows, int T) { return T > 0 ? (int)(((rows + T - 1) / T + POS_PIECE - 1) / POS_PIECE) : 0; }
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

template <typename T, int VEC>
cudaError_t run_sum(const EmbedBwdProb& p, int P, int chunks, int pos_pieces, cudaStream_t s) {
  const int vecs = (p.d + VEC - 1) / VEC, ll = lanes_log2_for(vecs, 7), per_block = SUM_THREADS >> ll;
  const int sum_blocks = (chunks + per_block - 1) / per_block;
  const long long pos_workers = p.dpos ? (long long)p.T * pos_pieces : 0;
  const long long pos_blocks = (pos_workers + per_block - 1) / per_block;
  const long long zero_blocks = ((long long)p.vocab + ZERO_ROWS - 1) / ZERO_ROWS;
  const dim3 grid((unsigned)(sum_blocks + pos_blocks + zero_blocks), (unsigned)((vecs + (1 << ll) - 1) >> ll));
  return launch_kernel(embed_sum_kernel<T, VEC>, grid, SUM_THREADS, 0, s, p, ll, P, sum_blocks, (int)pos_blocks, pos_pieces);
}

}  // namespace

cudaError_t launch_embed_fwd(const EmbedProb& p, int* d_status, bool is_bf16, cudaStream_t s) {
  const int full = is_bf16 ? 8 : 4;
  const int vec = p.d % full == 0 && aligned16(p.tok, p.pos, p.h) ? full : 1;
  const int ll = lanes_log2_for((p.d + vec - 1) / vec, 5);
  const dim3 grid((unsigned)((((long long)p.rows << ll) + 127) / 128));
  if (is_bf16)
    return vec == 8 ? launch_kernel(embed_fwd_kernel<bf16, 8>, grid, 128, 0, s, p, ll, d_status)
                    : launch_kernel(embed_fwd_kernel<bf16, 1>, grid, 128, 0, s, p, ll, d_status);
  return vec == 4 ? launch_kernel(embed_fwd_kernel<float, 4>, grid, 128, 0, s, p, ll, d_status)
                  : launch_kernel(embed_fwd_kernel<float, 1>, grid, 128, 0, s, p, ll, d_status);
}

// Workspace: sorted rows, token segments, pieces of long tokens, pieces of the position sums.  Pieces of positions are
// stored only if a position has more than POS_PIECE rows; then T < rows / POS_PIECE and T * pieces(T) < 3 rows / POS_PIECE.
size_t embed_bwd_workspace(int rows, int vocab, int d) {
  const size_t chunks = ((size_t)rows + piece_rows(rows) - 1) / piece_rows(rows);
  const size_t pos_rows = 3 * ((size_t)rows / POS_PIECE) + 3;
  return up256((size_t)rows * sizeof(int2)) + up256((size_t)vocab * sizeof(int2)) + up256(2 * chunks * d * sizeof(float)) +
         up256(pos_rows * d * sizeof(float));
}

cudaError_t launch_embed_bwd(EmbedBwdProb p, void* workspace, int* d_status, bool is_bf16, cudaStream_t s) {
  const int P = piece_rows(p.rows), chunks = (int)(((long long)p.rows + P - 1) / P), pos_pieces = p.dpos ? pos_pieces_for(p.rows, p.T) : 0;
  char* w = (char*)workspace;
  p.sorted = (int2*)w;  w += up256((size_t)p.rows * sizeof(int2));
  p.seg = (int2*)w;     w += up256((size_t)p.vocab * sizeof(int2));
  p.part = (float*)w;   w += up256(2 * (size_t)chunks * p.d * sizeof(float));
  p.pos_part = (float*)w;
  int n_log2 = 0;
  while (n_log2 < 7 && (1 << n_log2) < p.vocab) ++n_log2;
  while ((((long long)p.vocab + (1 << n_log2) - 1) >> n_log2) > SORT_MAX_LOCAL) ++n_log2;
  const int local = (int)(((long long)p.vocab + (1 << n_log2) - 1) >> n_log2);
  const size_t smem = ((size_t)SORT_WARPS * (local | 1) + 2 * (size_t)local) * sizeof(int);
  static SmemLimit limit;
  cudaError_t e = limit.raise((const void*)embed_sort_kernel, (SORT_WARPS * (SORT_MAX_LOCAL | 1) + 2 * SORT_MAX_LOCAL) * (int)sizeof(int));
  if (e != cudaSuccess) return e;
  e = launch_kernel(embed_sort_kernel, dim3(1u << n_log2), SORT_WARPS * 32, smem, s, p, n_log2, local, P, d_status);
  if (e != cudaSuccess) return e;
  const int full = is_bf16 ? 8 : 4;
  const bool vec = p.d % full == 0 && aligned16(p.dh, p.dtok, p.dpos);
  if (is_bf16) e = vec ? run_sum<bf16, 8>(p, P, chunks, pos_pieces, s) : run_sum<bf16, 1>(p, P, chunks, pos_pieces, s);
  else e = vec ? run_sum<float, 4>(p, P, chunks, pos_pieces, s) : run_sum<float, 1>(p, P, chunks, pos_pieces, s);
  if (e != cudaSuccess) return e;
  const int long_chunks = p.rows > P ? chunks : 0, long_pos = pos_pieces > 1 ? p.T : 0;
  if (long_chunks + long_pos == 0) return cudaSuccess;
  return launch_kernel(embed_combine_kernel, dim3((unsigned)(long_chunks + long_pos), (unsigned)((p.d + 127) / 128)), 256, 0, s, p, P,
                       long_chunks, pos_pieces);
}

}  // namespace lp
