// Attention over packed sequences of any lengths in fp32, forward and backward, on the fp32 pipes; the
// tensor-core kernels of the bf16 mode are in attention_packed_tc.cu.
//
//   s = scale q k^T, lse = log sum exp s, out = exp(s - lse) v                       (forward)
//   p = exp(s - lse), delta = rowsum(dout * out), ds = p (dout v^T - delta)
//   dv = p^T dout, dk = scale ds^T q, dq = scale ds k                                 (backward)
//
// A block of 128 threads works on 32 x 32 scores at a time, 4 x 2 of them to a thread; operands are
// staged in shared memory, rows behind the end of a sequence are zero there.  Tiles of 64 with 256 threads need
// fewer reads of shared memory for a product, but leave one block of eight warps to an SM and a quarter of the
// blocks.  What bounds it is the wait for a thread's own sums and reads with eight to sixteen warps on an SM:
// 18 TFLOP/s forward and 16 backward at 16 images of 197 rows, 12 heads of 64 (103 and 302 us).  The backward pass has
// two kinds of blocks, one that keeps a tile of keys and walks over the queries (dk, dv) and one that keeps a tile
// of queries and walks over the keys (dq): seven products instead of five, but every gradient is summed by one
// block, or by two and in order, so that results do not depend on the schedule.
#include "vit_internal.h"
#include "attention_packed.cuh"
#include "sm100_ptx.cuh"

namespace vit {

namespace {

constexpr int BT = 32;              // rows and columns of a tile of scores
constexpr int THREADS = 128;
constexpr int PS = BT + 4;          // row stride of a tile of probabilities

__device__ __forceinline__ float4 load4(const float* a) { return *reinterpret_cast<const float4*>(a); }

// rows [row0, row0 + 32) of one head as [32][DP + 4], on their way with cp.async by N threads; rows behind the
// `rows` that exist and columns >= d become zero
template <int DP, int N>
__device__ __forceinline__ void fetch_tile(float* dst, const float* base, int64_t ld, int64_t row0, int rows, int d, int tid) {
  for (int i = tid; i < BT * (DP / 4); i += N) {
    const int r = i / (DP / 4), c = (i % (DP / 4)) * 4;
    const bool there = r < rows && c < d;
    ptx::cp_async_16(ptx::smem_u32(dst + r * (DP + 4) + c), there ? base + (row0 + r) * ld + c : base, there ? 16u : 0u);
  }
}
__device__ __forceinline__ void fetched() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void wait_fetched() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// acc[i][j] = a[ty * 4 + i] . b[tx + 16 j] over the head's channels
template <int DP>
__device__ __forceinline__ void scores(float (&acc)[4][2], const float* a, const float* b, int tx, int ty) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = 0.f;
#pragma unroll 4
  for (int c = 0; c < DP; c += 4) {
    float4 x[4], y[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = load4(a + (ty * 4 + i) * (DP + 4) + c);
#pragma unroll
    for (int j = 0; j < 2; ++j) y[j] = load4(b + (tx + 16 * j) * (DP + 4) + c);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        acc[i][j] = fmaf(x[i].x, y[j].x, fmaf(x[i].y, y[j].y, fmaf(x[i].z, y[j].z, fmaf(x[i].w, y[j].w, acc[i][j]))));
  }
}

// acc[i][cc] += sum over t of w[t][ty * 4 + i] * x[t][2 tx + 32 cc, + 1]      (rows of w and x are the summed index)
template <int DP, int N = BT>
__device__ __forceinline__ void accumulate_t(float2 (&acc)[4][DP / 32], const float* w, const float* x, int tx, int ty) {
#pragma unroll 4
  for (int t = 0; t < N; ++t) {
    const float4 p = load4(w + t * PS + ty * 4);
#pragma unroll
    for (int cc = 0; cc < DP / 32; ++cc) {
      const float2 v = *reinterpret_cast<const float2*>(x + t * (DP + 4) + 2 * tx + 32 * cc);
      acc[0][cc] = __ffma2_rn(make_float2(p.x, p.x), v, acc[0][cc]);
      acc[1][cc] = __ffma2_rn(make_float2(p.y, p.y), v, acc[1][cc]);
      acc[2][cc] = __ffma2_rn(make_float2(p.z, p.z), v, acc[2][cc]);
      acc[3][cc] = __ffma2_rn(make_float2(p.w, p.w), v, acc[3][cc]);
    }
  }
}
// a row's channels of this thread
template <int DP>
__device__ __forceinline__ void store_row(float* dst, const float2 (&acc)[DP / 32], float by, int tx, int d) {
#pragma unroll
  for (int cc = 0; cc < DP / 32; ++cc)
    if (2 * tx + 32 * cc < d) *reinterpret_cast<float2*>(dst + 2 * tx + 32 * cc) = make_float2(acc[cc].x * by, acc[cc].y * by);
}

template <int DP>
__global__ void __launch_bounds__(THREADS)
packed_forward_kernel(const PackedCall c) {
  extern __shared__ __align__(16) float sm[];
  constexpr int TILE = BT * (DP + 4);
  float *qs = sm, *kv_s = qs + TILE, *ps = kv_s + 4 * TILE;   // kv_s: [stage][keys, values]; ps: [key][query]
  const int tiles = (c.p.max_q + BT - 1) / BT;
  const int tile = blockIdx.x % tiles, head = blockIdx.x / tiles % c.p.heads, seq = blockIdx.x / tiles / c.p.heads;
  SeqRange r;
  if (!seq_range(c.p, seq, r, c.dev_status, threadIdx.x == 0)) return;
  const int q0 = tile * BT;
  if (q0 >= r.q_len) return;
  const int q_here = min(BT, r.q_len - q0), d = c.p.d;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int kv = head / (c.p.heads / c.p.kv_heads);
  const float* k = static_cast<const float*>(c.k) + (int64_t)kv * d;
  const float* v = static_cast<const float*>(c.v) + (int64_t)kv * d;
  const float sl2 = c.p.scale * 1.4426950408889634f;
  auto fetch = [&](int k0, int stage) {
    const int here = min(BT, r.k_len - k0);
    fetch_tile<DP, THREADS>(kv_s + 2 * stage * TILE, k, c.ldk, (int64_t)r.k_begin + k0, here, d, threadIdx.x);
    fetch_tile<DP, THREADS>(kv_s + (2 * stage + 1) * TILE, v, c.ldv, (int64_t)r.k_begin + k0, here, d, threadIdx.x);
  };
  fetch_tile<DP, THREADS>(qs, static_cast<const float*>(c.q) + (int64_t)head * d, c.ldq, (int64_t)r.q_begin + q0, q_here, d, threadIdx.x);
  if (r.k_len > 0) fetch(0, 0);
  fetched();
  float m[4], l[4];
  float2 o[4][DP / 32];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int cc = 0; cc < DP / 32; ++cc) o[i][cc] = make_float2(0.f, 0.f);
  }
  int stage = 0;
  for (int k0 = 0; k0 < r.k_len; k0 += BT, stage ^= 1) {
    const int k_here = min(BT, r.k_len - k0);
    const float *ks = kv_s + 2 * stage * TILE, *vs = ks + TILE;
    if (k0 + BT < r.k_len) fetch(k0 + BT, stage ^ 1);
    fetched();
    wait_fetched<1>();
    __syncthreads();
    float s[4][2];
    scores<DP>(s, qs, ks, tx, ty);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float top = m[i];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        s[i][j] = tx + 16 * j < k_here ? s[i][j] * sl2 : -INFINITY;
        top = fmaxf(top, s[i][j]);
      }
#pragma unroll
      for (int x = 8; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
      const float ref = top == -INFINITY ? 0.f : top;      // a row of minus infinities keeps probabilities of zero
      const float keep = exp2f(m[i] - ref);
      m[i] = top;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        s[i][j] = exp2f(s[i][j] - ref);
        sum += s[i][j];
        ps[(tx + 16 * j) * PS + ty * 4 + i] = s[i][j];
      }
      l[i] = l[i] * keep + sum;                            // this lane's part of the row sum
#pragma unroll
      for (int cc = 0; cc < DP / 32; ++cc) o[i][cc] = __fmul2_rn(o[i][cc], make_float2(keep, keep));
    }
    __syncthreads();
    accumulate_t<DP>(o, ps, vs, tx, ty);
    __syncthreads();                                       // this stage and ps may be written again
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int x = 8; x > 0; x >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
    const int row = ty * 4 + i;
    if (row >= q_here) continue;
    const int64_t at = (int64_t)r.q_begin + q0 + row;
    const float inv = l[i] == 0.f ? 0.f : 1.0f / l[i];     // no keys: zero
    store_row<DP>(static_cast<float*>(c.out) + at * c.ldo + (int64_t)head * d, o[i], inv, tx, d);
    if (tx == 0) c.lse[(int64_t)head * c.p.q_rows + at] = l[i] == 0.f ? -INFINITY : (m[i] + log2f(l[i])) * 0.69314718055994531f;
  }
  wait_fetched<0>();
}

// What the other kernels say of bad offsets, for a call that has no rows to work on
__global__ void __launch_bounds__(THREADS)
check_offsets_kernel(const PackedCall c) {
  SeqRange r;
  for (int64_t i = (int64_t)blockIdx.x * THREADS + threadIdx.x; i < c.p.sequences; i += (int64_t)gridDim.x * THREADS)
    seq_range(c.p, (int)i, r, c.dev_status, true);
}

// (lse log2(e), delta)[head][row], delta = sum over the head's channels of dout * out, of the rows of the sequences
// that the gradients accept and of no others.  A block takes a few rows of one head, a warp two of them.
constexpr int DELTA_ROWS = 2 * THREADS / 32;
__global__ void __launch_bounds__(THREADS)
packed_delta_kernel(const PackedCall c) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int tiles = (c.p.max_q + DELTA_ROWS - 1) / DELTA_ROWS;
  const int head = blockIdx.x % c.p.heads, tile = blockIdx.x / c.p.heads % tiles, seq = blockIdx.x / c.p.heads / tiles;
  SeqRange r;
  if (!seq_range(c.p, seq, r, c.dev_status, threadIdx.x == 0)) return;
  const int lane = threadIdx.x & 31, row0 = tile * DELTA_ROWS + 2 * (int)(threadIdx.x >> 5);
  const int64_t col = (int64_t)head * c.p.d + lane * 4;
  float4 a[2], b[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    a[i] = b[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (row0 + i < r.q_len && lane * 4 < c.p.d) {
      const int64_t row = (int64_t)r.q_begin + row0 + i;
      a[i] = load4(static_cast<const float*>(c.out) + row * c.ldo + col);
      b[i] = load4(static_cast<const float*>(c.dout) + row * c.lddo + col);
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (row0 + i >= r.q_len) return;                       // the same for the whole warp
    float sum = fmaf(a[i].x, b[i].x, fmaf(a[i].y, b[i].y, fmaf(a[i].z, b[i].z, a[i].w * b[i].w)));
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
    const int64_t at = (int64_t)head * c.p.q_rows + r.q_begin + row0 + i;
    if (lane == 0) c.delta[at] = make_float2(c.lse[at] * 1.4426950408889634f, sum);
  }
}

// The gradient kernels have two groups of 128 threads: one has the scores and their probabilities, the other the
// gradients of the probabilities; then each has one sum (dv and dk, or half of the keys for dq).
// Where there are few blocks, a tile's walk is shared out over a cluster of two, whose sums are joined in the first
// one's shared memory, in order: 115 -> 76 us at 5 images of up to 257 rows, 4 heads of 80 (dq, dk and dv, delta),
// 898 -> 576 us at 1 x 1024 rows, 8 heads of 128 on 2. A cluster of four's sums do not fit there at 128 channels.
constexpr int GRAD_THREADS = 2 * THREADS;
constexpr int MAX_SPLITS = 2;
template <int DP>                                           // all groups' sums but the first one's, over the tiles and ps, ds
constexpr bool SUMS_FIT = (size_t)(2 * MAX_SPLITS - 1) * 4 * (DP / 32) * THREADS * sizeof(float2) <= sizeof(float) * (6 * BT * (DP + 4) + 2 * BT * PS);

// This thread's sums to slot `slot` of the cluster's first block, and from there: [slot][value][thread]
template <int DP>
__device__ __forceinline__ void push_sums(float* slots, int slot, int tid, const float2 (&acc)[4][DP / 32]) {
  const uint32_t base = ptx::map_to_cta(ptx::smem_u32(slots) + (uint32_t)((slot * 4 * (DP / 32) * THREADS + tid) * 8), 0);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int cc = 0; cc < DP / 32; ++cc)
      asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(base + (uint32_t)((i * (DP / 32) + cc) * THREADS * 8)), "f"(acc[i][cc].x),
                   "f"(acc[i][cc].y) : "memory");
}
template <int DP>
__device__ __forceinline__ void add_sums(const float* slots, int slot, int tid, float2 (&acc)[4][DP / 32]) {
  const float2* from = reinterpret_cast<const float2*>(slots) + slot * 4 * (DP / 32) * THREADS + tid;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int cc = 0; cc < DP / 32; ++cc) acc[i][cc] = __fadd2_rn(acc[i][cc], from[(i * (DP / 32) + cc) * THREADS]);
}

// One tile's P (by group 0) and dS (by group 1): [row of w][column of w] as the sums want it
template <int DP, bool BY_QUERY>
__device__ __forceinline__ void grad_scores(float* ps, float* ds, const float* qs, const float* os, const float* ks, const float* vs,
                                            const float2* rows, float sl2, int q_here, int k_here, int group, int tx, int ty) {
  float s[4][2];
  scores<DP>(s, group ? os : qs, group ? vs : ks, tx, ty);
  auto place = [&](int i, int j) { return BY_QUERY ? (ty * 4 + i) * PS + tx + 16 * j : (tx + 16 * j) * PS + ty * 4 + i; };
  if (group == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const bool there = ty * 4 + i < q_here && tx + 16 * j < k_here;
        ps[place(i, j)] = there ? exp2f(fmaf(s[i][j], sl2, -rows[ty * 4 + i].x)) : 0.f;
      }
  }
  __syncthreads();
  if (group == 1) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const bool there = ty * 4 + i < q_here && tx + 16 * j < k_here;
        ds[place(i, j)] = there ? ps[place(i, j)] * (s[i][j] - rows[ty * 4 + i].y) : 0.f;
      }
  }
}

template <int DP>
__device__ __forceinline__ void dkdv_tile(const PackedCall& c, int splits, int block) {
  static_assert(SUMS_FIT<DP>, "the joined sums lie over the tiles");
  extern __shared__ __align__(16) float sm[];
  constexpr int TILE = BT * (DP + 4);
  float *ks = sm, *vs = ks + TILE, *qo = vs + TILE, *ps = qo + 4 * TILE, *ds = ps + BT * PS;   // qo: [stage][q, dout]; ps, ds: [query][key]
  float2* rows = reinterpret_cast<float2*>(ds + BT * PS);                                      // [stage][32]: lse log2(e), delta
  const int tiles = (c.p.max_k + BT - 1) / BT;
  const int rank = block % splits, item = block / splits;
  const int tile = item % tiles, kv = item / tiles % c.p.kv_heads, seq = item / tiles / c.p.kv_heads;
  SeqRange r;
  if (!seq_range(c.p, seq, r, c.dev_status, threadIdx.x == 0)) return;
  const int k0 = tile * BT;
  if (k0 >= r.k_len) return;
  const int k_here = min(BT, r.k_len - k0), d = c.p.d, heads = c.p.heads / c.p.kv_heads;
  const int group = threadIdx.x / THREADS, tid = threadIdx.x % THREADS, tx = tid & 15, ty = tid >> 4;
  const float sl2 = c.p.scale * 1.4426950408889634f;
  const int q_tiles = (r.q_len + BT - 1) / BT, whole = heads * q_tiles;
  const int first = (int)((int64_t)whole * rank / splits), n = (int)((int64_t)whole * (rank + 1) / splits);
  auto fetch = [&](int t, int stage) {                      // queries (group 0) or their dout (group 1), and their numbers
    const int head = kv * heads + t / q_tiles, q0 = t % q_tiles * BT, here = min(BT, r.q_len - q0);
    const int64_t at = (int64_t)r.q_begin + q0;
    if (group == 0) fetch_tile<DP, THREADS>(qo + 2 * stage * TILE, static_cast<const float*>(c.q) + (int64_t)head * d, c.ldq, at, here, d, tid);
    else fetch_tile<DP, THREADS>(qo + (2 * stage + 1) * TILE, static_cast<const float*>(c.dout) + (int64_t)head * d, c.lddo, at, here, d, tid);
    if (group == 0 && tid < here) rows[stage * BT + tid] = c.delta[(int64_t)head * c.p.q_rows + at + tid];
  };
  if (group == 0) fetch_tile<DP, THREADS>(ks, static_cast<const float*>(c.k) + (int64_t)kv * d, c.ldk, (int64_t)r.k_begin + k0, k_here, d, tid);
  else fetch_tile<DP, THREADS>(vs, static_cast<const float*>(c.v) + (int64_t)kv * d, c.ldv, (int64_t)r.k_begin + k0, k_here, d, tid);
  if (n > first) fetch(first, 0);
  fetched();
  float2 acc[4][DP / 32];                                   // of dv (group 0) or dk (group 1)
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int cc = 0; cc < DP / 32; ++cc) acc[i][cc] = make_float2(0.f, 0.f);
  for (int t = first; t < n; ++t) {
    const int stage = (t - first) & 1, q_here = min(BT, r.q_len - t % q_tiles * BT);
    if (t + 1 < n) fetch(t + 1, stage ^ 1);
    fetched();
    wait_fetched<1>();
    __syncthreads();
    const float *qs = qo + 2 * stage * TILE, *os = qs + TILE;
    grad_scores<DP, true>(ps, ds, qs, os, ks, vs, rows + stage * BT, sl2, q_here, k_here, group, tx, ty);
    if (group == 0) accumulate_t<DP>(acc, ps, os, tx, ty);
    else asm volatile("bar.sync 1, 128;" ::: "memory");     // ds is written and read by this group alone
    if (group == 1) accumulate_t<DP>(acc, ds, qs, tx, ty);
    __syncthreads();                                        // this stage, ps and ds may be written again
  }
  wait_fetched<0>();
  if (splits > 1) {
    ptx::cluster_sync();                                    // the first block's tiles are no longer needed
    if (rank > 0) push_sums<DP>(sm, 2 * (rank - 1) + group, tid, acc);
    ptx::cluster_sync();
    if (rank > 0) return;
    for (int i = 1; i < splits; ++i) add_sums<DP>(sm, 2 * (i - 1) + group, tid, acc);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = ty * 4 + i;
    if (row >= k_here) continue;
    const int64_t at = (int64_t)r.k_begin + k0 + row;
    if (group == 0) store_row<DP>(static_cast<float*>(c.dv) + at * c.lddv + (int64_t)kv * d, acc[i], 1.f, tx, d);
    else store_row<DP>(static_cast<float*>(c.dk) + at * c.lddk + (int64_t)kv * d, acc[i], gradient_scale(c.p, r.k_len), tx, d);
  }
}

template <int DP>
__device__ __forceinline__ void dq_tile(const PackedCall& c, int splits, int block) {
  static_assert(SUMS_FIT<DP>, "the joined sums lie over the tiles");
  extern __shared__ __align__(16) float sm[];
  constexpr int TILE = BT * (DP + 4);
  float *qs = sm, *os = qs + TILE, *kv_s = os + TILE, *ps = kv_s + 4 * TILE, *ds = ps + BT * PS;    // kv_s: [stage][k, v]; ps, ds: [key][query]
  float2* rows = reinterpret_cast<float2*>(ds + BT * PS);
  const int tiles = (c.p.max_q + BT - 1) / BT;
  const int rank = block % splits, item = block / splits;
  const int tile = item % tiles, head = item / tiles % c.p.heads, seq = item / tiles / c.p.heads;
  SeqRange r;
  if (!seq_range(c.p, seq, r, c.dev_status, threadIdx.x == 0)) return;
  const int q0 = tile * BT;
  if (q0 >= r.q_len) return;
  const int q_here = min(BT, r.q_len - q0), d = c.p.d, kv = head / (c.p.heads / c.p.kv_heads);
  const int group = threadIdx.x / THREADS, tid = threadIdx.x % THREADS, tx = tid & 15, ty = tid >> 4;
  const float sl2 = c.p.scale * 1.4426950408889634f;
  const int64_t at = (int64_t)r.q_begin + q0;
  const float* base = static_cast<const float*>(group ? c.v : c.k) + (int64_t)kv * d;
  auto fetch = [&](int k0, int stage) {                     // keys (group 0) or values (group 1)
    fetch_tile<DP, THREADS>(kv_s + (2 * stage + group) * TILE, base, group ? c.ldv : c.ldk, (int64_t)r.k_begin + k0, min(BT, r.k_len - k0), d, tid);
  };
  if (group == 0) fetch_tile<DP, THREADS>(qs, static_cast<const float*>(c.q) + (int64_t)head * d, c.ldq, at, q_here, d, tid);
  else fetch_tile<DP, THREADS>(os, static_cast<const float*>(c.dout) + (int64_t)head * d, c.lddo, at, q_here, d, tid);
  const int k_tiles = (r.k_len + BT - 1) / BT;
  const int first = (int)((int64_t)k_tiles * rank / splits) * BT, end = min(r.k_len, (int)((int64_t)k_tiles * (rank + 1) / splits) * BT);
  if (first < end) fetch(first, 0);
  fetched();
  if (group == 0 && tid < q_here) rows[tid] = c.delta[(int64_t)head * c.p.q_rows + at + tid];
  float2 acc[4][DP / 32];                                   // of dq, over one half of every tile's keys
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int cc = 0; cc < DP / 32; ++cc) acc[i][cc] = make_float2(0.f, 0.f);
  int stage = 0;
  for (int k0 = first; k0 < end; k0 += BT, stage ^= 1) {
    const int k_here = min(BT, r.k_len - k0);
    if (k0 + BT < end) fetch(k0 + BT, stage ^ 1);
    fetched();
    wait_fetched<1>();
    __syncthreads();
    const float *ks = kv_s + 2 * stage * TILE, *vs = ks + TILE;
    grad_scores<DP, false>(ps, ds, qs, os, ks, vs, rows, sl2, q_here, k_here, group, tx, ty);
    __syncthreads();
    accumulate_t<DP, BT / 2>(acc, ds + group * (BT / 2) * PS, ks + group * (BT / 2) * (DP + 4), tx, ty);
    __syncthreads();                                        // this stage, ps and ds may be written again
  }
  // the halves, in order: of the cluster's blocks and of their groups
  wait_fetched<0>();
  if (splits > 1) ptx::cluster_sync();                      // the first block's tiles are no longer needed
  else __syncthreads();
  if (rank + group > 0) push_sums<DP>(sm, 2 * rank + group - 1, tid, acc);
  if (splits > 1) ptx::cluster_sync();
  else __syncthreads();
  if (rank + group > 0) return;
  for (int i = 1; i < 2 * splits; ++i) add_sums<DP>(sm, i - 1, tid, acc);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (ty * 4 + i < q_here) store_row<DP>(static_cast<float*>(c.dq) + (at + ty * 4 + i) * c.lddq + (int64_t)head * d, acc[i], gradient_scale(c.p, r.k_len), tx, d);
}

// Both in one launch: neither fills the device by itself where there are few rows, and neither waits for the other's
// last blocks.  The first `dkdv_blocks` have dk and dv.  (5 images of up to 257 rows, 4 heads of 80:
// 74 us in two launches, 58 in one; 16 images of 197, 12 heads of 64: 328 and 301.)
template <int DP>
__global__ void __launch_bounds__(GRAD_THREADS)
packed_grads_kernel(const PackedCall c, int splits, int dkdv_blocks) {
  asm volatile("griddepcontrol.wait;" ::: "memory");       // launched while the kernel that leaves delta ends
  if ((int)blockIdx.x < dkdv_blocks) dkdv_tile<DP>(c, splits, blockIdx.x);
  else dq_tile<DP>(c, splits, blockIdx.x - dkdv_blocks);
}


template <int DP>
cudaError_t launch_forward(const PackedCall& c, cudaStream_t s) {
  constexpr size_t smem = 5 * (size_t)BT * (DP + 4) * 4 + (size_t)BT * PS * 4;
  static PerDeviceFlag done;
  if (cudaError_t e = ensure_dynamic_smem(done, packed_forward_kernel<DP>, (int)smem)) return e;
  packed_forward_kernel<DP><<<(unsigned)(c.p.sequences * c.p.heads * ((c.p.max_q + BT - 1) / BT)), THREADS, smem, s>>>(c);
  return cudaGetLastError();
}

template <int DP>
cudaError_t launch_grads(const PackedCall& c, cudaStream_t s) {
  constexpr size_t smem = 6 * (size_t)BT * (DP + 4) * 4 + 2 * (size_t)BT * PS * 4 + 2 * BT * sizeof(float2);
  static PerDeviceFlag done;
  if (cudaError_t e = ensure_dynamic_smem(done, packed_grads_kernel<DP>, (int)smem)) return e;
  const int64_t q_tiles = (c.p.max_q + BT - 1) / BT, k_tiles = (c.p.max_k + BT - 1) / BT, sequences = c.p.sequences;
  const int64_t dkdv = c.p.k_rows > 0 ? sequences * c.p.kv_heads * k_tiles : 0, dq = c.p.q_rows > 0 ? sequences * c.p.heads * q_tiles : 0;
  // Two blocks share a tile's walk (of four tiles or more) where that takes a sixth of the rounds away.  Two blocks to an SM
  // are counted for every head size: so many fit from 65 channels on, where this was measured (80 and 128); three do below.
  const int64_t wave = 2 * 148, rounds = (dkdv + dq + wave - 1) / wave, halves = (2 * (dkdv + dq) + wave - 1) / wave;
  const int splits = 3 * halves <= 5 * rounds && k_tiles >= 4 && c.p.heads / c.p.kv_heads * q_tiles >= 4 ? MAX_SPLITS : 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((dkdv + dq) * splits));
  cfg.blockDim = dim3(GRAD_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  int attrs = 0;
  if (splits > 1) {
    attr[attrs].id = cudaLaunchAttributeClusterDimension;
    attr[attrs].val.clusterDim.x = (unsigned)splits;
    attr[attrs].val.clusterDim.y = attr[attrs].val.clusterDim.z = 1;
    ++attrs;
  }
  // Launched while delta's kernel ends, if there is one and every SM gets two blocks: 63 -> 58 us at 5 images of up to 257
  // rows, 4 heads of 80.  Fewer would be put two to an SM beside its last blocks: 18.6 -> 28.7 us at 2 images of 70, 4 of 64.
  if (c.p.q_rows > 0 && c.p.max_q > 0 && (dkdv + dq) * splits >= 2 * 148) {
    attr[attrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[attrs].val.programmaticStreamSerializationAllowed = 1;
    ++attrs;
  }
  cfg.attrs = attr;
  cfg.numAttrs = (unsigned)attrs;
  return cudaLaunchKernelEx(&cfg, packed_grads_kernel<DP>, c, splits, (int)(dkdv * splits));
}

}  // namespace

cudaError_t launch_attention_packed_f32(const PackedCall& c, cudaStream_t s) {
  return c.p.d <= 32 ? launch_forward<32>(c, s) : c.p.d <= 64 ? launch_forward<64>(c, s) : c.p.d <= 96 ? launch_forward<96>(c, s) : launch_forward<128>(c, s);
}

cudaError_t launch_check_offsets(const PackedCall& c, cudaStream_t s) {
  const int blocks = (int)(((int64_t)c.p.sequences + THREADS - 1) / THREADS);
  check_offsets_kernel<<<(unsigned)(blocks < 1024 ? blocks : 1024), THREADS, 0, s>>>(c);
  return cudaGetLastError();
}
cudaError_t launch_attention_delta_f32(const PackedCall& c, cudaStream_t s) {
  packed_delta_kernel<<<(unsigned)(c.p.sequences * c.p.heads * ((c.p.max_q + DELTA_ROWS - 1) / DELTA_ROWS)), THREADS, 0, s>>>(c);
  return cudaGetLastError();
}
cudaError_t launch_attention_packed_grads_f32(const PackedCall& c, cudaStream_t s) {
  return c.p.d <= 32 ? launch_grads<32>(c, s) : c.p.d <= 64 ? launch_grads<64>(c, s) : c.p.d <= 96 ? launch_grads<96>(c, s) : launch_grads<128>(c, s);
}

}  // namespace vit
