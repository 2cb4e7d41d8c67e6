// Attention over packed sequences on the 5th-generation tensor cores (bf16), forward and backward, for
// sequences of any length and head sizes 16 ... 128.
//
// Operands are fetched by TMA through three-dimensional maps (channel of the head, head, row) in slabs of
// 64 channels, 128-byte swizzled; channels beyond the head come as zeros, so that one layout serves every
// head size and the products run over the head's own channels only.  Scores and accumulators live in
// tensor memory; probabilities (and the scores' gradients) are written back over the scores as packed bf16
// and are the A operand of the second products, so that nothing of the score matrix leaves the SM.  One
// thread owns one row of a tile of scores.
//
// Persistent blocks, one per SM, walk over the work with a static schedule; the operands of the next piece
// are fetched while the last one is finished.  A tile of queries (or of whatever stays) is held in tensor
// memory too where it fits, as the A operand of the scores: with both operands in shared memory a product
// of 128 x 64 x 16 reads 6 KB there in the 32 cycles that it takes, more than the 128 bytes a cycle that
// shared memory gives, and holds up everything else that goes through it.
//
// Every mbarrier wait is bounded; on expiry the block raises the device status word, lets the copies and
// products in flight finish (bounded), frees tensor memory and leaves.
#include "vit_internal.h"
#include "attention_packed.cuh"
#include "sm100_ptx.cuh"

#include <cuda.h>

namespace vit {

namespace {

using namespace ptx;

constexpr int RT = 128;                                // rows of a tile of scores = lanes of tensor memory
constexpr int CT = 64;                                 // columns of a tile of scores
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.69314718055994531f;
constexpr long long DRAIN_LIMIT_CYCLES = 1ll << 24;    // teardown after a failed wait: ~10 ms
constexpr long long LONG_WAIT_CYCLES = WAIT_LIMIT_CYCLES << 8;   // for other pieces, whose own waits are bounded

// Shared-memory matrix descriptor of a 128-byte-swizzled slab (rows of 128 bytes, groups of 8 rows 1024
// bytes apart).  lbo: distance of the slabs of 64 columns, for an operand whose rows are the summed index
// (K) and that is wider than one slab.
__device__ __forceinline__ uint64_t desc_sw128(uint32_t saddr, uint32_t lbo = 16) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)((lbo >> 4) & 0x3FFFu) << 16) | ((uint64_t)(1024 >> 4) << 32) |
         ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ uint32_t idesc(int n, bool b_rows_are_k) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (b_rows_are_k ? (1u << 16) : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(RT >> 4) << 24);
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&h);
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* tm, int c, int head, int row, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(tm)), "r"(c), "r"(head), "r"(row), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* tm) { asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(tm)) : "memory"); }
// a bounded wait of a whole warp: all lanes leave with the same answer.  Only the first look is in line: the
// kernels wait in many places, and their code has to fit the instruction cache.
__device__ __noinline__ bool wait_on(uint32_t bar, int parity, volatile int* abort_flag, long long limit) {
  return mbar_wait_limit(bar, (uint32_t)parity, abort_flag, limit);
}
__device__ __forceinline__ bool warp_wait(uint32_t bar, int parity, volatile int* abort_flag, long long limit = WAIT_LIMIT_CYCLES) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, (uint32_t)parity))) return true;
  return __all_sync(0xffffffffu, wait_on(bar, parity, abort_flag, limit));
}
// rows [from, rows) of a tile of `slabs` slabs become zero; one warp, then visible to the tensor core
__device__ __forceinline__ void zero_rows(uint32_t tile, int rows, int slabs, int from, int lane) {
  for (int s = 0; s < slabs; ++s)
    for (int i = from * 8 + lane; i < rows * 8; i += 32)
      asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(tile + (uint32_t)(s * rows * 128 + i * 16)), "r"(0u) : "memory");
  fence_proxy_async_smem();
  __syncwarp();
}

// waits for tensor-memory loads and names their registers, so that nothing reads them before
__device__ __forceinline__ void tmem_ld_wait_16(uint32_t (&r)[16], uint32_t (&t)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                 "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(t[0]), "+r"(t[1]), "+r"(t[2]),
                 "+r"(t[3]), "+r"(t[4]), "+r"(t[5]), "+r"(t[6]), "+r"(t[7]), "+r"(t[8]), "+r"(t[9]), "+r"(t[10]), "+r"(t[11]),
                 "+r"(t[12]), "+r"(t[13]), "+r"(t[14]), "+r"(t[15])
               :
               : "memory");
}
// One lane of the warp, chosen by the hardware.  The products are issued behind this and not behind
// `lane == 0`: their operands then stay in uniform registers (110 cycles -> what the product itself takes, 31 at 64 columns).
__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.b32 %0, 1, 0, p;\n}\n" : "=r"(one));
  return one != 0;
}
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __shfl_sync(0xffffffffu, v, 0); }

// S[128 x n] = X[128 rows] . Y[n rows]^T over the head's channels; X in tensor memory (packed pairs) or in
// shared memory, as slabs of 64 channels like Y (whose tiles have Y_ROWS rows)
template <int SLABS, int Y_ROWS>
__device__ __forceinline__ void issue_scores_ts(uint32_t d_tmem, uint32_t x_tmem, uint32_t y, int n, int ksteps) {
  const uint32_t id = idesc(n, false);
  const uint64_t yd = desc_sw128(y);
#pragma unroll
  for (int k = 0; k < 4 * SLABS; ++k)
    if (k < ksteps) umma_bf16_ts(d_tmem, x_tmem + (uint32_t)(8 * k), yd + (uint64_t)((k >> 2) * (Y_ROWS * 8) + 2 * (k & 3)), id, k > 0 ? 1u : 0u);
}
template <int SLABS, int Y_ROWS>
__device__ __forceinline__ void issue_scores_ss(uint32_t d_tmem, uint32_t x, uint32_t y, int n, int ksteps) {
  const uint32_t id = idesc(n, false);
  const uint64_t xd = desc_sw128(x), yd = desc_sw128(y);
#pragma unroll
  for (int k = 0; k < 4 * SLABS; ++k)
    if (k < ksteps)
      umma_bf16(d_tmem, xd + (uint64_t)((k >> 2) * (RT * 8) + 2 * (k & 3)), yd + (uint64_t)((k >> 2) * (Y_ROWS * 8) + 2 * (k & 3)), id,
                k > 0 ? 1u : 0u);
}
// D[128 x d] (+)= P[128 x 64] . Y[64 rows x d], `ksteps` of the four steps of 16 rows; P packed in tensor memory, in
// 32 columns or (HALVES) in 16 at the start of each half of 64; y: the first of the 64 rows in a tile of Y_ROWS
template <int Y_ROWS, bool HALVES>
__device__ __forceinline__ void issue_weighted(uint32_t d_tmem, uint32_t p_tmem, uint32_t y, int d, int ksteps, bool first) {
  const uint32_t id = idesc(d, true);
  const uint64_t yd = desc_sw128(y, Y_ROWS * 128);
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (k < ksteps) umma_bf16_ts(d_tmem, p_tmem + (uint32_t)(8 * k + (HALVES && k >= 2 ? 16 : 0)), yd + (uint64_t)(k * 128), id, first && k == 0 ? 0u : 1u);
}
// The 16 channels 16 g ... of a row of a swizzled tile of 128 rows in shared memory
__device__ __forceinline__ void read_16(uint32_t (&w)[8], uint32_t tile, int row, int g) {
  const uint32_t at = tile + (uint32_t)((g >> 2) * RT * 128 + row * 128);
  const int c = 2 * (g & 3), x = row & 7;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at + (uint32_t)((c ^ x) << 4)));
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "r"(at + (uint32_t)(((c + 1) ^ x) << 4)));
}
// A row of a tile from shared memory into tensor memory.  Rows behind the end of a sequence bring whatever lies
// there: every row of a product depends on its own row of this operand only.
template <int SLABS>
__device__ __forceinline__ void row_to_tmem(uint32_t taddr, uint32_t tile, int row, int d) {
#pragma unroll
  for (int g = 0; g < 4 * SLABS; ++g)
    if (g < d / 16) {
      uint32_t w[8];
      read_16(w, tile, row, g);
      tmem_st8(taddr + (uint32_t)(8 * g), w);
    }
}
__device__ __forceinline__ float dot2(uint32_t a, uint32_t b, float acc) {
  acc = fmaf(__uint_as_float(a << 16), __uint_as_float(b << 16), acc);
  return fmaf(__uint_as_float(a & 0xffff0000u), __uint_as_float(b & 0xffff0000u), acc);
}

// The accumulator rows of a warp (32 rows, columns [0, cols)) times a factor per row to global memory.  A row
// belongs to a lane, and lanes that wrote their rows themselves would touch 32 lines with every store: the
// rows go through 2 KB of shared memory, 32 columns at a time, and leave as 64 bytes each of eight rows.
// stage: this warp's 2 KB; rows: how many of the 32 exist; dst: row 0, its columns; ld in elements.
__device__ __forceinline__ void store_rows(bf16* dst, int64_t ld, uint32_t taddr, int cols, float by, int rows, uint32_t stage, int lane) {
  for (int c = 0; c < cols; c += 32) {
    uint32_t o[2][16];
    tmem_ld16(taddr + (uint32_t)c, o[0]);
    if (c + 16 < cols) tmem_ld16(taddr + (uint32_t)(c + 16), o[1]);
    tmem_ld_wait_16(o[0], o[1]);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[e] = pack_bf16(__uint_as_float(o[q >> 1][8 * (q & 1) + 2 * e]) * by, __uint_as_float(o[q >> 1][8 * (q & 1) + 2 * e + 1]) * by);
      // 16-byte piece q of this lane's row, turned by the row so that eight lanes meet different banks
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stage + (uint32_t)(lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4))), "r"(w[0]),
                   "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
    }
    __syncwarp();
    const int q = lane & 3;
    uint4 v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 8 * e + (lane >> 2);
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[e].x), "=r"(v[e].y), "=r"(v[e].z), "=r"(v[e].w)
                   : "r"(stage + (uint32_t)(r * 64 + ((q ^ ((r >> 1) & 3)) << 4))));
    }
    __syncwarp();
    if (c + 8 * q < cols) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (8 * e + (lane >> 2) < rows) *reinterpret_cast<uint4*>(dst + (8 * e + (lane >> 2)) * ld + c + 8 * q) = v[e];
    }
  }
}

// the same in fp32, 16 columns at a time
__device__ __forceinline__ void store_rows(float* dst, int64_t ld, uint32_t taddr, int cols, float by, int rows, uint32_t stage, int lane) {
  for (int c = 0; c < cols; c += 16) {
    uint32_t o[16];
    tmem_ld16(taddr + (uint32_t)c, o);
    tmem_ld_wait();
    asm volatile("" : "+r"(o[0]), "+r"(o[1]), "+r"(o[2]), "+r"(o[3]), "+r"(o[4]), "+r"(o[5]), "+r"(o[6]), "+r"(o[7]), "+r"(o[8]), "+r"(o[9]),
                 "+r"(o[10]), "+r"(o[11]), "+r"(o[12]), "+r"(o[13]), "+r"(o[14]), "+r"(o[15]));      // nothing reads them before the wait
#pragma unroll
    for (int q = 0; q < 4; ++q)
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stage + (uint32_t)(lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4))), "r"(o[4 * q]),
                   "r"(o[4 * q + 1]), "r"(o[4 * q + 2]), "r"(o[4 * q + 3]) : "memory");
    __syncwarp();
    const int q = lane & 3;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 8 * e + (lane >> 2);
      float4 v;
      asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                   : "r"(stage + (uint32_t)(r * 64 + ((q ^ ((r >> 1) & 3)) << 4))));
      if (r < rows) *reinterpret_cast<float4*>(dst + r * ld + c + 4 * q) = make_float4(v.x * by, v.y * by, v.z * by, v.w * by);
    }
    __syncwarp();
  }
}

// A piece of work: rows [x0, x0 + span) of one head of one sequence against tiles [t_begin, t_begin + n) of what they meet.
struct Piece { int head, x0; SeqRange r; int t_begin, n; };
// Which pieces a block gets.  `blocks` = 0: whole ones, in rounds of one to every block, every other round in the
// other direction (128 images of 257 rows: a block would get all of one kind, 256 rows or one).  Else `blocks` blocks share all tiles equally, one piece
// after the other, so that a block's first and last piece may be parts; a piece counts for `least` tiles at least,
// which bounds their number in a block.
struct Order { int span; bool of_keys; int heads, repeats /* of the tiles that a piece meets */, blocks, least; };
// A block's pieces are looked up once, at its start.
constexpr int MAX_PIECES = 128, SEQ_CHUNK = 512, SCAN_INTS = SEQ_CHUNK + 4 + SEQ_CHUNK / 32;   // of a block; sequences looked at together; scan_sequences' `before`
constexpr uint32_t TABLE_BYTES = MAX_PIECES * 32;
__device__ __forceinline__ Piece piece_at(uint32_t table, int n) {
  Piece w;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.head), "=r"(w.x0), "=r"(w.r.q_begin), "=r"(w.r.q_len) : "r"(table + 32u * n));
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.r.k_begin), "=r"(w.r.k_len), "=r"(w.t_begin), "=r"(w.n) : "r"(table + 32u * n + 16));
  return w;
}
__device__ __forceinline__ int tiles_met(const Order& o, const int4& r) { return o.repeats * (((o.of_keys ? r.y : r.w) + CT - 1) / CT); }
__device__ __forceinline__ int piece_weight(const Order& o, const int4& r) { return o.blocks > 0 ? max(tiles_met(o, r), o.least) : 1; }
// Sequences [s0, s0 + chunk), by all threads of a block: ranges (q_begin, q_len, k_begin, k_len), and the weight of all pieces
// before each of them.  Returns that behind the last one.
__device__ __forceinline__ int scan_sequences(const vit_attention_problem& p, int* status, const Order& o, int s0, int chunk, int carry, int32_t* before, int4* ranges) {
  __syncthreads();                                               // `before` is read no more
  const int warps = (int)blockDim.x / 32, warp = (int)threadIdx.x / 32, lane = (int)threadIdx.x & 31;
  for (int b = warp * 32; b < chunk; b += warps * 32) {          // running sums of 32 sequences each
    const int s = b + lane;
    SeqRange r{0, 0, 0, 0};
    if (s < chunk) seq_range(p, s0 + s, r, status, true);
    const int4 v = make_int4(r.q_begin, r.q_len, r.k_begin, r.k_len);
    const int n = ((o.of_keys ? r.k_len : r.q_len) + o.span - 1) / o.span * o.heads * piece_weight(o, v);
    int up = n;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int lower = __shfl_up_sync(0xffffffffu, up, d);
      if (lane >= d) up += lower;
    }
    if (s < chunk) {
      before[s] = up - n;
      ranges[s] = v;
    }
    if (lane == 31) before[SEQ_CHUNK + 4 + b / 32] = up;
  }
  __syncthreads();
  int sum = carry, mine = 0;                                     // and of all of them
  for (int b = 0; b < chunk; b += 32) {
    if (b == warp * 32) mine = sum;
    sum += before[SEQ_CHUNK + 4 + b / 32];
  }
  for (int b = warp * 32, at = mine; b < chunk; b += warps * 32) {
    if (b + lane < chunk) before[b + lane] += at;
    for (int k = b; k < b + warps * 32 && k < chunk; k += 32) at += before[SEQ_CHUNK + 4 + k / 32];
  }
  if (threadIdx.x == 0) before[chunk] = sum;
  __syncthreads();
  return sum;
}
// the last of `chunk` sequences with before[...] <= i
__device__ __forceinline__ int sequence_of(const int32_t* before, int chunk, int i) {
  int lo = 0, hi = chunk;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (before[mid] <= i) lo = mid;
    else hi = mid;
  }
  return lo;
}
__device__ __forceinline__ int share_begin(int total, int block, int blocks) { return (int)((int64_t)total * block / blocks); }
__device__ __forceinline__ int share_of(int total, int tile, int blocks) { return (int)(((int64_t)(tile + 1) * blocks - 1) / total); }   // whose it is

// All threads of the block; ends with a barrier.  before: shared memory for SCAN_INTS + 4 SEQ_CHUNK numbers that is not needed
// afterwards.  Returns the number of the block's pieces.
__device__ __forceinline__ int find_pieces(const vit_attention_problem& p, int* status, const Order& o, int32_t* table, int32_t* before) {
  int4* ranges = reinterpret_cast<int4*>(before + SCAN_INTS);
  auto put = [&](int j, const int4& r, int k, int t_begin, int n) {     // piece k of a sequence
    const int tiles = ((o.of_keys ? r.w : r.y) + o.span - 1) / o.span, head = k / tiles;
    int4* to = reinterpret_cast<int4*>(table + 8 * j);
    to[0] = make_int4(head, (k - head * tiles) * o.span, r.x, r.y);
    to[1] = make_int4(r.z, r.w, t_begin, n);
  };
  const int grid = (int)gridDim.x, self = (int)blockIdx.x;
  int carry = 0, found = 0;
  if (o.blocks == 0) {
    for (int s0 = 0; s0 < p.sequences; s0 += SEQ_CHUNK) {
      const int chunk = min(SEQ_CHUNK, p.sequences - s0), end = scan_sequences(p, status, o, s0, chunk, carry, before, ranges);
      for (int j = threadIdx.x; j < MAX_PIECES; j += (int)blockDim.x) {
        const int i = j * grid + (j & 1 ? grid - 1 - self : self);
        if (i < carry || i >= end) continue;
        const int at = sequence_of(before, chunk, i);
        put(j, ranges[at], i - before[at], 0, tiles_met(o, ranges[at]));
      }
      carry = end;
    }
    const int rounds = carry / grid, rest = carry - rounds * grid;
    found = rounds + ((rounds & 1 ? grid - 1 - self : self) < rest ? 1 : 0);
  } else {
    for (int s0 = 0; s0 < p.sequences; s0 += SEQ_CHUNK)
      carry = scan_sequences(p, status, o, s0, min(SEQ_CHUNK, p.sequences - s0), carry, before, ranges);
    const int blocks = min(grid, carry);                         // nobody's share is empty
    const int begin = self < blocks ? share_begin(carry, self, blocks) : carry, end = self < blocks ? share_begin(carry, self + 1, blocks) : carry;
    carry = 0;
    for (int s0 = 0; s0 < p.sequences && carry < end && begin < end; s0 += SEQ_CHUNK) {
      const int chunk = min(SEQ_CHUNK, p.sequences - s0);
      const int chunk_end = p.sequences <= SEQ_CHUNK ? before[chunk] : scan_sequences(p, status, o, s0, chunk, carry, before, ranges);
      if (begin < chunk_end) {
        for (int s = sequence_of(before, chunk, max(begin, carry)); s < chunk && before[s] < end; ++s) {
          const int from = max(begin, before[s]) - before[s], to = min(end, before[s + 1]) - before[s];
          if (to <= from) continue;
          const int4 r = ranges[s];
          const int whole = tiles_met(o, r), weight = piece_weight(o, r), first = from / weight, last = (to - 1) / weight;
          // a part that has none of the piece's tiles is left out
          const bool skip = whole > 0 ? from - first * weight >= whole : from > first * weight;
          for (int k = first + (skip ? 1 : 0) + (int)threadIdx.x; k <= last; k += (int)blockDim.x) {
            const int t0 = max(from - k * weight, 0), t1 = min(min(to - k * weight, weight), whole);
            const int j = found + k - first - (skip ? 1 : 0);
            if (j < MAX_PIECES) put(j, r, k, t0, max(t1 - t0, 0));
          }
          found += last - first + 1 - (skip ? 1 : 0);
        }
      }
      carry = chunk_end;
    }
    found = min(found, MAX_PIECES);                              // (`least` sees to it)
  }
  fence_proxy_async_smem();                                      // the copies come to where `before` was
  __syncthreads();
  return found;
}
// Place in a ring of stages and the parity of its present round
template <int N>
struct Ring {
  int at = 0, parity = 0;
  __device__ __forceinline__ void step() {
    if (++at == N) {
      at = 0;
      parity ^= 1;
    }
  }
};

// ============================================================================================ forward
// A piece is 256 queries of a head: warps 0-3 and 4-7 hold 128 of them each and share the keys, which come
// in tiles of 128; warps 8 and 9 issue the products of one warpgroup each, warp 10 the copies.  The scores of
// a warpgroup's next tile come only after its last probabilities were used: the two warpgroups fall into step
// so that one runs its exponentials while the tensor core works for the other.  What bounds the kernel is this
// chain: a warp of each warpgroup shares a scheduler and its exp2 unit, 8 cycles for 32 of them, 2048 cycles for
// 2 x 128 x 128 scores, and a round takes 3200 (4 x 4096 rows, 16 heads of 64 channels: 402 us, 684 TFLOP/s; 411 us,
// 836 at 80 channels; 466 us, 1179 at 128).  Scores in halves of a tile, issued one ahead, cost as much in waits as they save at 64 channels; four
// warpgroups with 64 keys each are slower (470 us for 417).  What is kept in registers over the tiles decides more:
// with 100 bytes spilled the kernel is 5 % slower.  The accumulator is rescaled only when a row's maximum has grown
// by more than 2^8 since the last time (probabilities stay below 2^8, the row sum in fp32): rarely after the first tile.
struct ForwardMaps { CUtensorMap q, k, v; };
constexpr int F_MMA_WARP = 8 /* two */, F_TMA_WARP = 10, F_THREADS = 352;
constexpr uint32_t TMEM_ALL = 512;

template <int SLABS>
struct ForwardCfg {
  static constexpr int STAGES = SLABS == 1 ? 3 : 2;
  static constexpr uint32_t TILE = SLABS * RT * 128;             // of queries, keys or values
  static constexpr uint32_t OFF_K = 2 * TILE, OFF_V = OFF_K + STAGES * TILE, OFF_OUT = OFF_V + STAGES * TILE;
  static constexpr uint32_t OFF_BARS = OFF_OUT + 8 * 2048, OFF_SEQ = OFF_BARS + 512;
  static constexpr uint32_t BYTES = OFF_SEQ + TABLE_BYTES + 1024;
  static_assert(BYTES <= 227 * 1024, "fits an SM");
};
// Columns of a warpgroup (256): scores (128), the accumulator (d), the queries (d / 2) where they fit (XT).
// Probabilities of keys [0, 64) lie in [0, 32), of keys [64, 128) in [64, 96).
constexpr uint32_t F_WG = 256, F_O = RT;
enum FwdBar : int {
  F_KFULL = 0, F_KFREE = F_KFULL + 3, F_VFULL = F_KFREE + 3, F_VFREE = F_VFULL + 3, F_QFULL = F_VFREE + 3 /* [wg] shared memory */,
  F_QFREE = F_QFULL + 2, F_Q = F_QFREE + 2 /* [wg] tensor memory */, F_S = F_Q + 2 /* [wg] */, F_P = F_S + 2 /* [wg][half] */,
  F_PV = F_P + 4 /* [wg] */, F_TURN = F_PV + 2 /* [warp] */, F_DRAIN = F_TURN + 8 /* [MMA warp] */, F_BARS = F_DRAIN + 2
};

// Row sums and packed probabilities of 32 scores
__device__ __forceinline__ void exp_32(const uint32_t (&x)[32], float2 sl2v, float2 nmv, float2 (&l2)[2], uint32_t (&pk)[16]) {
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const float2 y = __ffma2_rn(make_float2(__uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1])), sl2v, nmv);
    const float2 p = make_float2(ex2_approx(y.x), ex2_approx(y.y));
    l2[e & 1] = __fadd2_rn(l2[e & 1], p);
    pk[e] = pack_bf16(p.x, p.y);
  }
}
__device__ __forceinline__ float max_32(const uint32_t (&x)[32], float top) {
  float m[2] = {top, -INFINITY};
#pragma unroll
  for (int e = 0; e < 32; e += 4) {
    asm("max.f32 %0, %0, %1, %2;" : "+f"(m[0]) : "f"(__uint_as_float(x[e])), "f"(__uint_as_float(x[e + 1])));
    asm("max.f32 %0, %0, %1, %2;" : "+f"(m[1]) : "f"(__uint_as_float(x[e + 2])), "f"(__uint_as_float(x[e + 3])));
  }
  return fmaxf(m[0], m[1]);
}
// keys behind the end: minus infinity
__device__ __forceinline__ void mask_32(uint32_t (&x)[32], int left) {
  if (left < 32) {
#pragma unroll
    for (int e = 0; e < 32; ++e)
      if (e >= left) x[e] = 0xff800000u;
  }
}

template <int SLABS, bool XT>
__global__ void __launch_bounds__(F_THREADS, 1)
packed_forward_tc_kernel(const __grid_constant__ ForwardMaps maps, const PackedCall c) {
  using L = ForwardCfg<SLABS>;
  extern __shared__ uint8_t smem_raw[];
  const int d = c.p.d, group = c.p.heads / c.p.kv_heads;
  const int warp = (int)uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t sb = smem_u32(smem), bars = sb + L::OFF_BARS;
  auto bar = [&](int i) { return bars + (uint32_t)(8 * i); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::OFF_BARS + 8 * F_BARS);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int i = 0; i < F_BARS; ++i) {
      const bool stage_free = (i >= F_KFREE && i < F_KFREE + 3) || (i >= F_VFREE && i < F_VFREE + 3);   // by both MMA warps
      const bool by_warps = (i >= F_P && i < F_P + 4) || i == F_Q || i == F_Q + 1 || (XT && (i == F_QFREE || i == F_QFREE + 1));
      mbar_init(bar(i), stage_free ? 2 : by_warps ? 4 : 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == F_MMA_WARP) tmem_alloc(smem_u32(tmem_slot), TMEM_ALL);
  if (warp == F_TMA_WARP && lane < 3) prefetch_map(&maps.q + lane);
  const int pieces = find_pieces(c.p, c.dev_status, Order{2 * RT, false, c.p.heads, 1, 0, 0}, reinterpret_cast<int32_t*>(smem + L::OFF_SEQ),
                                 reinterpret_cast<int32_t*>(smem));
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = uniform(*tmem_slot);
  Piece w;
  int at_piece = 0;
  auto advance = [&] {
    if (at_piece >= pieces) return false;
    w = piece_at(sb + L::OFF_SEQ, at_piece++);
    return true;
  };

  if (warp == F_TMA_WARP) {
    // ------------------------------------------------------------------ TMA producer
    if (lane == 0) {
      Ring<L::STAGES> ring;
      int q0 = 0, q1 = 0, n_all = 0;                             // tiles of queries of each warpgroup, of keys so far
      bool ok = true;
      while (ok && advance()) {
        const int n = (w.r.k_len + RT - 1) / RT, kv = group == 1 ? w.head : w.head / group;
        if (n == 0) continue;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          int& q = h ? q1 : q0;
          if (w.x0 + h * RT >= w.r.q_len || !ok) continue;
          if (!mbar_wait_limit(bar(F_QFREE + h), (q & 1) ^ 1, abort_flag, LONG_WAIT_CYCLES)) { ok = false; continue; }
          mbar_arrive_expect_tx(bar(F_QFULL + h), L::TILE);
          ++q;
          for (int s = 0; s < SLABS; ++s)
            tma_load_3d(sb + h * L::TILE + s * RT * 128, &maps.q, 64 * s, w.head, w.r.q_begin + w.x0 + h * RT, bar(F_QFULL + h));
        }
        for (int j = 0; j < n && ok; ++j, ring.step()) {
          const int st = ring.at, krow = w.r.k_begin + j * RT;
          if (!mbar_wait(bar(F_KFREE + st), ring.parity ^ 1, abort_flag)) { ok = false; break; }
          mbar_arrive_expect_tx(bar(F_KFULL + st), L::TILE);
          for (int s = 0; s < SLABS; ++s) tma_load_3d(sb + L::OFF_K + st * L::TILE + s * RT * 128, &maps.k, 64 * s, kv, krow, bar(F_KFULL + st));
          if (!mbar_wait(bar(F_VFREE + st), ring.parity ^ 1, abort_flag)) { ok = false; break; }
          mbar_arrive_expect_tx(bar(F_VFULL + st), L::TILE);
          for (int s = 0; s < SLABS; ++s) tma_load_3d(sb + L::OFF_V + st * L::TILE + s * RT * 128, &maps.v, 64 * s, kv, krow, bar(F_VFULL + st));
          ++n_all;
        }
      }
      if (*abort_flag) {
        // a wait gave up somewhere: let the copies that were started land before the block leaves
        volatile int never = 0;
        if (q0) mbar_wait_limit(bar(F_QFULL), (q0 - 1) & 1, &never, DRAIN_LIMIT_CYCLES);
        if (q1) mbar_wait_limit(bar(F_QFULL + 1), (q1 - 1) & 1, &never, DRAIN_LIMIT_CYCLES);
        // (one tile of keys more than of values may be under way)
        for (int t = n_all > L::STAGES ? n_all - L::STAGES : 0; t <= n_all; ++t) {
          if (t < n_all || !ok) mbar_wait_limit(bar(F_KFULL + t % L::STAGES), (t / L::STAGES) & 1, &never, DRAIN_LIMIT_CYCLES);
          if (t < n_all) mbar_wait_limit(bar(F_VFULL + t % L::STAGES), (t / L::STAGES) & 1, &never, DRAIN_LIMIT_CYCLES);
        }
      }
    }
  } else if (warp >= F_MMA_WARP) {
    // ------------------------------------------------------------------ MMA issuers, one per warpgroup (the whole warp keeps step)
    const int h = warp - F_MMA_WARP;
    const uint32_t base = tmem + h * F_WG, q_smem = sb + h * L::TILE;
    Ring<L::STAGES> ring;
    int seen = 0, turn = 0;                                      // parities: pieces and tiles of this warpgroup so far
    bool ok = true;
    while (ok && advance()) {
      const int n = (w.r.k_len + RT - 1) / RT;
      if (n == 0) continue;
      const bool mine = w.x0 + h * RT < w.r.q_len;               // else the stages are passed on only
      if (mine) {
        if (!warp_wait(bar((XT ? F_Q : F_QFULL) + h), seen, abort_flag)) break;
        seen ^= 1;
      }
      // the scores of tile j (the elected lane): they overwrite P of tile j - 1, whose product this warp issued before
      auto issue_scores = [&](int j, int st) {
        const uint32_t ks = sb + L::OFF_K + st * L::TILE;
        if (mine) {
          const int cols = (min(RT, w.r.k_len - j * RT) + 15) / 16 * 16;
          if (XT) issue_scores_ts<SLABS, RT>(base, base + F_O + d, ks, cols, d / 16);
          else issue_scores_ss<SLABS, RT>(base, q_smem, ks, cols, d / 16);
          umma_commit(bar(F_S + h));
          if (!XT && j == n - 1) umma_commit(bar(F_QFREE + h));
        }
        umma_commit(bar(F_KFREE + st));
      };
      if (!warp_wait(bar(F_KFULL + ring.at), ring.parity, abort_flag)) break;
      if (elect_one()) {
        tc_fence_after();
        issue_scores(0, ring.at);
      }
      __syncwarp();                                              // lanes that poll would hold up the one that issues
      for (int j = 0; j < n; ++j) {
        const int st = ring.at, here = min(RT, w.r.k_len - j * RT), n16 = (here + 15) / 16;
        const uint32_t vs = sb + L::OFF_V + st * L::TILE;
        if (!warp_wait(bar(F_VFULL + st), ring.parity, abort_flag)) { ok = false; break; }
        ring.step();
        // rows of V behind the last key meet probabilities of zero: make them zero too, whatever lies there
        // (both warps write the same zeros; neither reads before its own are there)
        if (mine && here < 16 * n16) zero_rows(vs, RT, SLABS, here, lane);
        // the next tile's keys, so that its scores follow this tile's last product at once
        if (j + 1 < n && !warp_wait(bar(F_KFULL + ring.at), ring.parity, abort_flag)) { ok = false; break; }
        if (mine) {
          if (!warp_wait(bar(F_P + 2 * h), turn, abort_flag)) { ok = false; break; }
          if (n16 > 4) {
            if (elect_one()) {
              tc_fence_after();
              issue_weighted<RT, false>(base + F_O, base, vs, d, 4, j == 0);
            }
            __syncwarp();
            if (!warp_wait(bar(F_P + 2 * h + 1), turn, abort_flag)) { ok = false; break; }
          }
          turn ^= 1;
        }
        if (elect_one()) {
          if (mine) {
            tc_fence_after();
            if (n16 > 4) issue_weighted<RT, false>(base + F_O, base + 64, vs + 64 * 128, d, n16 - 4, false);
            else issue_weighted<RT, false>(base + F_O, base, vs, d, n16, j == 0);
            umma_commit(bar(F_PV + h));
          }
          umma_commit(bar(F_VFREE + st));
          if (j + 1 < n) issue_scores(j + 1, ring.at);
        }
        __syncwarp();
      }
    }
    __syncwarp();
    if (*abort_flag && lane == 0) {
      volatile int never = 0;
      umma_commit(bar(F_DRAIN + h));
      mbar_wait_limit(bar(F_DRAIN + h), 0, &never, DRAIN_LIMIT_CYCLES);
    }
  } else {
    // ------------------------------------------------------------------ softmax and epilogue
    const int wg = warp >> 2, quarter = warp & 3;
    const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + wg * F_WG;
    const float sl2 = c.p.scale * LOG2E;
    const float2 sl2v = make_float2(sl2, sl2);
    // the next piece that has keys and rows for this warpgroup; queries without keys are finished on the way
    auto next = [&] {
      while (advance()) {
        if (w.x0 + wg * RT >= w.r.q_len) continue;
        if (w.r.k_len > 0) return true;
        const int row = w.x0 + wg * RT + quarter * 32 + lane;
        if (row < w.r.q_len) {
          const int64_t at = (int64_t)w.r.q_begin + row;
          bf16* out = static_cast<bf16*>(c.out) + at * c.ldo + (int64_t)w.head * d;
          for (int e = 0; e < d; e += 8) *reinterpret_cast<uint4*>(out + e) = make_uint4(0u, 0u, 0u, 0u);
          c.lse[(int64_t)w.head * c.p.q_rows + at] = -INFINITY;
        }
      }
      return false;
    };
    int turn = 0, seen = 0;                                      // parities: tiles and pieces of this warpgroup so far
    // A warp of each warpgroup shares a scheduler and its exp2 unit.  They take turns there, so that one fetches
    // its scores, finds their maximum and waits for the tensor core while the other runs its exponentials.
    int go = 0;
    // this thread's query of the next piece into tensor memory (the scores that used the last one are complete)
    auto load_query = [&] {
      if (!warp_wait(bar(F_QFULL + wg), seen, abort_flag, LONG_WAIT_CYCLES)) return false;
      seen ^= 1;
      row_to_tmem<SLABS>(taddr + F_O + d, sb + wg * L::TILE, quarter * 32 + lane, d);
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(bar(F_Q + wg));
        mbar_arrive(bar(F_QFREE + wg));
      }
      return true;
    };
    bool more = next();
    bool ok = !XT || !more || load_query();
    while (more && ok) {
      const int k_len = w.r.k_len, number = at_piece - 1;
      const int rows = min(32, w.r.q_len - (w.x0 + wg * RT + quarter * 32));   // of this warp that exist; none if not positive
      const bool pair = w.r.q_len - w.x0 > RT;
      more = next();                                             // looked up while the first scores are computed
      float m = -INFINITY, l = 0.f;                              // row maximum in use (raw scores), row sum
      for (int k0 = 0; k0 < k_len; k0 += RT) {
        const int here = min(RT, k_len - k0);
        // a warpgroup without rows in the pieces before this one waits for all of them: what bounds the wait is
        // the limit of the warps that are at work
        if (!warp_wait(bar(F_S + wg), turn, abort_flag, k0 == 0 ? LONG_WAIT_CYCLES : WAIT_LIMIT_CYCLES)) { ok = false; break; }
        tc_fence_after();
        if (rows > 0) {
          // row maximum; the scores of the second 64 keys are fetched a second time when it is their turn
          uint32_t x[2][32], pk[16];
          float top = -INFINITY;
#pragma unroll
          for (int h = 1; h >= 0; --h) {
            if (64 * h >= here) continue;
            tmem_ld32(taddr + 64 * h, x[0]);
            tmem_ld32(taddr + 64 * h + 32, x[1]);
            tmem_ld_wait_for(x[0]);
            tmem_ld_wait_for(x[1]);
            if (here < 64 * h + 64) {
              mask_32(x[0], here - 64 * h);
              mask_32(x[1], here - 64 * h - 32);
            }
            top = max_32(x[1], max_32(x[0], top));
          }
          const bool grow = (top - m) * sl2 > 8.f;               // false for NaN and for -infinity over -infinity
          if (__any_sync(0xffffffffu, grow)) {
            const float factor = grow ? (m == -INFINITY ? 0.f : ex2_approx((m - top) * sl2)) : 1.f;
            if (grow) m = top;
            l *= factor;
            if (k0 > 0) {                                        // the products of the last tile are complete: these scores are
              for (int e = 0; e < d / 16; ++e) {
                uint32_t o[16];
                tmem_ld16(taddr + F_O + (uint32_t)(16 * e), o);
                tmem_ld_wait();
#pragma unroll
                for (int f = 0; f < 16; ++f) o[f] = __float_as_uint(__uint_as_float(o[f]) * factor);
                tmem_st16(taddr + F_O + (uint32_t)(16 * e), o);
              }
            }
          }
          if (pair && !warp_wait(bar(F_TURN + warp), wg == 0 ? go ^ 1 : go, abort_flag)) { ok = false; break; }
          // p = exp2((s - m) sl2), row sum, P (bf16 pairs) over scores that have been read
          const float nm = m == -INFINITY ? 0.f : -m * sl2;
          const float2 nmv = make_float2(nm, nm);
          float2 l2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
          exp_32(x[0], sl2v, nmv, l2, pk);
          tmem_st16(taddr, pk);
          if (here > 64) tmem_ld32(taddr + 64, x[0]);
          exp_32(x[1], sl2v, nmv, l2, pk);
          if (here > 64) tmem_ld_wait_for(x[0]);
          tmem_st16(taddr + 16, pk);
          if (here > 64) {
            tmem_ld32(taddr + 96, x[1]);
            if (here < 96) mask_32(x[0], here - 64);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(F_P + 2 * wg));
            exp_32(x[0], sl2v, nmv, l2, pk);
            tmem_ld_wait_for(x[1]);
            tmem_st16(taddr + 64, pk);
            if (here > 96) {
              if (here < RT) mask_32(x[1], here - 96);
              exp_32(x[1], sl2v, nmv, l2, pk);
            }
            if (pair && lane == 0) mbar_arrive(bar(F_TURN + (warp ^ 4)));
            if (here > 96) tmem_st16(taddr + 80, pk);
            tmem_st_wait();
          } else {
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(F_P + 2 * wg));
            if (pair && lane == 0) mbar_arrive(bar(F_TURN + (warp ^ 4)));
          }
          l2[0] = __fadd2_rn(l2[0], l2[1]);
          l += l2[0].x + l2[0].y;
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(F_P + 2 * wg + 1));
        } else {
          if (pair && !warp_wait(bar(F_TURN + warp), wg == 0 ? go ^ 1 : go, abort_flag)) { ok = false; break; }
          if (pair && lane == 0) mbar_arrive(bar(F_TURN + (warp ^ 4)));
          tc_fence_before();
          if (lane == 0) {
            mbar_arrive(bar(F_P + 2 * wg));
            mbar_arrive(bar(F_P + 2 * wg + 1));
          }
        }
        turn ^= 1;
        if (pair) go ^= 1;
      }
      if (!ok) break;
      if (XT && more && !load_query()) break;
      if (!warp_wait(bar(F_PV + wg), turn ^ 1, abort_flag)) break;
      tc_fence_after();
      if (rows > 0) {
        const Piece done = piece_at(sb + L::OFF_SEQ, number);    // looked up again: not kept in registers meanwhile
        const int64_t at0 = (int64_t)done.r.q_begin + done.x0 + wg * RT + quarter * 32;
        store_rows(static_cast<bf16*>(c.out) + at0 * c.ldo + (int64_t)done.head * d, c.ldo, taddr + F_O, d, l == 0.f ? 0.f : 1.0f / l, rows,
                   sb + L::OFF_OUT + warp * 2048, lane);
        if (lane < rows) c.lse[(int64_t)done.head * c.p.q_rows + at0 + lane] = l == 0.f ? -INFINITY : fmaf(m, c.p.scale, log2f(l) * LN2);
      }
    }
  }
  // ---------------------------------------------------------------------- teardown
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (threadIdx.x == 0 && *abort_flag) atomicExch(c.dev_status, (int)VIT_ERR_TIMEOUT);
  if (warp == F_MMA_WARP) {
    __syncwarp();
    tmem_dealloc(tmem, TMEM_ALL);
  }
}

// ============================================================================================ backward
// Two kernels of one form.  A piece is a tile of 128 rows X1, X2 of a head, which stays, and tiles of 64 rows
// Y1, Y2 go by:
//   S = X1 Y1^T, dP = X2 Y2^T;  P = exp2(S sl2 - lse2), dS = P (dP - delta)
//   DQ:   X = Q, dout; Y = K, V;  dq += dS Y1.  It comes first and also writes lse2 and delta of its rows.
//   DKDV: X = K, V; Y = Q, dout of every query head that shares the key head (scores transposed);
//         dv += P Y2, dk += dS Y1
// Seven products instead of the five of a single pass, but every gradient is summed in one place in a fixed
// order.  Tiles alternate between places in tensor memory for S and dP, and between two pairs of warpgroups that
// take 32 of the 64 columns each: while one pair is in its exp2 phase the tensor core works for the other, and four
// warps a scheduler hide each other's latencies.  Warps 16 and 19 issue S and dP, warp 17 the second products.
// Up to 64 channels there are three places (2 x 128 x 3 columns, then the accumulators), so that scores are ready
// before a pair comes to them: 4 x 4096 rows, 16 heads of 64: 1208 us with two, 1045 with three.  X is in tensor
// memory (XT) where it fits beside that: for DQ, and for DKDV between 65 and 80 channels; else in shared memory,
// twice where there is room.  What bounds both kernels is the length of a tile's way from S to P to the second
// products and, with four or five tiles to a piece, the change of pieces (18 % and 23 % of the tensor pipe at 64
// images of 197 rows, 52 % and 56 % at four of up to 4097).
// Where pieces do not come out even, the blocks share all tiles equally: the sums of a piece that is not one block's go
// to partial [2 block + (0: its first piece, 1: its last)][dk, dv or dq][128][d] in fp32, and a last kernel adds them in order.
struct BackwardMaps { CUtensorMap x1, x2, x3, y1, y2; };
struct Shares { int blocks, least; };                    // blocks = 0: pieces are not shared
__device__ __forceinline__ Order order_of(const vit_attention_problem& p, bool dkdv, const Shares& s) {
  return Order{RT, dkdv, dkdv ? p.kv_heads : p.heads, dkdv ? p.heads / p.kv_heads : 1, s.blocks, s.least};
}
constexpr int B_MMA_WARP = 16 /* S; 17: second products, 19: dP */, B_TMA_WARP = 18, B_THREADS = 640;

template <int SLABS, bool DKDV, bool XT>
struct BackwardCfg {
  static constexpr int PLACES = SLABS == 1 ? 3 : 2;    // for S and dP in tensor memory
  static constexpr int XBUF = !XT && SLABS == 1 ? 2 : 1;
  static constexpr int XS = DKDV ? 2 : 3;              // tiles of X in shared memory; DQ: out, for delta
  static constexpr int STAGES = SLABS == 1 ? 5 : DKDV ? 4 : 3;
  static constexpr uint32_t XTILE = SLABS * RT * 128, YTILE = SLABS * CT * 128;
  static constexpr uint32_t OFF_Y = XBUF * XS * XTILE, OFF_COL = OFF_Y + STAGES * 2 * YTILE;   // DKDV: float [STAGES][2][64] -lse2, -delta of the columns
  static constexpr uint32_t OFF_ROW = OFF_COL + (DKDV ? STAGES * CT * 8 : 0);           // DQ: float2 [2][128] of the rows
  static constexpr uint32_t OFF_OUT = OFF_ROW + (DKDV ? 0 : 2 * RT * 8), OFF_BARS = OFF_OUT + 8 * 2048, OFF_SEQ = OFF_BARS + 512;
  static constexpr uint32_t BYTES = OFF_SEQ + TABLE_BYTES + 1024;
  static_assert(BYTES <= 227 * 1024, "fits an SM");
};
// columns: S and dP of the two warpgroups, then the accumulators (d each), then X1 and X2 (d / 2 each)
constexpr uint32_t B_WG = 2 * CT;
enum BwdBar : int {
  B_FULL = 0, B_FREE = B_FULL + 5, B_XS = B_FREE + 5 /* X in shared memory */, B_XSFREE = B_XS + 2, B_X = B_XSFREE + 2 /* in tensor memory */, B_XFREE,
  B_S /* [tile % 6, or % 2] */, B_P = B_S + 6 /* [place] */, B_SFREE = B_P + 3, B_ACC = B_SFREE + 3, B_ACCFREE, B_DRAIN /* [MMA warp] */, B_BARS = B_DRAIN + 4
};

template <int SLABS, bool DKDV, bool XT>
__global__ void __launch_bounds__(B_THREADS, 1)
packed_backward_tc_kernel(const __grid_constant__ BackwardMaps maps, const PackedCall c, const Shares shares) {
  using L = BackwardCfg<SLABS, DKDV, XT>;
  constexpr int PLACES = L::PLACES, XBUF = L::XBUF, ROUND = PLACES == 3 ? 6 : 2;   // tiles until place and warpgroups are the same again
  constexpr uint32_t B_COLS = PLACES * B_WG;
  extern __shared__ uint8_t smem_raw[];
  const int d = c.p.d, group = c.p.heads / c.p.kv_heads;
  const int warp = (int)uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t sb = smem_u32(smem), bars = sb + L::OFF_BARS;
  auto bar = [&](int i) { return bars + (uint32_t)(8 * i); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::OFF_BARS + 8 * B_BARS);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int i = 0; i < B_BARS; ++i)
    {
      const bool x_free = i == B_XSFREE || i == B_XSFREE + 1;
      int count = 1;
      if ((i >= B_P && i < B_P + PLACES) || i == B_ACCFREE) count = 8;
      else if (i == B_X) count = 16;
      else if ((i >= B_S && i < B_S + ROUND) || i == B_XFREE || (!XT && x_free)) count = 2;    // S and dP
      else if (x_free) count = DKDV ? 8 : 12;
      mbar_init(bar(i), count);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == B_MMA_WARP) tmem_alloc(smem_u32(tmem_slot), TMEM_ALL);
  if (warp == B_TMA_WARP && lane < 5) prefetch_map(&maps.x1 + lane);
  const int pieces_in_all = find_pieces(c.p, c.dev_status, order_of(c.p, DKDV, shares), reinterpret_cast<int32_t*>(smem + L::OFF_SEQ),
                                        reinterpret_cast<int32_t*>(smem));
  if (DKDV) asm volatile("griddepcontrol.wait;" ::: "memory");               // the kernel before this one leaves delta
  else asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = uniform(*tmem_slot);
  const uint32_t acc2 = B_COLS, acc1 = B_COLS + d, x1_col = B_COLS + (DKDV ? 2 : 1) * d, x2_col = x1_col + d / 2;   // dk or dq; dv
  Piece w;
  int at_piece = 0, y_tiles = 0;                                  // of piece w: tiles of a head of Y
  auto advance = [&] {
    if (at_piece >= pieces_in_all) return false;
    w = piece_at(sb + L::OFF_SEQ, at_piece++);
    y_tiles = ((DKDV ? w.r.q_len : w.r.k_len) + CT - 1) / CT;
    return true;
  };

  if (warp == B_TMA_WARP) {
    // ------------------------------------------------------------------ producer (the whole warp keeps step)
    Ring<L::STAGES> ring;
    int pieces = 0, n_all = 0;
    bool ok = true;
    while (ok && advance()) {
      const int y_begin = DKDV ? w.r.q_begin : w.r.k_begin, y_len = DKDV ? w.r.q_len : w.r.k_len;
      if (w.n == 0) continue;
      const int x_at = XBUF == 2 ? pieces & 1 : 0;
      const uint32_t xs = sb + x_at * L::XS * L::XTILE;
      if (!warp_wait(bar(B_XSFREE + x_at), (pieces / XBUF & 1) ^ 1, abort_flag)) break;
      if (lane == 0) {
        const int row = (DKDV ? w.r.k_begin : w.r.q_begin) + w.x0;
        mbar_arrive_expect_tx(bar(B_XS + x_at), L::XS * L::XTILE);
        for (int s = 0; s < SLABS; ++s) {
          tma_load_3d(xs + s * RT * 128, &maps.x1, 64 * s, w.head, row, bar(B_XS + x_at));
          tma_load_3d(xs + L::XTILE + s * RT * 128, &maps.x2, 64 * s, w.head, row, bar(B_XS + x_at));
          if (!DKDV) tma_load_3d(xs + 2 * L::XTILE + s * RT * 128, &maps.x3, 64 * s, w.head, row, bar(B_XS + x_at));
        }
      }
      ++pieces;
      const int heads_on = DKDV && w.t_begin > 0 ? w.t_begin / y_tiles : 0;
      int y0 = (w.t_begin - heads_on * y_tiles) * CT, yh = DKDV ? w.head * group + heads_on : group == 1 ? w.head : w.head / group;
      for (int t = 0; t < w.n; ++t, ring.step()) {
        const int st = ring.at;
        const uint32_t y = sb + L::OFF_Y + st * 2 * L::YTILE;
        // DKDV: the numbers of the tile's columns travel with it, negated; beyond the sequence
        // P = exp2(0 - infinity) = 0 and dS = 0.  They are in flight while this warp waits for the stage.
        float2 v[2];
        if (DKDV) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            v[e] = make_float2(INFINITY, 0.f);
            if (y0 + 32 * e + lane < y_len) v[e] = c.delta[(int64_t)yh * c.p.q_rows + y_begin + y0 + 32 * e + lane];
          }
        }
        if (!warp_wait(bar(B_FREE + st), ring.parity ^ 1, abort_flag)) { ok = false; break; }
        if (DKDV) {
          float* col = reinterpret_cast<float*>(smem + L::OFF_COL) + st * 2 * CT;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            col[32 * e + lane] = -v[e].x;
            col[CT + 32 * e + lane] = -v[e].y;
          }
          __syncwarp();
        }
        ++n_all;
        if (lane == 0) {
          mbar_arrive_expect_tx(bar(B_FULL + st), 2 * L::YTILE);
          for (int s = 0; s < SLABS; ++s) {
            tma_load_3d(y + s * CT * 128, &maps.y1, 64 * s, yh, y_begin + y0, bar(B_FULL + st));
            tma_load_3d(y + L::YTILE + s * CT * 128, &maps.y2, 64 * s, yh, y_begin + y0, bar(B_FULL + st));
          }
        }
        y0 += CT;
        if (y0 >= y_len) { y0 = 0; ++yh; }
      }
    }
    __syncwarp();
    if (*abort_flag && lane == 0) {
      // a wait gave up somewhere: let the copies that were started land before the block leaves
      volatile int never = 0;
      for (int i = pieces > XBUF ? pieces - XBUF : 0; i < pieces; ++i)
        mbar_wait_limit(bar(B_XS + i % XBUF), i / XBUF & 1, &never, DRAIN_LIMIT_CYCLES);
      for (int t = n_all > L::STAGES ? n_all - L::STAGES : 0; t < n_all; ++t)
        mbar_wait_limit(bar(B_FULL + t % L::STAGES), (t / L::STAGES) & 1, &never, DRAIN_LIMIT_CYCLES);
    }
  } else if (warp >= B_MMA_WARP) {
    // ------------------------------------------------------------------ MMA issuers (whole warps keep step): one of S, one
    // of dP, one of the second products
    const bool scores = warp != B_MMA_WARP + 1, first = warp == B_MMA_WARP;
    Ring<L::STAGES> ring;
    int pieces = 0, phase = 0;                                   // bit b of phase: parity of the next wait for warpgroup b's columns
    bool ok = true;
    while (ok && advance()) {
      const int y_len = DKDV ? w.r.q_len : w.r.k_len;
      if (w.n == 0) continue;
      const int x_at = XBUF == 2 ? pieces & 1 : 0;
      const uint32_t xs = sb + x_at * L::XS * L::XTILE;
      if (scores && !warp_wait(bar(XT ? B_X : B_XS + x_at), pieces / XBUF & 1, abort_flag)) break;
      int left = y_len - (w.t_begin > 0 ? w.t_begin % y_tiles : 0) * CT;   // rows of this head from the present tile on
      int b = -1;                                                // place of tile t
      for (int t = 0; t < w.n; ++t, ring.step()) {
        b = b + 1 == PLACES ? 0 : b + 1;
        const int st = ring.at, here = min(CT, left), n16 = (here + 15) / 16;
        const uint32_t y = sb + L::OFF_Y + st * 2 * L::YTILE, s_col = tmem + b * B_WG;
        left = left > CT ? left - CT : y_len;
        if (scores) {
          if (!warp_wait(bar(B_FULL + st), ring.parity, abort_flag)) { ok = false; break; }
          // rows of Y behind the end of the sequence become zero, whatever lies there: they meet weights of
          // zero in the second products, and give scores of zero in the first
          if (here < 16 * n16) {
            zero_rows(first ? y : y + L::YTILE, CT, SLABS, here, lane);
          }
          // S and dP overwrite P and dS of tile t - 2, once their products are complete
          if (!warp_wait(bar(B_SFREE + b), (phase >> b & 1) ^ 1, abort_flag)) { ok = false; break; }
          phase ^= 1 << b;
          if (elect_one()) {
            tc_fence_after();
            if (XT) issue_scores_ts<SLABS, CT>(first ? s_col : s_col + CT, tmem + (first ? x1_col : x2_col), first ? y : y + L::YTILE, 16 * n16, d / 16);
            else issue_scores_ss<SLABS, CT>(first ? s_col : s_col + CT, first ? xs : xs + L::XTILE, first ? y : y + L::YTILE, 16 * n16, d / 16);
            umma_commit(bar(B_S + t % ROUND));
            if (t == w.n - 1) umma_commit(bar(XT ? B_XFREE : B_XSFREE + x_at));
          }
        } else {
          if (!warp_wait(bar(B_P + b), phase >> b & 1, abort_flag)) { ok = false; break; }
          phase ^= 1 << b;
          // the accumulators of the last piece have been read
          if (t == 0 && !warp_wait(bar(B_ACCFREE), (pieces & 1) ^ 1, abort_flag)) { ok = false; break; }
          if (elect_one()) {
            tc_fence_after();
            if (DKDV) issue_weighted<CT, true>(tmem + acc1, s_col, y + L::YTILE, d, n16, t == 0);
            issue_weighted<CT, true>(tmem + acc2, s_col + CT, y, d, n16, t == 0);
            umma_commit(bar(B_SFREE + b));
            umma_commit(bar(B_FREE + st));
            if (t == w.n - 1) umma_commit(bar(B_ACC));
          }
        }
        __syncwarp();                                            // lanes that poll would hold up the one that issues
      }
      ++pieces;
    }
    __syncwarp();
    if (*abort_flag && lane == 0) {
      volatile int never = 0;
      umma_commit(bar(B_DRAIN + warp - B_MMA_WARP));
      mbar_wait_limit(bar(B_DRAIN + warp - B_MMA_WARP), 0, &never, DRAIN_LIMIT_CYCLES);
    }
  } else {
    // ------------------------------------------------------------------ probabilities and their gradients
    // warpgroups 0, 1: the two halves of the even tiles' columns; 2, 3: of the odd tiles'
    const int wg = warp >> 2, odd = wg >> 1, half = wg & 1, quarter = warp & 3, in_tile = quarter * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
    const uint32_t stage = sb + L::OFF_OUT + (warp & 7) * 2048;
    const float sl2 = c.p.scale * LOG2E;
    const float2 sl2v = make_float2(sl2, sl2);
    Ring<L::STAGES> ring;                                        // of every tile, this warpgroup's or not
    int pieces = 0, s_phase = 0;
    // the next piece with something to walk over; rows that nothing meets get gradients of zero on the way
    auto next = [&] {
      while (advance()) {
        if (w.n > 0) return true;
        const int row = w.x0 + in_tile;
        const int64_t at = (int64_t)(DKDV ? w.r.k_begin : w.r.q_begin) + row;
        if (wg == 0 && row < (DKDV ? w.r.k_len : w.r.q_len)) {
          bf16* g2 = DKDV ? static_cast<bf16*>(c.dk) + at * c.lddk + (int64_t)w.head * d : static_cast<bf16*>(c.dq) + at * c.lddq + (int64_t)w.head * d;
          bf16* g1 = static_cast<bf16*>(c.dv) + at * c.lddv + (int64_t)w.head * d;
          for (int e = 0; e < d; e += 8) {
            *reinterpret_cast<uint4*>(g2 + e) = make_uint4(0u, 0u, 0u, 0u);
            if (DKDV) *reinterpret_cast<uint4*>(g1 + e) = make_uint4(0u, 0u, 0u, 0u);
          }
        }
      }
      return false;
    };
    // Rows of X1 (first warpgroup) and X2 (second) of piece w into tensor memory; the third of DQ takes the
    // product of dout and out.  All of them answer for it, so that none is a piece behind.
    auto load_x = [&] {
      if (wg < (DKDV ? 2 : 3)) {
        if (!warp_wait(bar(B_XS), pieces & 1, abort_flag)) return false;
        if (wg < 2) {
          row_to_tmem<SLABS>(lanes + (wg == 0 ? x1_col : x2_col), sb + wg * L::XTILE, in_tile, d);
          tmem_st_wait();
          tc_fence_before();
        } else {
          const int row = w.x0 + in_tile;
          const int64_t i = (int64_t)w.head * c.p.q_rows + w.r.q_begin + row;
          const bool there = row < w.r.q_len;
          const float lse = there ? c.lse[i] : 0.f;
          float delta = 0.f;
#pragma unroll 2
          for (int g = 0; g < d / 16; ++g) {
            uint32_t u[8], v[8];
            read_16(u, sb + L::XTILE, in_tile, g);
            read_16(v, sb + 2 * L::XTILE, in_tile, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) delta = dot2(u[e], v[e], delta);
          }
          const float2 mine = make_float2(lse * LOG2E, delta);
          reinterpret_cast<float2*>(smem + L::OFF_ROW)[(pieces & 1) * RT + in_tile] = mine;
          if (there) c.delta[i] = mine;
        }
      }
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(bar(B_X));
        if (wg < (DKDV ? 2 : 3)) mbar_arrive(bar(B_XSFREE));
      }
      return true;
    };
    bool more = next();
    bool ok = !XT || !more || load_x();
    while (more && ok) {
      const int y_len = DKDV ? w.r.q_len : w.r.k_len;
      const int number = at_piece - 1, rows = min(32, (DKDV ? w.r.k_len : w.r.q_len) - (w.x0 + quarter * 32));
      float2 nls = make_float2(0.f, 0.f), nde = nls;             // DQ: of this thread's row
      if (!DKDV) {
        if (!warp_wait(bar(B_X), pieces & 1, abort_flag)) break;
        const float2 mine = reinterpret_cast<const float2*>(smem + L::OFF_ROW)[(pieces & 1) * RT + in_tile];
        nls = make_float2(-mine.x, -mine.x);
        nde = make_float2(-mine.y, -mine.y);
      }
      const int n = w.n;                                         // (w moves on)
      int left = y_len - (w.t_begin > 0 ? w.t_begin % y_tiles : 0) * CT;   // rows of this head from the present tile on
      for (int t = 0; t < n; ++t, ring.step()) {
        const int here = min(CT, left) - 32 * half;              // of this warpgroup's 32 columns
        left = left > CT ? left - CT : y_len;
        if ((t & 1) != odd) continue;
        const int st = ring.at, place = t % PLACES, s_bar = t % ROUND;
        const uint32_t taddr = lanes + place * B_WG + half * 32;
        // four columns each: -lse2, then -delta
        const float4* col = reinterpret_cast<const float4*>(smem + L::OFF_COL) + st * (CT / 2) + 8 * half;
        if (DKDV && !warp_wait(bar(B_FULL + st), ring.parity, abort_flag)) { ok = false; break; }
        if (!warp_wait(bar(B_S + s_bar), s_phase >> s_bar & 1, abort_flag)) { ok = false; break; }
        s_phase ^= 1 << s_bar;
        tc_fence_after();
        if (rows > 0 && here > 0) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (16 * h >= here) break;
            uint32_t sh[16], gh[16];
            tmem_ld16(taddr + 16 * h, sh);
            tmem_ld16(taddr + CT + 16 * h, gh);
            tmem_ld_wait_16(sh, gh);
            uint32_t pk[8], dk[8];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              float4 a4 = make_float4(nls.x, nls.x, nls.x, nls.x), b4 = make_float4(nde.x, nde.x, nde.x, nde.x);
              if (DKDV) {
                a4 = col[4 * h + q];
                b4 = col[CT / 4 + 4 * h + q];
              }
#pragma unroll
              for (int f = 0; f < 2; ++f) {
                const int e = 2 * q + f;
                const float2 a = f ? make_float2(a4.z, a4.w) : make_float2(a4.x, a4.y), b = f ? make_float2(b4.z, b4.w) : make_float2(b4.x, b4.y);
                const float2 x = __ffma2_rn(make_float2(__uint_as_float(sh[2 * e]), __uint_as_float(sh[2 * e + 1])), sl2v, a);
                float2 pr = make_float2(ex2_approx(x.x), ex2_approx(x.y));
                if (!DKDV && here < 32) {                        // keys behind the end
                  if (16 * h + 2 * e >= here) pr.x = 0.f;
                  if (16 * h + 2 * e + 1 >= here) pr.y = 0.f;
                }
                const float2 y = __fmul2_rn(pr, __fadd2_rn(make_float2(__uint_as_float(gh[2 * e]), __uint_as_float(gh[2 * e + 1])), b));
                if (DKDV) pk[e] = pack_bf16(pr.x, pr.y);
                dk[e] = pack_bf16(y.x, y.y);
              }
            }
            // over scores that this warp has read: step h takes columns [8 h, 8 h + 8) of its 32
            if (DKDV) tmem_st8(taddr + 8 * h, pk);
            tmem_st8(taddr + CT + 8 * h, dk);
          }
          tmem_st_wait();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_P + place));
      }
      if (!ok) break;
      ++pieces;
      more = next();
      if (XT && more) {
        // every score of the last piece is complete: its X may be overwritten
        if (!warp_wait(bar(B_XFREE), (pieces - 1) & 1, abort_flag)) break;
        tc_fence_after();
        if (!load_x()) break;
      }
      if (wg >= 2) continue;
      // the first two warpgroups store the sums
      if (!warp_wait(bar(B_ACC), (pieces - 1) & 1, abort_flag)) break;
      tc_fence_after();
      if (rows > 0) {
        const Piece done = piece_at(sb + L::OFF_SEQ, number);    // looked up again: not kept in registers meanwhile
        const int64_t at0 = (int64_t)(DKDV ? done.r.k_begin : done.r.q_begin) + done.x0 + quarter * 32;
        const int whole = ((DKDV ? done.r.q_len : done.r.k_len) + CT - 1) / CT * (DKDV ? group : 1), head = done.head;
        const int64_t slot = 2 * blockIdx.x + (done.t_begin > 0 ? 0 : 1);
        float* sums = n < whole ? c.partial + ((slot * (DKDV ? 2 : 1) + (DKDV ? wg & 1 : 0)) * RT + quarter * 32) * d : nullptr;
        const int from = DKDV || wg == 0 ? 0 : d / 32 * 16, to = DKDV || wg == 1 ? d : d / 32 * 16;   // dk, dv; or a part of dq each
        if (sums) {
          store_rows(sums + from, d, lanes + (DKDV && wg == 1 ? acc1 : acc2) + from, to - from, 1.f, rows, stage, lane);
        } else if (DKDV) {
          const int64_t ld = wg == 0 ? c.lddk : c.lddv;
          store_rows(static_cast<bf16*>(wg == 0 ? c.dk : c.dv) + at0 * ld + (int64_t)head * d, ld, lanes + (wg == 0 ? acc2 : acc1), d,
                     wg == 0 ? gradient_scale(c.p, done.r.k_len) : 1.f, rows, stage, lane);
        } else {
          store_rows(static_cast<bf16*>(c.dq) + at0 * c.lddq + (int64_t)head * d + from, c.lddq, lanes + acc2 + from, to - from, gradient_scale(c.p, done.r.k_len), rows,
                     stage, lane);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_ACCFREE));
    }
  }
  // ---------------------------------------------------------------------- teardown
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (threadIdx.x == 0 && *abort_flag) atomicExch(c.dev_status, (int)VIT_ERR_TIMEOUT);
  if (warp == B_MMA_WARP) {
    __syncwarp();
    tmem_dealloc(tmem, TMEM_ALL);
  }
}

// The sums of the pieces that were shared, in order, times the factor of the gradient, rounded once.  Block (i, j)
// takes 32 j ... of the piece whose first border between two shares is that behind share i.
constexpr int ADD_ROWS = 32;
template <bool DKDV>
__global__ void __launch_bounds__(256) add_parts_kernel(const PackedCall c, const Shares shares) {
  __shared__ int32_t before[SCAN_INTS];
  __shared__ int4 ranges[SEQ_CHUNK];
  const Order o = order_of(c.p, DKDV, shares);
  int total = 0, carry = 0, chunk = 0;
  for (int s0 = 0; s0 < c.p.sequences; s0 += SEQ_CHUNK)
    total = scan_sequences(c.p, c.dev_status, o, s0, min(SEQ_CHUNK, c.p.sequences - s0), total, before, ranges);
  const int blocks = min(shares.blocks, total);                  // as find_pieces has it
  if ((int)blockIdx.x + 1 >= blocks) return;
  const int border = share_begin(total, blockIdx.x + 1, blocks);
  for (int s0 = 0; s0 < c.p.sequences; s0 += SEQ_CHUNK) {        // the sequence that has it
    chunk = min(SEQ_CHUNK, c.p.sequences - s0);
    const int end = c.p.sequences <= SEQ_CHUNK ? total : scan_sequences(c.p, c.dev_status, o, s0, chunk, carry, before, ranges);
    if (border < end) break;
    carry = end;
  }
  const int at = sequence_of(before, chunk, border);
  const int4 r = ranges[at];
  const int whole = tiles_met(o, r), weight = piece_weight(o, r), k = (border - before[at]) / weight, begin = before[at] + k * weight;
  const int first = share_of(total, begin, blocks);
  if (border == begin || border >= begin + whole || first != (int)blockIdx.x) return;    // not inside, or not the first
  const int last = share_of(total, begin + whole - 1, blocks);
  const int tiles = ((DKDV ? r.w : r.y) + RT - 1) / RT, head = k / tiles, x0 = (k - head * tiles) * RT + (int)blockIdx.y * ADD_ROWS;
  const int rows = min(ADD_ROWS, (DKDV ? r.w : r.y) - x0), d = c.p.d, eights = d / 8;
#pragma unroll
  for (int tensor = 0; tensor < (DKDV ? 2 : 1); ++tensor) {
    const int64_t ld = DKDV ? (tensor ? c.lddv : c.lddk) : c.lddq;
    bf16* to = static_cast<bf16*>(DKDV ? (tensor ? c.dv : c.dk) : c.dq) + ((int64_t)(DKDV ? r.z : r.x) + x0) * ld + (int64_t)head * d;
    const float by = tensor ? 1.f : gradient_scale(c.p, r.w);
    for (int i = threadIdx.x; i < rows * eights; i += 256) {
      const int row = i / eights, ch = (i - row * eights) * 8;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
      for (int share = first; share <= last; ++share) {          // the first one's last piece, the others' first
        const int64_t slot = 2 * share + (share == first ? 1 : 0);
        const float4* from = reinterpret_cast<const float4*>(c.partial + ((slot * (DKDV ? 2 : 1) + tensor) * RT + blockIdx.y * ADD_ROWS + row) * d + ch);
        const float4 u = from[0], v = from[1];
        a.x += u.x; a.y += u.y; a.z += u.z; a.w += u.w;
        b.x += v.x; b.y += v.y; b.z += v.z; b.w += v.w;
      }
      *reinterpret_cast<uint4*>(to + row * ld + ch) = make_uint4(pack_bf16(a.x * by, a.y * by), pack_bf16(a.z * by, a.w * by),
                                                                 pack_bf16(b.x * by, b.y * by), pack_bf16(b.z * by, b.w * by));
    }
  }
}

// ============================================================================================ launches
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encoder() {
  static const EncodeTiledFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiledFn>(p);
  }();
  return fn;
}

// (channel, head, row) of a buffer [rows, heads * d] with row stride ld; boxes of 64 channels x 1 head x box_rows rows
bool encode_heads(CUtensorMap* tm, const void* base, int64_t rows, int heads, int d, int64_t ld, int box_rows) {
  const EncodeTiledFn fn = encoder();
  if (!fn) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)heads, (cuuint64_t)rows};
  const cuuint64_t strides[2] = {(cuuint64_t)d * 2, (cuuint64_t)ld * 2};
  const cuuint32_t box[3] = {64, 1, (cuuint32_t)box_rows}, one[3] = {1, 1, 1};
  return fn(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// One persistent block per SM; more where its table of pieces would not hold its share: just above 128 pieces to an SM
// (18944 in all, counted with max_q) a second round of few blocks takes as long as the first.
int grid_of(int total, int sms) {
  const int least = (total + MAX_PIECES - 1) / MAX_PIECES, most = total < sms ? total : sms;
  return least > most ? least : most;
}

template <int SLABS, bool XT>
cudaError_t launch_forward(const PackedCall& c, cudaStream_t s) {
  using L = ForwardCfg<SLABS>;
  ForwardMaps m;
  if (!encode_heads(&m.q, c.q, c.p.q_rows, c.p.heads, c.p.d, c.ldq, RT)) return cudaErrorInvalidValue;
  if (c.p.k_rows > 0) {
    if (!encode_heads(&m.k, c.k, c.p.k_rows, c.p.kv_heads, c.p.d, c.ldk, RT)) return cudaErrorInvalidValue;
    if (!encode_heads(&m.v, c.v, c.p.k_rows, c.p.kv_heads, c.p.d, c.ldv, RT)) return cudaErrorInvalidValue;
  } else {
    m.k = m.v = m.q;                                   // no keys at all: never used
  }
  static PerDeviceFlag done;
  if (cudaError_t e = ensure_dynamic_smem(done, packed_forward_tc_kernel<SLABS, XT>, (int)L::BYTES)) return e;
  const int sms = current_device_sm_count();
  if (sms < 1) return cudaErrorInvalidDevice;
  const int tiles = (c.p.max_q + 2 * RT - 1) / (2 * RT), total = c.p.sequences * c.p.heads * tiles;
  packed_forward_tc_kernel<SLABS, XT><<<grid_of(total, sms), F_THREADS, L::BYTES, s>>>(m, c);
  return cudaGetLastError();
}

// Whether the blocks of the backward pass share the tiles (in shares of eight at least): where that takes less time,
// counted in tiles.  A piece takes three besides its own, shares cost each block two parts and a launch more, and
// without them the last round is as long as a full one.
// (4 sequences of up to 4097, 8 heads over 2 key heads of 128: dq 161 us in whole pieces, 144 and 8 for the sums in
// shares; dk and dv 269 in whole pieces, 172 and 9 in shares.)
constexpr int SHARE_BLOCKS = 148;
Shares shares_of(const vit_attention_problem& p, bool dkdv) {
  const int64_t pieces = (int64_t)p.sequences * (dkdv ? p.kv_heads : p.heads) * (((dkdv ? p.max_k : p.max_q) + RT - 1) / RT);
  const int64_t tiles = (int64_t)(dkdv ? p.heads / p.kv_heads : 1) * (((dkdv ? p.max_q : p.max_k) + CT - 1) / CT);
  if (pieces == 0 || tiles == 0 || tiles > (1 << 30) / pieces) return Shares{0, 0};
  const int64_t most = pieces * tiles / 8, blocks = most < SHARE_BLOCKS ? most : SHARE_BLOCKS;
  if (blocks < 2 || pieces > 100 * blocks) return Shares{0, 0};
  const int64_t whole = (pieces + SHARE_BLOCKS - 1) / SHARE_BLOCKS * (tiles + 3), shared = pieces * (tiles + 3) / blocks + 16;
  if (shared >= whole) return Shares{0, 0};
  // a block's share is pieces * tiles / blocks of such weights at most: 120 pieces, and one more at either end
  return Shares{(int)blocks, (int)((pieces * tiles + 120 * blocks - 1) / (120 * blocks))};
}
size_t partial_floats(const vit_attention_problem& p, bool dkdv) { return (size_t)shares_of(p, dkdv).blocks * 2 * (dkdv ? 2 : 1) * RT * p.d; }

template <int SLABS, bool DKDV, bool XT>
cudaError_t launch_backward(const PackedCall& c, cudaStream_t s) {
  using L = BackwardCfg<SLABS, DKDV, XT>;
  BackwardMaps m;
  const void *x1 = DKDV ? c.k : c.q, *x2 = DKDV ? c.v : c.dout, *y1 = DKDV ? c.q : c.k, *y2 = DKDV ? c.dout : c.v;
  const int64_t lx1 = DKDV ? c.ldk : c.ldq, lx2 = DKDV ? c.ldv : c.lddo, ly1 = DKDV ? c.ldq : c.ldk, ly2 = DKDV ? c.lddo : c.ldv;
  const int64_t xr = DKDV ? c.p.k_rows : c.p.q_rows, yr = DKDV ? c.p.q_rows : c.p.k_rows;
  const int xh = DKDV ? c.p.kv_heads : c.p.heads, yh = DKDV ? c.p.heads : c.p.kv_heads;
  if (!encode_heads(&m.x1, x1, xr, xh, c.p.d, lx1, RT) || !encode_heads(&m.x2, x2, xr, xh, c.p.d, lx2, RT)) return cudaErrorInvalidValue;
  if (yr > 0) {
    if (!encode_heads(&m.y1, y1, yr, yh, c.p.d, ly1, CT) || !encode_heads(&m.y2, y2, yr, yh, c.p.d, ly2, CT)) return cudaErrorInvalidValue;
  } else {
    m.y1 = m.y2 = m.x1;
  }
  if (DKDV) m.x3 = m.x1;
  else if (!encode_heads(&m.x3, c.out, xr, xh, c.p.d, c.ldo, RT)) return cudaErrorInvalidValue;
  static PerDeviceFlag done;
  if (cudaError_t e = ensure_dynamic_smem(done, packed_backward_tc_kernel<SLABS, DKDV, XT>, (int)L::BYTES)) return e;
  const int sms = current_device_sm_count();
  if (sms < 1) return cudaErrorInvalidDevice;
  const Shares shares = shares_of(c.p, DKDV);
  const int total = c.p.sequences * xh * (((DKDV ? c.p.max_k : c.p.max_q) + RT - 1) / RT);
  // dk and dv look their pieces up while the last blocks of dq (or of its sums) are at work, if that was launched before them
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(shares.blocks > 0 ? shares.blocks : grid_of(total, sms)));
  cfg.blockDim = dim3(B_THREADS);
  cfg.dynamicSmemBytes = L::BYTES;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = DKDV && c.p.q_rows > 0 && c.p.max_q > 0 ? 1 : 0;
  if (cudaError_t e = cudaLaunchKernelEx(&cfg, packed_backward_tc_kernel<SLABS, DKDV, XT>, m, c, shares)) return e;
  if (shares.blocks > 0) {
    add_parts_kernel<DKDV><<<dim3((unsigned)shares.blocks - 1, RT / ADD_ROWS), 256, 0, s>>>(c, shares);
    return cudaGetLastError();
  }
  return cudaSuccess;
}

}  // namespace

bool attention_in_parts(const vit_attention_problem& p, bool dkdv) { return shares_of(p, dkdv).blocks > 0; }
// Columns of tensor memory decide where a piece's rows are held: 128 + d + d / 2 of a warpgroup's 256 in
// the forward pass, 256 + 2 d + d of 512 for dk and dv, 256 + d + d for dq.
size_t attention_partial_floats(const vit_attention_problem& p) {
  const size_t a = partial_floats(p, true), b = partial_floats(p, false);    // one after the other
  return a > b ? a : b;
}
cudaError_t launch_attention_packed_bf16(const PackedCall& c, cudaStream_t s) {
  if (c.p.d <= 64) return launch_forward<1, true>(c, s);
  return c.p.d <= 80 ? launch_forward<2, true>(c, s) : launch_forward<2, false>(c, s);
}
cudaError_t launch_attention_packed_dkdv_bf16(const PackedCall& c, cudaStream_t s) {
  if (c.p.d <= 64) return launch_backward<1, true, false>(c, s);
  return c.p.d <= 80 ? launch_backward<2, true, true>(c, s) : launch_backward<2, true, false>(c, s);
}
cudaError_t launch_attention_packed_dq_bf16(const PackedCall& c, cudaStream_t s) {
  return c.p.d <= 64 ? launch_backward<1, false, true>(c, s) : launch_backward<2, false, true>(c, s);
}

}  // namespace vit
