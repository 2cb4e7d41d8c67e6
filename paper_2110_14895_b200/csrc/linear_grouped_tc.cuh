// Pieces of the tensor-core kernels of linear layers by group: tiles, descriptors, copies, products, the way out.
#pragma once
#include "linear_grouped.cuh"

#include <cuda.h>

namespace vit {
namespace grouped {

using namespace ptx;

constexpr int BM = 128;                        // rows of an operand tile = lanes of tensor memory
constexpr int BK = 64;                         // of the summed index per stage: 128 bytes, one swizzle row
constexpr uint32_t SLAB_BYTES = 64 * 128;      // 64 rows of the summed index by 64 columns
constexpr long long DRAIN_LIMIT_CYCLES = 1ll << 24;    // teardown after a failed wait: ~10 ms per barrier

// Shared-memory matrix descriptor of 128-byte-swizzled rows, groups of 8 rows 1024 bytes apart.  lbo: distance of the slabs
// of 64 columns of an operand whose rows are the summed index.
__device__ __forceinline__ uint64_t smem_desc(uint32_t saddr, uint32_t lbo = 16) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)((lbo >> 4) & 0x3FFFu) << 16) | ((uint64_t)(1024 >> 4) << 32) |
         ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// kind::f16: fp32 accumulate, bf16 x bf16; an operand is `across` if its rows are the summed index
__host__ __device__ constexpr uint32_t instr_desc(int rows, int cols, bool a_across, bool b_across) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (a_across ? 1u << 15 : 0u) | (b_across ? 1u << 16 : 0u) | ((uint32_t)(cols >> 3) << 17) |
         ((uint32_t)(rows >> 4) << 24);
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* tm) { asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(tm)) : "memory"); }

template <int CTAS>
__device__ __forceinline__ void load_2d(uint32_t dst, const CUtensorMap* tm, int x, int y, uint32_t bar) {
  if (CTAS == 2) tma_load_2d_pair(dst, tm, x, y, bar);
  else tma_load_2d(dst, tm, x, y, bar);
}
template <int CTAS>
__device__ __forceinline__ void load_3d(uint32_t dst, const CUtensorMap* tm, int x, int y, int z, uint32_t bar) {
  if (CTAS == 2)
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(tm)), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
  else
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(tm)), "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
}
template <int CTAS>
__device__ __forceinline__ void product(uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t accumulate) {
  if (CTAS == 2) umma_bf16_pair(d, a, b, id, accumulate);
  else umma_bf16(d, a, b, id, accumulate);
}
template <int CTAS>
__device__ __forceinline__ void commit(uint32_t bar) {
  if (CTAS == 2) umma_commit_pair(bar);
  else umma_commit(bar);
}
// an epilogue warp has done with an accumulator: to the warp that issues the products (the even block's of a pair)
template <int CTAS>
__device__ __forceinline__ void give_back(uint32_t bar) {
  if (CTAS == 2) mbar_arrive_cluster(map_to_cta(bar, 0));
  else mbar_arrive(bar);
}
// a bounded wait of a whole warp: all lanes leave with the same answer
static __device__ __noinline__ bool wait_on(uint32_t bar, int parity, volatile int* abort_flag) { return mbar_wait(bar, (uint32_t)parity, abort_flag); }
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  return __all_sync(0xffffffffu, wait_on(bar, (int)parity, abort_flag));
}
// One lane of the warp, chosen by the hardware: behind it the operands of the products stay in uniform registers.
__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.b32 %0, 1, 0, p;\n}\n" : "=r"(one));
  return one != 0;
}
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __shfl_sync(0xffffffffu, v, 0); }

// After a wait gave up: the copies of the last `stages` fills may still be in flight.  Waits, bounded, until each of those
// stages has received its bytes, so that nothing lands in shared memory after the block has left.
__device__ __forceinline__ void drain_stages(uint32_t full, int stages, long long fills) {
  volatile int never = 0;
  for (long long f = fills > stages ? fills - stages : 0; f < fills; ++f)
    mbar_wait_limit(full + 8 * (uint32_t)(f % stages), (uint32_t)((f / stages) & 1), &never, DRAIN_LIMIT_CYCLES);
}
// and the products issued so far (by the thread that the hardware elects) are done before tensor memory is freed.  A commit
// tracks the products of its own kind only: a pair's are committed as a pair's.
template <int CTAS>
__device__ __forceinline__ void drain_products(uint32_t bar) {
  volatile int never = 0;
  if (elect_one()) {
    if (CTAS == 2) umma_commit_pair_here(bar);
    else umma_commit(bar);
    mbar_wait_limit(bar, 0, &never, DRAIN_LIMIT_CYCLES);
  }
}

// The stages of the weights' gradients.  A stage's copies, in a pair those of both blocks, are counted on `ready` of the even block,
// where the products wait.  A stage with a group's last rows, of which some have to be cleared first, comes to `landed` of its own
// block.  The warp that clears it there arrives at `ready`, the odd block's by way of the even one's, which waits at `cleared`.
// `landed` and `cleared` have turns of their own for every stage: a bit of `turns`.
__device__ __forceinline__ bool has_tail(int rows) { return rows < DW_ROWS && (rows & 15); }         // rows: from the unit's first to the group's last
// announces the bytes of a block's copies; the barrier to which they come
template <int CTAS>
__device__ __forceinline__ uint32_t announce(uint32_t landed, uint32_t ready, bool tail, uint32_t place, uint32_t bytes) {
  if (tail) mbar_arrive_expect_tx(landed, bytes);
  else if (CTAS == 1 || !(place & 1)) mbar_arrive_expect_tx(ready, CTAS * bytes);
  if (CTAS == 1) return tail ? landed : ready;
  return tail ? map_to_cta(landed, place) : map_to_cta(ready, place & ~1u);
}
// All lanes have written their zeros: a stage is handed on to the products.
template <int CTAS>
__device__ __forceinline__ bool hand_on(uint32_t ready, uint32_t cleared, uint32_t turn, uint32_t place, int lane, volatile int* abort_flag) {
  fence_proxy_async_smem();
  __syncwarp();
  if (CTAS == 2 && (place & 1)) {
    if (lane == 0) mbar_arrive_cluster(map_to_cta(cleared, place & ~1u));
    __syncwarp();
    return true;
  }
  if (CTAS == 2) {
    if (!warp_wait(cleared, turn, abort_flag)) return false;
    mbar_try_wait_cluster(cleared, turn);               // (it is complete) what the other block wrote before it arrived is acquired
  }
  if (lane == 0) mbar_arrive(ready);
  __syncwarp();
  return true;
}
// After a wait gave up, as drain_stages: tails: the stages whose last fill had a tail.  The copies of an odd block's other stages are
// counted in the even one, which it does not leave before.
__device__ __forceinline__ void drain_fills(uint32_t landed, uint32_t ready, int stages, long long fills, uint32_t tails, uint32_t turns, bool even) {
  volatile int never = 0;
  for (long long f = fills > stages ? fills - stages : 0; f < fills; ++f) {
    const uint32_t s = (uint32_t)(f % stages);
    if (tails >> s & 1) mbar_wait_limit(landed + 8 * s, (turns >> s & 1) ^ 1, &never, DRAIN_LIMIT_CYCLES);
    else if (even) mbar_wait_limit(ready + 8 * s, (uint32_t)((f / stages) & 1), &never, DRAIN_LIMIT_CYCLES);
  }
}

// A warp's 32 rows of 64 columns as bf16 in a swizzled 4 KB piece; a lane owns a row.
__device__ __forceinline__ uint32_t chunk_at(uint32_t piece, int row, int chunk) { return piece + (uint32_t)(row * 128 + ((chunk ^ (row & 7)) << 4)); }
__device__ __forceinline__ void read_chunk(uint32_t (&w)[4], uint32_t piece, int row, int chunk) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(chunk_at(piece, row, chunk)) : "memory");
}
__device__ __forceinline__ void put_half(const float2 (&v)[16], uint32_t piece, int lane, int half) {
#pragma unroll
  for (int ck = 0; ck < 4; ++ck) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      __nv_bfloat162 h = __floats2bfloat162_rn(v[4 * ck + e].x, v[4 * ck + e].y);
      w[e] = *reinterpret_cast<uint32_t*>(&h);
    }
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(chunk_at(piece, lane, 4 * half + ck)), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3])
                 : "memory");
  }
}
// Sends the piece: by TMA where all 32 rows are the group's, else row by row.
__device__ __forceinline__ void send_rows(const CUtensorMap* tm, bf16* out, int64_t ld, uint32_t piece, int row0, int c0, int rows, int width,
                                          int lane) {
  if (rows == 32) {
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) tma_store_2d(tm, piece, c0, row0);       // columns beyond the width are clipped
    return;
  }
  __syncwarp();
  const int ck = lane & 7;
  for (int r = lane >> 3; r < rows; r += 4) {
    uint32_t w[4];
    read_chunk(w, piece, r, ck);
    if (c0 + 8 * ck < width) *reinterpret_cast<uint4*>(out + (int64_t)(row0 + r) * ld + c0 + 8 * ck) = make_uint4(w[0], w[1], w[2], w[3]);
  }
  fence_proxy_async_smem();                                 // the next copy into the piece comes by TMA, behind these reads and writes
  __syncwarp();
}

// ---- host
// What is done with the sums: bias, GELU, GELU with its argument kept, a residual added, GELU's slope at what is read.
enum Finish : int { F_BIAS = 0, F_GELU = 1, F_GELU_PRE = 2, F_RESIDUAL = 3, F_SLOPE = 4 };
// maps of matrices in 128-byte-swizzled boxes of 64 columns by `box_rows` rows
bool encode_rows(CUtensorMap* tm, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_rows);
// the weights of all groups, [groups][rows][cols]
bool encode_weights(CUtensorMap* tm, const void* base, int groups, int rows, int cols, int box_rows);

}  // namespace grouped

// few tiles with a long sum, shared by clusters (linear_grouped_few.cu)
int grouped_few_split(const GroupedShape& shape, int width, int sum);
cudaError_t launch_grouped_few_bf16(const GroupedCall& c, grouped::Finish finish, int split, cudaStream_t s);

}  // namespace vit
