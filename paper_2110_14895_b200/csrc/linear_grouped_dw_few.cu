// Gradients of the weights and bias of one linear layer with few tiles (bf16): what linear_grouped_dw.cu does, with the sum of a
// tile of 256 x 256 shared by two or four pairs of blocks of a cluster and joined in its shared memory.
//
// Parts of tiles that go through memory cost 256 KB each way and a second kernel, 7 to 10 us in all; here the pairs leave their sums
// where the operands were, and each block adds up an equal number of rows, in the order of the pairs.  The pairs of a cluster
// have equal shares of the rows, and there is one tile to a cluster.
// 577 rows, 1280 x 1280: 14 us, 20 by way of memory; 3152 rows, 1024 x 2048: 22 and 29; 8224 rows, 1280 x 1280: 39 and
// 40 (a pair has 65 units there instead of 44, at the 0.4 us that they take on all SMs).
//
// Every wait on a barrier in memory is bounded; on expiry the block raises the device status word and goes on to the barriers of
// the block and the cluster, which all threads reach the same number of times.
#include "linear_grouped.cuh"
#include "linear_grouped_tc.cuh"

namespace vit {

using namespace grouped;

namespace {

constexpr int TN = 256, EPI_WARPS = 8, SUM_WARPS = 4, THREADS = 32 * (2 + EPI_WARPS + SUM_WARPS + 1), STAGES = 6;
constexpr int A_BYTES = 2 * SLAB_BYTES, STAGE_BYTES = 2 * A_BYTES, LD = TN + 4;              // LD: of the sums, where the stages were
constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + 1024 + 1024;
static_assert(BM * LD * 4 <= STAGES * STAGE_BYTES, "the sums lie where the stages were");

struct DwFewArgs {
  GroupedShape shape;
  int in, out, tiles_in, split;
  bf16* dw;
  float* dbias;
  int* dev_status;
};
struct DwFewMaps { CUtensorMap dout, x; };

__device__ __forceinline__ float4 read_cluster(uint32_t here, uint32_t rank) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(map_to_cta(here, rank)) : "memory");
  return v;
}
// to the barriers of both blocks of a pair anywhere in the cluster
__device__ __forceinline__ void commit_to(uint32_t bar, uint32_t even) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
      "h"((uint16_t)(3u << even))
      : "memory");
}

__global__ void __launch_bounds__(THREADS, 1)
grouped_dw_few_kernel(const __grid_constant__ DwFewMaps m, const __grid_constant__ DwFewArgs p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t tiles = smem_u32(smem);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + STAGES * STAGE_BYTES);
  const uint32_t landed = smem_u32(bars), cleared = landed + 8 * STAGES, ready = cleared + 8 * STAGES, used = ready + 8 * STAGES, summed = used + 8 * STAGES,
                 done = summed + 8 * STAGES, drain = done + 8;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 5 * STAGES + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const uint32_t bias_sums = tiles + STAGES * STAGE_BYTES + 512;                             // [128] floats
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t place = cluster_ctarank(), rank = place & 1, even = place & ~1u;
  const int pair = (int)place >> 1, tile = (int)blockIdx.x / (2 * p.split);

  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(landed + 8 * i, 1);
      mbar_init(cleared + 8 * i, 1);
      mbar_init(ready + 8 * i, 1);
      mbar_init(used + 8 * i, 1);
      mbar_init(summed + 8 * i, SUM_WARPS);
    }
    mbar_init(done, 1);
    mbar_init(drain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_map(&m.dout);
    prefetch_map(&m.x);
  }
  if (warp == 1) tmem_alloc_pair(smem_u32(tmem_slot), TN);
  tc_fence_before();
  __syncthreads();
  cluster_sync();                          // the others' barriers are initialised before anyone signals them
  tc_fence_after();
  grid_dependency_wait();
  grid_launch_dependents();
  const uint32_t tmem = *tmem_slot;
  if (blockIdx.x == 0 && warp == 2) report_bad_groups(p.shape, p.dev_status, lane);

  int begin, end;
  int stage = 0;
  uint32_t phase = 0, tails = 0, turns = 0;
  long long fills = 0;
  if (group_rows(p.shape, 0, begin, end)) {
    const int n0 = tile / p.tiles_in * (2 * BM) + (int)rank * BM, kt = tile % p.tiles_in, k0 = kt * TN;
    const bool sums = p.dbias && kt == 0;                                                    // columns are summed, behind the products
    const int rows = end - begin, all = (rows + DW_ROWS - 1) / DW_ROWS, share = (all + p.split - 1) / p.split;
    const int from = min(all, pair * share), to = min(all, from + share);                    // of the tile's units of 64 rows
    if (warp == 0) {
      // ---------------------------------------------------------------- TMA producer
      for (int kb = from; kb < to; ++kb) {
        if (!warp_wait(used + 8 * stage, phase ^ 1, abort_flag) || (sums && !warp_wait(summed + 8 * stage, phase ^ 1, abort_flag))) break;
        ++fills;
        const int row = begin + kb * DW_ROWS;
        const bool tail = has_tail(end - row);
        tails = tail ? tails | 1u << stage : tails & ~(1u << stage);
        turns ^= (tail ? 1u : 0u) << stage;
        if (elect_one()) {
          const uint32_t sa = tiles + stage * STAGE_BYTES, at = announce<2>(landed + 8 * stage, ready + 8 * stage, tail, place, STAGE_BYTES);
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            tma_load_2d_pair(sa + s * SLAB_BYTES, &m.dout, n0 + 64 * s, row, at);
            tma_load_2d_pair(sa + A_BYTES + s * SLAB_BYTES, &m.x, k0 + (int)rank * (TN / 2) + 64 * s, row, at);
          }
        }
        __syncwarp();
        if (++stage == STAGES) { stage = 0; phase ^= 1; }
      }
    } else if (warp == 1) {
      // ---------------------------------------------------------------- products
      if (rank == 0) {
        constexpr uint32_t id = instr_desc(2 * BM, TN, true, true);
        for (int kb = from; kb < to; ++kb) {
          if (!warp_wait(ready + 8 * stage, phase, abort_flag)) break;
          tc_fence_after();
          const uint32_t sa = uniform(tiles + stage * STAGE_BYTES);
          const int steps = (min(DW_ROWS, rows - kb * DW_ROWS) + 15) / 16;
          const uint64_t ad = smem_desc(sa, SLAB_BYTES), bd = smem_desc(sa + A_BYTES, SLAB_BYTES);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (k < steps) umma_bf16_pair(tmem, ad + (uint64_t)(128 * k), bd + (uint64_t)(128 * k), id, (kb > from || k > 0) ? 1u : 0u);
            commit_to(used + 8 * stage, even);
          }
          __syncwarp();
          if (++stage == STAGES) { stage = 0; phase ^= 1; }
        }
        if (elect_one()) commit_to(done, even);
        __syncwarp();
      }
    } else if (warp == 2 + EPI_WARPS + SUM_WARPS) {
      // ---------------------------------------------------------------- the group's last rows
      for (int kb = from; kb < to; ++kb) {
        const int some = rows - kb * DW_ROWS;
        if (has_tail(some)) {                            // the others of their 16 become zero
          if (!warp_wait(landed + 8 * stage, turns >> stage & 1, abort_flag)) break;
          const uint32_t sa = tiles + stage * STAGE_BYTES;
          for (int s = 0; s < 4; ++s)
            for (int i = some * 8 + lane; i < (some + 15) / 16 * 128; i += 32)
              asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(sa + (uint32_t)(s * SLAB_BYTES + i * 16)), "r"(0u) : "memory");
          if (!hand_on<2>(ready + 8 * stage, cleared + 8 * stage, turns >> stage & 1, place, lane, abort_flag)) break;
          turns ^= 1u << stage;
        }
        if (++stage == STAGES) stage = 0;
      }
    } else if (warp >= 2 + EPI_WARPS && sums) {
      // ---------------------------------------------------------------- sums of dout's columns
      // a warp has 32 columns; a lane 8 of them and every eighth row, such that eight lanes meet all banks
      const int sw = warp - 2 - EPI_WARPS, slab = sw >> 1, ck = (sw & 1) * 4 + (lane & 3), first = (lane >> 3) | (lane & 4);
      float2 sum[4] = {};
      for (int kb = from; kb < to; ++kb) {
        if (!warp_wait(used + 8 * stage, phase, abort_flag)) break;
        const uint32_t slab_at = tiles + stage * STAGE_BYTES + slab * SLAB_BYTES;
        uint32_t w[8][4];
#pragma unroll
        for (int i = 0; i < 8; ++i) read_chunk(w[i], slab_at, first + 8 * i, ck);
        __syncwarp();
        if (lane == 0) mbar_arrive(summed + 8 * stage);  // releases behind what has been read
        float2 some[4] = {};
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (first + 8 * i < rows - kb * DW_ROWS) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              some[e] = __fadd2_rn(some[e], make_float2(__uint_as_float(w[i][e] << 16), __uint_as_float(w[i][e] & 0xffff0000u)));
          }
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = __fadd2_rn(sum[e], some[e]);
        if (++stage == STAGES) { stage = 0; phase ^= 1; }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
          sum[e].x += __shfl_xor_sync(0xffffffffu, sum[e].x, o);
          sum[e].y += __shfl_xor_sync(0xffffffffu, sum[e].y, o);
        }
      if (lane < 4) {
        const uint32_t here = bias_sums + (uint32_t)(slab * 64 + ck * 8) * 4;
#pragma unroll
        for (int h = 0; h < 2; ++h)
          asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(here + 16u * h), "f"(sum[2 * h].x), "f"(sum[2 * h].y), "f"(sum[2 * h + 1].x),
                       "f"(sum[2 * h + 1].y)
                       : "memory");
      }
    } else if (warp < 2 + EPI_WARPS) {
      warp_wait(done, 0, abort_flag);
      tc_fence_after();
    }
    __syncthreads();                                     // nobody reads the stages any more
    if (warp >= 2 && warp < 2 + EPI_WARPS && !*abort_flag) {
      const int quarter = warp & 3, half = ((warp - 2) >> 2) * 128, row = quarter * 32 + lane;
#pragma unroll 1
      for (int q = 0; q < 4; ++q) {
        uint32_t r[32];
        tmem_ld32(tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half + 32 * q), r);
        tmem_ld_wait_for(r);
        const bool none = from == to;                    // no rows for this pair: its sums are zero
#pragma unroll
        for (int e = 0; e < 8; ++e)
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(tiles + (uint32_t)((row * LD + half + 32 * q + 4 * e) * 4)),
                       "r"(none ? 0u : r[4 * e]), "r"(none ? 0u : r[4 * e + 1]), "r"(none ? 0u : r[4 * e + 2]), "r"(none ? 0u : r[4 * e + 3])
                       : "memory");
      }
      tc_fence_before();
    }
    __syncwarp();
    cluster_sync();                                      // the sums of all pairs can be read
    tc_fence_after();
    if (!*abort_flag) {
      // a share of the block's 128 rows, eight columns at a time
      const int mine = BM / p.split, first_row = pair * mine;
      for (int i = threadIdx.x; i < mine * (TN / 8); i += THREADS) {
        const int r = first_row + i / (TN / 8), c = i % (TN / 8) * 8;
        if (n0 + r >= p.out || k0 + c >= p.in) continue;
        const uint32_t here = tiles + (uint32_t)((r * LD + c) * 4);
        float4 a[4], b[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (k < p.split) {
            a[k] = read_cluster(here, (uint32_t)(2 * k) + rank);
            b[k] = read_cluster(here + 16, (uint32_t)(2 * k) + rank);
          }
        float2 v[4] = {make_float2(a[0].x, a[0].y), make_float2(a[0].z, a[0].w), make_float2(b[0].x, b[0].y), make_float2(b[0].z, b[0].w)};
#pragma unroll
        for (int k = 1; k < 4; ++k)
          if (k < p.split) {
            v[0] = __fadd2_rn(v[0], make_float2(a[k].x, a[k].y));
            v[1] = __fadd2_rn(v[1], make_float2(a[k].z, a[k].w));
            v[2] = __fadd2_rn(v[2], make_float2(b[k].x, b[k].y));
            v[3] = __fadd2_rn(v[3], make_float2(b[k].z, b[k].w));
          }
        uint4 o;
        __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&o);
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = __floats2bfloat162_rn(v[e].x, v[e].y);
        *reinterpret_cast<uint4*>(p.dw + (int64_t)(n0 + r) * p.in + k0 + c) = o;
      }
      if (p.dbias && kt == 0 && pair == 0 && threadIdx.x < BM / 4 && n0 + 4 * (int)threadIdx.x < p.out) {
        float4 sum = read_cluster(bias_sums + 16 * threadIdx.x, rank);
        for (int k = 1; k < p.split; ++k) {
          const float4 v = read_cluster(bias_sums + 16 * threadIdx.x, (uint32_t)(2 * k) + rank);
          sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
        }
        *reinterpret_cast<float4*>(p.dbias + n0 + 4 * threadIdx.x) = sum;
      }
    }
  }

  if (*abort_flag) {
    if (warp == 0) drain_fills(landed, ready, STAGES, fills, tails, turns, rank == 0);
    if (warp == 1 && rank == 0) drain_products<2>(drain);
    // the partner may be in a wait of its own that nothing will satisfy any more
    if (threadIdx.x == 0)
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_to_cta(smem_u32(const_cast<int*>(abort_flag)), place ^ 1u)), "r"(1) : "memory");
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_sync();                          // no block leaves while another may still touch it
  tc_fence_after();
  if (threadIdx.x == 0 && *abort_flag) atomicExch(p.dev_status, (int)VIT_ERR_TIMEOUT);
  if (warp == 1) {
    __syncwarp();
    tmem_dealloc_pair(tmem, TN);
  }
}

}  // namespace

cudaError_t launch_grouped_dw_few(const GroupedCall& c, const GroupedDw& plan, cudaStream_t s) {
  DwFewArgs p{c.shape, c.in, c.out_features, plan.tiles_in, plan.split, static_cast<bf16*>(c.dw), c.dbias, c.dev_status};
  DwFewMaps m;
  if (!encode_rows(&m.dout, c.dout, c.shape.rows, c.out_features, c.lddout, DW_ROWS) || !encode_rows(&m.x, c.x, c.shape.rows, c.in, c.ldx, DW_ROWS))
    return cudaErrorInvalidValue;
  static PerDeviceFlag configured;
  if (cudaError_t e = ensure_dynamic_smem(configured, grouped_dw_few_kernel, SMEM_BYTES)) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(plan.tiles * 2 * plan.split));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = SMEM_BYTES;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)(2 * plan.split);
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, grouped_dw_few_kernel, m, p);
}

}  // namespace vit
