// Linear layers by group with few tiles and a long sum (a few rows of a large layer, one token), bf16, forwards and backwards.
//
// Bound by the weights, which a few blocks could not fetch fast enough: a cluster of two to eight blocks shares the sum of a tile
// of 128 x 128, each with its own stretch of the summed index.  The blocks leave their sums of the rows that exist in their
// shared memory, and each adds up and finishes an equal share of the values, in the order of the blocks.
// 1 row, 4096 -> 1024: 9.3 us, 18 with one block to a tile; 197 rows of 8 groups, 1536 -> 384: 7.7 us, 10.1.  Sums below 1536 are as fast with
// one block (197 rows, 768 -> 768: 8.3 us, 9.3 here).
//
// Every wait on a barrier in memory is bounded; on expiry the block raises the device status word and goes on to the cluster's
// barriers, which all of its blocks reach the same number of times.
#include "linear_grouped.cuh"
#include "linear_grouped_tc.cuh"

namespace vit {

using namespace grouped;

namespace {

constexpr int BN = 128, EPI_WARPS = 8, THREADS = (2 + EPI_WARPS) * 32, STAGES = 4;
constexpr int A_BYTES = BM * BK * 2, STAGE_BYTES = A_BYTES + BN * BK * 2, LD = BN + 4;       // LD: of the sums in shared memory
constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + BM * LD * 4 + 1024 + 256;

struct FewArgs {
  GroupedShape shape;
  int width, sum, split;
  Finish finish;
  const float* bias;               // [groups][width] or nullptr
  bf16* out; int64_t ldo;
  bf16* other; int64_t ldother;    // GELU's argument, written or read, or the residual
  int tiles_n;
  int* dev_status;
};
struct FewMaps { CUtensorMap a, w; };

__device__ __forceinline__ float4 read_cluster(uint32_t here, uint32_t rank) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(map_to_cta(here, rank)) : "memory");
  return v;
}
__device__ __forceinline__ uint2 pack4(float2 lo, float2 hi) {
  __nv_bfloat162 a = __floats2bfloat162_rn(lo.x, lo.y), b = __floats2bfloat162_rn(hi.x, hi.y);
  return make_uint2(*reinterpret_cast<uint32_t*>(&a), *reinterpret_cast<uint32_t*>(&b));
}

template <bool ACROSS>
__global__ void __launch_bounds__(THREADS, 1)
grouped_few_kernel(const __grid_constant__ FewMaps m, const __grid_constant__ FewArgs p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t tiles = smem_u32(smem), sums = tiles + STAGES * STAGE_BYTES;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + STAGES * STAGE_BYTES + BM * LD * 4);
  const uint32_t full = smem_u32(bars), empty = full + 8 * STAGES, done = empty + 8 * STAGES, drain = done + 8;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * STAGES + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int unit = (int)blockIdx.x / p.split, units = (int)gridDim.x / p.split;

  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(full + 8 * i, 1);
      mbar_init(empty + 8 * i, 1);
    }
    mbar_init(done, 1);
    mbar_init(drain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_map(&m.a);
    prefetch_map(&m.w);
  }
  if (warp == 1) tmem_alloc(smem_u32(tmem_slot), (uint32_t)BN);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  grid_dependency_wait();
  grid_launch_dependents();
  const uint32_t tmem = *tmem_slot;
  if (blockIdx.x == 0 && warp == 2) report_bad_groups(p.shape, p.dev_status, lane);

  const int all = (p.sum + BK - 1) / BK, share = (all + p.split - 1) / p.split;      // blocks of 64 of the summed index
  const int k_begin = min(all, (int)rank * share), k_end = min(all, k_begin + share);
  GroupWalk<TileCount> walk(p.shape, TileCount{BM, p.tiles_n}, lane);
  GroupAt at;
  int stage = 0;
  uint32_t phase = 0, turn = 0;
  long long fills = 0;
  for (int tile = unit; walk.find(tile, at); tile += units, turn ^= 1) {
    const int local = tile - at.before, mt = local / p.tiles_n, row0 = at.begin + mt * BM, c0 = (local - mt * p.tiles_n) * BN;
    const int rows = min(BM, at.end - row0);
    if (warp == 0) {
      for (int kb = k_begin; kb < k_end; ++kb) {
        if (!warp_wait(empty + 8 * stage, phase ^ 1, abort_flag)) break;
        ++fills;
        if (lane == 0) {
          const uint32_t sa = tiles + stage * STAGE_BYTES, sb = sa + A_BYTES, fb = full + 8 * stage;
          mbar_arrive_expect_tx(fb, STAGE_BYTES);
          if (ACROSS) {
#pragma unroll
            for (int s = 0; s < BN / 64; ++s) load_3d<1>(sb + s * SLAB_BYTES, &m.w, c0 + 64 * s, kb * BK, at.group, fb);
          } else {
            load_3d<1>(sb, &m.w, kb * BK, c0, at.group, fb);
          }
          load_2d<1>(sa, &m.a, kb * BK, row0, fb);
        }
        __syncwarp();
        if (++stage == STAGES) { stage = 0; phase ^= 1; }
      }
    } else if (warp == 1) {
      constexpr uint32_t id = instr_desc(BM, BN, false, ACROSS);
      for (int kb = k_begin; kb < k_end; ++kb) {
        if (!warp_wait(full + 8 * stage, phase, abort_flag)) break;
        tc_fence_after();
        const uint32_t sa = uniform(tiles + stage * STAGE_BYTES);
        const uint64_t ad = smem_desc(sa), bd = smem_desc(sa + A_BYTES, ACROSS ? SLAB_BYTES : 16);
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < BK / 16; ++k)
            umma_bf16(tmem, ad + (uint64_t)(2 * k), bd + (uint64_t)(ACROSS ? 128 * k : 2 * k), id, (kb > k_begin || k > 0) ? 1u : 0u);
          umma_commit(empty + 8 * stage);
        }
        __syncwarp();
        if (++stage == STAGES) { stage = 0; phase ^= 1; }
      }
      if (elect_one()) umma_commit(done);
      __syncwarp();
    } else if (warp_wait(done, turn, abort_flag)) {
      tc_fence_after();
      const int ew = warp - 2, quarter = warp & 3, half = (ew >> 2) * 64, row = quarter * 32 + lane;
      if (quarter * 32 < rows) {
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          uint32_t r[32];
          tmem_ld32(tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half + 32 * h), r);
          tmem_ld_wait_for(r);
          if (row < rows) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const uint32_t to = sums + (uint32_t)((row * LD + half + 32 * h + 4 * e) * 4);
              const bool none = k_begin == k_end;                       // a stretch without anything in it
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(none ? 0u : r[4 * e]), "r"(none ? 0u : r[4 * e + 1]),
                           "r"(none ? 0u : r[4 * e + 2]), "r"(none ? 0u : r[4 * e + 3])
                           : "memory");
            }
          }
        }
      }
      tc_fence_before();
    }
    __syncwarp();
    cluster_sync();                                // the sums of all blocks can be read
    tc_fence_after();
    if (!*abort_flag) {
      // four columns of a row at a time; row by row, so that neighbours write side by side
      const int columns = min(BN, p.width - c0) / 4, items = rows * columns, mine = (items + p.split - 1) / p.split;
      const float* bias = p.bias ? p.bias + (int64_t)at.group * p.width + c0 : nullptr;
      for (int i = (int)rank * mine + (int)threadIdx.x; i < min(items, ((int)rank + 1) * mine); i += THREADS) {
        const int r = i / columns, c = (i - r * columns) * 4;
        const uint32_t here = sums + (uint32_t)((r * LD + c) * 4);
        float4 part[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) part[k] = k < p.split ? read_cluster(here, (uint32_t)k) : make_float4(0.f, 0.f, 0.f, 0.f);
        const int64_t row = row0 + r;
        uint2 o = make_uint2(0, 0);
        if (p.finish == F_RESIDUAL || p.finish == F_SLOPE) o = *reinterpret_cast<const uint2*>(p.other + row * p.ldother + c0 + c);
        float2 lo = make_float2(part[0].x, part[0].y), hi = make_float2(part[0].z, part[0].w);
#pragma unroll
        for (int k = 1; k < 8; ++k)
          if (k < p.split) {
            lo = __fadd2_rn(lo, make_float2(part[k].x, part[k].y));
            hi = __fadd2_rn(hi, make_float2(part[k].z, part[k].w));
          }
        if (bias) {
          const float4 b = *reinterpret_cast<const float4*>(bias + c);
          lo = __fadd2_rn(lo, make_float2(b.x, b.y));
          hi = __fadd2_rn(hi, make_float2(b.z, b.w));
        }
        const float2 ol = make_float2(__uint_as_float(o.x << 16), __uint_as_float(o.x & 0xffff0000u));
        const float2 oh = make_float2(__uint_as_float(o.y << 16), __uint_as_float(o.y & 0xffff0000u));
        if (p.finish == F_GELU_PRE) *reinterpret_cast<uint2*>(p.other + row * p.ldother + c0 + c) = pack4(lo, hi);
        if (p.finish == F_GELU || p.finish == F_GELU_PRE) {
          lo = gelu_2(lo);
          hi = gelu_2(hi);
        } else if (p.finish == F_RESIDUAL) {
          lo = __fadd2_rn(lo, ol);
          hi = __fadd2_rn(hi, oh);
        } else if (p.finish == F_SLOPE) {
          lo = __fmul2_rn(lo, gelu_slope_2(ol));
          hi = __fmul2_rn(hi, gelu_slope_2(oh));
        }
        *reinterpret_cast<uint2*>(p.out + row * p.ldo + c0 + c) = pack4(lo, hi);
      }
    }
    __syncwarp();
    cluster_sync();                                // nobody reads the sums any more
  }

  if (*abort_flag) {
    if (warp == 0) drain_stages(full, STAGES, fills);
    if (warp == 1) drain_products<1>(drain);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (threadIdx.x == 0 && *abort_flag) atomicExch(p.dev_status, (int)VIT_ERR_TIMEOUT);
  if (warp == 1) {
    __syncwarp();
    tmem_dealloc(tmem, (uint32_t)BN);
  }
}

template <bool ACROSS>
cudaError_t launch_few(const FewMaps& m, const FewArgs& p, int grid, cudaStream_t s) {
  static PerDeviceFlag configured;
  if (cudaError_t e = ensure_dynamic_smem(configured, grouped_few_kernel<ACROSS>, SMEM_BYTES)) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = SMEM_BYTES;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)p.split;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, grouped_few_kernel<ACROSS>, m, p);
}

}  // namespace

// Blocks that share a tile's sum: as many as find an SM each and have 256 of the sum or more; 1: not for this kernel.
int grouped_few_split(const GroupedShape& shape, int width, int sum) {
  const int sms = current_device_sm_count();
  const int64_t tiles = ((int64_t)shape.rows / BM + (shape.groups < shape.rows ? shape.groups : shape.rows)) * ((width + BN - 1) / BN);
  int split = 1;
  if (sum < 1536) return split;
  while (split < 8 && tiles * split * 2 <= sms * 7 / 8 && sum >= 512 * split) split *= 2;      // (not every SM finds partners for a cluster)
  return split;
}

cudaError_t launch_grouped_few_bf16(const GroupedCall& c, Finish finish, int split, cudaStream_t s) {
  const int width = c.backward ? c.in : c.out_features, sum = c.backward ? c.out_features : c.in;
  FewArgs p{c.shape, width, sum, split, finish, c.backward ? nullptr : c.bias, static_cast<bf16*>(c.y), c.ldy,
            static_cast<bf16*>(finish == F_RESIDUAL ? const_cast<void*>(c.residual) : c.pre), finish == F_RESIDUAL ? c.ldr : c.ldp,
            (width + BN - 1) / BN, c.dev_status};
  FewMaps m;
  if (!encode_rows(&m.a, c.x, c.shape.rows, sum, c.ldx, BM) ||
      !encode_weights(&m.w, c.w, c.shape.groups, c.out_features, c.in, c.backward ? BK : BN))
    return cudaErrorInvalidValue;
  const int64_t most = ((int64_t)c.shape.rows / BM + c.shape.groups) * p.tiles_n, units = current_device_sm_count() / split;
  const int grid = (int)(most < units ? most : units) * split;
  return c.backward ? launch_few<true>(m, p, grid, s) : launch_few<false>(m, p, grid, s);
}

}  // namespace vit
