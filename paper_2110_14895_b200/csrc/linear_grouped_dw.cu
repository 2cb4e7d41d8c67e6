// Gradients of the weights and biases of linear layers by group on the 5th-generation tensor cores (bf16):
//
//   dW_g = sum over the group's rows r of dout[r,:]^T x[r,:],   db_g = sum of dout[r,:]
//
// Both operands have the summed index across their rows and are read as they lie: slabs of 64 rows by 64 columns, swizzled by
// 128 bytes, in the other major order.  A pair of blocks makes a tile of 256 x 256 of dW, each block with its own half of the
// slabs: shared memory then takes in and gives out 64 KB for 64 rows, in the 512 cycles of their products, where the 96 KB of
// a single block's 128 x 256 are more than it can move.  Single blocks stay for narrow layers, where half a pair would idle.
// The rows behind a group's end are the next group's: they are cleared in the last stage, in both operands (zero times a
// value that is not a number would not be zero).  A warp of its own in each block sees such a stage land, clears it and hands it on
// to the warp that issues the products (the even block's, for both), from block to block with a release at cluster scope.  The
// copies of all other stages are counted where the products wait: a release for every stage takes twice the time.
// Four more warps add up dout's columns for db from the same stages, where the tile is its row's first.  They read a stage behind its
// products, which alone tell the odd block that its copies have landed, and only such a stage waits for them.
// The units of work get equal shares of it (linear_grouped.cuh), so that a single long sum with 25 tiles keeps all SMs busy.
// 25216 rows of 16 groups, 1024 x 4096: 193 us (tensor pipe active 65 %), 182 without biases; one group of 8192 rows, 4096 x 4096:
// 200 us (1370 TFLOP/s), 188 without; 32896 rows, 1280 x 1280: 100 us.
#include "linear_grouped.cuh"
#include "linear_grouped_tc.cuh"

#include <cmath>

namespace vit {

using namespace grouped;

namespace {

constexpr int TN = 256, EPI_WARPS = 8, SUM_WARPS = 4, DW_THREADS = 32 * (2 + EPI_WARPS + SUM_WARPS + 1);
template <int CTAS> struct DwCfg {
  static constexpr int B_SLABS = 4 / CTAS, A_BYTES = 2 * SLAB_BYTES, STAGE_BYTES = A_BYTES + B_SLABS * SLAB_BYTES, STAGES = CTAS == 2 ? 6 : 4;
  static constexpr int STAGING_BYTES = EPI_WARPS * 4096, SMEM_BYTES = STAGES * STAGE_BYTES + STAGING_BYTES + 1024 + 384;
};

struct DwArgs {
  GroupedShape shape;
  int in, out, tiles_in, tiles, least, cuts;  // tiles of a group: ceil(out / (128 blocks)) x ceil(in / 256)
  float* dbias;                    // [groups][out] or nullptr
  float* part_bias;                // [units][2][128 blocks]
  float* part;                     // [units][2][epilogue warps of the blocks][4][8][32][4]: parts of tiles, as the warps hold them
  int* table;                      // where the units' shares begin
  int* dev_status;
};
struct DwMaps { CUtensorMap dout, x, dw; };

__device__ __forceinline__ void tma_store_3d(const CUtensorMap* tm, uint32_t src, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(reinterpret_cast<uint64_t>(tm)), "r"(src),
               "r"(x), "r"(y), "r"(z)
               : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}

template <int CTAS>
__global__ void __launch_bounds__(DW_THREADS, 1)
grouped_dw_kernel(const __grid_constant__ DwMaps m, const __grid_constant__ DwArgs p) {
  using C = DwCfg<CTAS>;
  constexpr int STAGES = C::STAGES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t tiles = smem_u32(smem), staging = tiles + STAGES * C::STAGE_BYTES;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + STAGES * C::STAGE_BYTES + C::STAGING_BYTES);
  const uint32_t landed = smem_u32(bars), cleared = landed + 8 * STAGES, ready = cleared + 8 * STAGES, used = ready + 8 * STAGES, multiplied = used + 8 * STAGES,
                 summed = multiplied + 8 * STAGES, tfull = summed + 8 * STAGES, tempty = tfull + 16, drain = tempty + 16;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 6 * STAGES + 5);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CTAS == 2 ? cluster_ctarank() : 0u;
  const int self = (int)blockIdx.x / CTAS, units = (int)gridDim.x / CTAS;

  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(landed + 8 * i, 1);
      mbar_init(cleared + 8 * i, 1);
      mbar_init(ready + 8 * i, 1);
      mbar_init(used + 8 * i, 1);                                       // by the products
      mbar_init(multiplied + 8 * i, 1);                                 // the same, where columns are summed
      mbar_init(summed + 8 * i, SUM_WARPS);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(tfull + 8 * i, 1);
      mbar_init(tempty + 8 * i, EPI_WARPS * CTAS);
    }
    mbar_init(drain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_map(&m.dout);
    prefetch_map(&m.x);
    prefetch_map(&m.dw);
  }
  if (warp == 1) {
    if (CTAS == 2) tmem_alloc_pair(smem_u32(tmem_slot), 512);
    else tmem_alloc(smem_u32(tmem_slot), 512);
  }
  tc_fence_before();
  __syncthreads();
  if (CTAS == 2) cluster_sync();          // the partner's barriers are initialised before anyone signals them
  tc_fence_after();
  grid_dependency_wait();
  grid_launch_dependents();
  const uint32_t tmem = *tmem_slot;
  const Share share = find_share(p.shape, p.tiles, units, self, p.least, p.cuts, reinterpret_cast<int*>(smem + STAGES * C::STAGE_BYTES) /* staging */,
                                 rank == 0 ? p.table : nullptr);
  __syncthreads();
  PartWalk work(p.shape, p.tiles, lane, share, self, units);
  Part part;
  int stage = 0;
  uint32_t phase = 0;

  if (warp == 0) {
    // ---------------------------------------------------------------- TMA producer
    long long fills = 0;
    uint32_t tails = 0, turns = 0, sums = 0, sum_turns = 0;             // (sums: the stages whose last fill has its columns summed)
    bool ok = true;
    while (ok && work.next(part)) {
      const bool mine = p.dbias && part.tile % p.tiles_in == 0;
      const int n0 = part.tile / p.tiles_in * (BM * CTAS) + (int)rank * BM, k0 = part.tile % p.tiles_in * TN + (int)rank * (TN / CTAS);
      for (int kb = 0; kb < part.blocks(); ++kb) {
        if (!warp_wait(used + 8 * stage, phase ^ 1, abort_flag) ||
            ((sums >> stage & 1) && !warp_wait(summed + 8 * stage, (sum_turns >> stage & 1) ^ 1, abort_flag))) {
          ok = false;
          break;
        }
        ++fills;
        sums = mine ? sums | 1u << stage : sums & ~(1u << stage);
        sum_turns ^= (mine ? 1u : 0u) << stage;
        const int row = part.begin + part.unit(kb) * DW_ROWS;
        const bool tail = has_tail(part.end - row);
        tails = tail ? tails | 1u << stage : tails & ~(1u << stage);
        turns ^= (tail ? 1u : 0u) << stage;
        if (elect_one()) {                             // (by lane 0 instead: 212 us for 198 at 8192 rows, 4096 x 4096)
          const uint32_t sa = tiles + stage * C::STAGE_BYTES, to = announce<CTAS>(landed + 8 * stage, ready + 8 * stage, tail, rank, C::STAGE_BYTES);
#pragma unroll
          for (int s = 0; s < 2; ++s) load_2d<CTAS>(sa + s * SLAB_BYTES, &m.dout, n0 + 64 * s, row, to);
#pragma unroll
          for (int s = 0; s < C::B_SLABS; ++s) load_2d<CTAS>(sa + C::A_BYTES + s * SLAB_BYTES, &m.x, k0 + 64 * s, row, to);
        }
        __syncwarp();
        if (++stage == STAGES) { stage = 0; phase ^= 1; }
      }
    }
    if (*abort_flag && lane == 0) drain_fills(landed, ready, STAGES, fills, tails, turns, rank == 0);
  } else if (warp == 1) {
    // ---------------------------------------------------------------- products
    if (rank == 0) {
      constexpr uint32_t id = instr_desc(BM * CTAS, TN, true, true);
      int buf = 0;
      uint32_t aphase = 0;
      bool ok = true;
      while (ok && work.next(part)) {
        if (!warp_wait(tempty + 8 * buf, aphase ^ 1, abort_flag)) break;
        tc_fence_after();
        const uint32_t d = tmem + (uint32_t)(buf * TN);
        const bool mine = p.dbias && part.tile % p.tiles_in == 0;
        for (int kb = 0; kb < part.blocks(); ++kb) {
          if (!warp_wait(ready + 8 * stage, phase, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint32_t sa = uniform(tiles + stage * C::STAGE_BYTES);
          const int steps = (min(DW_ROWS, part.end - part.begin - part.unit(kb) * DW_ROWS) + 15) / 16;
          const uint64_t ad = smem_desc(sa, SLAB_BYTES), bd = smem_desc(sa + C::A_BYTES, SLAB_BYTES);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < 4; ++k)                // 16 rows of 128 bytes
              if (k < steps) product<CTAS>(d, ad + (uint64_t)(128 * k), bd + (uint64_t)(128 * k), id, (kb > 0 || k > 0) ? 1u : 0u);
            commit<CTAS>(used + 8 * stage);
            if (mine) commit<CTAS>(multiplied + 8 * stage);
          }
          __syncwarp();
          if (++stage == STAGES) { stage = 0; phase ^= 1; }
        }
        if (!ok) break;
        if (elect_one()) commit<CTAS>(tfull + 8 * buf);
        __syncwarp();
        if (++buf == 2) { buf = 0; aphase ^= 1; }
      }
      if (*abort_flag) drain_products<CTAS>(drain);
    }
  } else if (warp == 2 + EPI_WARPS + SUM_WARPS) {
    // ---------------------------------------------------------------- the groups' last rows
    uint32_t turns = 0;
    bool ok = true;
    while (ok && work.next(part)) {
      for (int kb = 0; kb < part.blocks(); ++kb) {
        const int rows = part.end - part.begin - part.unit(kb) * DW_ROWS;
        if (has_tail(rows)) {                          // the others of their 16 become zero
          if (!warp_wait(landed + 8 * stage, turns >> stage & 1, abort_flag)) { ok = false; break; }
          const uint32_t sa = tiles + stage * C::STAGE_BYTES;
          for (int s = 0; s < 2 + C::B_SLABS; ++s)
            for (int i = rows * 8 + lane; i < (rows + 15) / 16 * 128; i += 32)
              asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(sa + (uint32_t)(s * SLAB_BYTES + i * 16)), "r"(0u) : "memory");
          if (!hand_on<CTAS>(ready + 8 * stage, cleared + 8 * stage, turns >> stage & 1, rank, lane, abort_flag)) { ok = false; break; }
          turns ^= 1u << stage;
        }
        if (++stage == STAGES) stage = 0;
      }
    }
  } else if (warp < 2 + EPI_WARPS) {
    // ---------------------------------------------------------------- epilogue
    if (blockIdx.x == 0 && warp == 2) report_bad_groups(p.shape, p.dev_status, lane);
    const int ew = warp - 2, quarter = warp & 3, half = ew >> 2;
    const uint32_t stg = staging + ew * 4096;
    int buf = 0;
    uint32_t aphase = 0;
    while (work.next(part)) {
      if (!warp_wait(tfull + 8 * buf, aphase, abort_flag)) break;
      tc_fence_after();
      const int n0 = part.tile / p.tiles_in * (BM * CTAS) + (int)rank * BM + quarter * 32, k0 = part.tile % p.tiles_in * TN + half * 128;
      const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * TN + half * 128);
      if (part.whole()) {
#pragma unroll 1
        for (int cb = 0; cb < 2; ++cb) {
          if (k0 + 64 * cb >= p.in || n0 >= p.out) break;
          if (lane == 0) tma_store_wait_read();
          __syncwarp();
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t r[32];
            tmem_ld32(taddr + 64 * cb + 32 * h, r);
            tmem_ld_wait_for(r);
            float2 v[16];
#pragma unroll
            for (int e = 0; e < 16; ++e)
              v[e] = part.end > part.begin ? make_float2(__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1])) : make_float2(0.f, 0.f);
            put_half(v, stg, lane, h);
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) tma_store_3d(&m.dw, stg, k0 + 64 * cb, n0, part.group);      // rows and columns beyond are clipped
        }
      } else {
        // 4 columns of 32 rows side by side; columns and rows that do not exist, too: they are not looked at
        float* to = p.part + (((int64_t)(self * 2 + part.slot()) * CTAS + rank) * EPI_WARPS + ew) * (32 * 128) + lane * 4;
#pragma unroll 1
        for (int q = 0; q < 4; ++q) {
          uint32_t r[32];
          tmem_ld32(taddr + 32 * q, r);
          tmem_ld_wait_for(r);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            *reinterpret_cast<uint4*>(to + (q * 8 + e) * 128) = make_uint4(r[4 * e], r[4 * e + 1], r[4 * e + 2], r[4 * e + 3]);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) give_back<CTAS>(tempty + 8 * buf);
      if (++buf == 2) { buf = 0; aphase ^= 1; }
    }
    if (lane == 0) tma_store_wait_all();
  } else if (warp < 2 + EPI_WARPS + SUM_WARPS && p.dbias) {
    // ---------------------------------------------------------------- sums of dout's columns
    // a warp has 32 columns; a lane 8 of them and every eighth row, such that eight lanes meet all banks
    const int sw = warp - 2 - EPI_WARPS, slab = sw >> 1, ck = (sw & 1) * 4 + (lane & 3), first = (lane >> 3) | (lane & 4);
    uint32_t turns = 0;
    bool ok = true;
    while (ok && work.next(part)) {
      if (part.tile % p.tiles_in != 0) {
        stage = (stage + part.blocks()) % STAGES;
        continue;
      }
      float2 sum[4] = {};
      for (int kb = 0; kb < part.blocks(); ++kb) {
        if (!warp_wait(multiplied + 8 * stage, turns >> stage & 1, abort_flag)) { ok = false; break; }
        turns ^= 1u << stage;
        const uint32_t from = tiles + stage * C::STAGE_BYTES + slab * SLAB_BYTES;
        const int rows = part.end - part.begin - part.unit(kb) * DW_ROWS;
        uint32_t w[8][4];
#pragma unroll
        for (int i = 0; i < 8; ++i) read_chunk(w[i], from, first + 8 * i, ck);
        __syncwarp();
        if (lane == 0) mbar_arrive(summed + 8 * stage);  // releases behind what has been read
        float2 some[4] = {};
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (first + 8 * i < rows) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              some[e] = __fadd2_rn(some[e], make_float2(__uint_as_float(w[i][e] << 16), __uint_as_float(w[i][e] & 0xffff0000u)));
          }
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = __fadd2_rn(sum[e], some[e]);
        if (++stage == STAGES) stage = 0;
      }
      if (!ok) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
          sum[e].x += __shfl_xor_sync(0xffffffffu, sum[e].x, o);
          sum[e].y += __shfl_xor_sync(0xffffffffu, sum[e].y, o);
        }
      const int c = slab * 64 + ck * 8, n0 = part.tile / p.tiles_in * (BM * CTAS) + (int)rank * BM;
      if (lane < 4 && n0 + c < p.out) {
        float4* to = reinterpret_cast<float4*>(part.whole() ? p.dbias + (int64_t)part.group * p.out + n0 + c
                                                            : p.part_bias + (((int64_t)self * 2 + part.slot()) * CTAS + rank) * BM + c);
        to[0] = make_float4(sum[0].x, sum[0].y, sum[1].x, sum[1].y);
        to[1] = make_float4(sum[2].x, sum[2].y, sum[3].x, sum[3].y);
      }
    }
  }

  __syncwarp();
  if (CTAS == 2 && *abort_flag)
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_to_cta(smem_u32(const_cast<int*>(abort_flag)), rank ^ 1u)), "r"(1) : "memory");
  tc_fence_before();
  __syncthreads();
  if (CTAS == 2) cluster_sync();          // neither block leaves while the other may still touch it
  tc_fence_after();
  if (threadIdx.x == 0 && *abort_flag) atomicExch(p.dev_status, (int)VIT_ERR_TIMEOUT);
  if (warp == 1) {
    __syncwarp();
    if (CTAS == 2) tmem_dealloc_pair(tmem, 512);
    else tmem_dealloc(tmem, 512);
  }
}

// Tiles that were cut between blocks: their parts are added in the order of their rows.  A block of this kernel looks at the
// begin of one share; it is its task if the tile there began in the share before.  Several blocks share a tile: a warp's 32 x 128
// of the tensor-core kernel, 16 rows of the fp32 one.
template <typename T> __device__ __forceinline__ void store4(T* to, float4 v);
template <> __device__ __forceinline__ void store4(float* to, float4 v) { *reinterpret_cast<float4*>(to) = v; }
template <> __device__ __forceinline__ void store4(bf16* to, float4 v) {
  uint2 o;
  __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y), hi = __floats2bfloat162_rn(v.z, v.w);
  o.x = *reinterpret_cast<uint32_t*>(&lo);
  o.y = *reinterpret_cast<uint32_t*>(&hi);
  *reinterpret_cast<uint2*>(to) = o;
}
constexpr int JOIN_THREADS = 256;
template <typename T, int ROWS, int COLS>
__global__ void __launch_bounds__(JOIN_THREADS, 4)
grouped_join_kernel(const GroupedShape shape, int in, int out, int tiles_in, int tiles, int blocks, const int* __restrict__ table,
                    const float* __restrict__ part, const float* __restrict__ part_bias, T* __restrict__ dw, float* __restrict__ dbias) {
  constexpr bool WARPS = sizeof(T) == 2;                          // parts lie as the epilogue warps of the tensor-core kernel hold them
  constexpr int N = (WARPS ? 32 * 128 : 16 * COLS) / 4 / JOIN_THREADS;
  const int lane = threadIdx.x & 31, block = (int)blockIdx.x + 1;
  grid_dependency_wait();
  grid_launch_dependents();
  const int begin = table[block], end = table[block + 1];
  if (begin >= end || begin == table[0]) return;
  PartWalk work(shape, tiles, lane, Share{0, begin, begin + 1, 1}, 0, 1);
  Part here;
  if (!work.next(here) || here.from == 0) return;                                // a tile begins here: nothing is cut
  const int tile_begin = begin - here.from, tile_end = tile_begin + here.all;
  int before = block - 1;
  while (table[before] == begin) --before;                                       // blocks without a share
  if (table[before] > tile_begin) return;                                        // cut before, too: not this block's task
  const int n0 = here.tile / tiles_in * ROWS, k0 = here.tile % tiles_in * COLS, piece = (int)blockIdx.y;
  const float* mine = part + (WARPS ? piece * (32 * 128) : piece * 16 * COLS) + 4 * threadIdx.x;
  float4 sum[N];
#pragma unroll
  for (int i = 0; i < N; ++i) sum[i] = *reinterpret_cast<const float4*>(mine + ((int64_t)before * 2 + 1) * ROWS * COLS + 4 * JOIN_THREADS * i);
  const bool bias = dbias && k0 == 0 && piece == 0 && threadIdx.x < ROWS;
  float b = bias ? part_bias[((int64_t)before * 2 + 1) * ROWS + threadIdx.x] : 0.f;
  // two parts at a time, all their values under way together
  for (int first = block; first < blocks && table[first] < tile_end; first += 2) {
    float4 v[2][N];
    float c[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int who = first + k;
      const bool some = who < blocks && table[who] < tile_end && table[who + 1] > table[who];          // (blocks without a share add zeros)
#pragma unroll
      for (int i = 0; i < N; ++i)
        v[k][i] = some ? *reinterpret_cast<const float4*>(mine + (int64_t)who * 2 * ROWS * COLS + 4 * JOIN_THREADS * i) : make_float4(0.f, 0.f, 0.f, 0.f);
      c[k] = bias && some ? part_bias[(int64_t)who * 2 * ROWS + threadIdx.x] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
      for (int i = 0; i < N; ++i) sum[i] = make_float4(sum[i].x + v[k][i].x, sum[i].y + v[k][i].y, sum[i].z + v[k][i].z, sum[i].w + v[k][i].w);
      b += c[k];
    }
  }
  if (bias && n0 + (int)threadIdx.x < out) dbias[(int64_t)here.group * out + n0 + threadIdx.x] = b;
  if (WARPS) {
    // rows belong to lanes there; here they are written side by side
    __shared__ float turned[32][128 + 4];
    // warp 2 + w of a block has the rows of its quarter of tensor memory
    const int block_of_pair = piece / EPI_WARPS, w = piece % EPI_WARPS;
    const int row0 = block_of_pair * BM + ((w + 2) & 3) * 32, col0 = (w >> 2) * 128;
#pragma unroll
    for (int i = 0; i < N; ++i) *reinterpret_cast<float4*>(&turned[lane][4 * ((JOIN_THREADS / 32) * i + (threadIdx.x >> 5))]) = sum[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = i * JOIN_THREADS + (int)threadIdx.x, r = at / 32, c = at % 32 * 4, n = n0 + row0 + r, k = k0 + col0 + c;
      if (n < out && k < in) store4(dw + ((int64_t)here.group * out + n) * in + k, *reinterpret_cast<const float4*>(&turned[r][c]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = (i * JOIN_THREADS + (int)threadIdx.x) * 4, n = n0 + piece * 16 + at / COLS, k = k0 + at % COLS;
      if (n < out && k < in) store4(dw + ((int64_t)here.group * out + n) * in + k, sum[i]);
    }
  }
}

struct DwTiling { int rows, cols, tiles_in, tiles, blocks, least, split; bool cuts; };       // blocks: units of work, pairs where a tile has 256 rows
DwTiling tiling_of(bool act_bf16, const GroupedShape& shape, int in, int out) {
  DwTiling t;
  // A pair's tile takes 0.87 of the time of its two halves from single blocks (180 against 207 us at 25216 rows of 16 groups,
  // 1024 x 4096), and is wasted where it hangs over (1536 x 384: 57 against 50 us).
  const bool pair = act_bf16 && (out + 255) / 256 * 1.74 <= (out + 127) / 128;
  t.rows = pair ? 256 : 128;
  t.cols = act_bf16 ? TN : 128;
  t.tiles_in = (in + t.cols - 1) / t.cols;
  const int64_t tiles = (int64_t)t.tiles_in * ((out + t.rows - 1) / t.rows);
  t.tiles = (int)tiles;
  // as many as the rows can need: the kernels, which see the groups' lengths, may use fewer
  const int64_t units = tiles * ((int64_t)shape.rows / DW_ROWS + shape.groups), whole = tiles * shape.groups;
  // A tile cut into n parts saves (1 - 1 / n) of its time, 0.3 (5) us a unit, and costs about 0.35 us a part when they are joined:
  // shares of sqrt(1.2 (0.07) units of a tile) are the best (12608 rows, 768 x 192: 31 us with 8 units, 24 with 14).
  const int root = (int)std::sqrt((double)(shape.rows / DW_ROWS));
  t.least = act_bf16 ? (root > DW_LEAST ? root : DW_LEAST) : (root / 4 > DW_LEAST_F32 ? root / 4 : DW_LEAST_F32);
  const int64_t least = t.least, wanted = units / least > whole ? units / least : whole;
  const int64_t most = pair ? DW_BLOCKS / 2 : act_bf16 ? DW_BLOCKS : DW_BLOCKS_F32;
  // few rows: no tile is worth a cut, and neither parts nor a second kernel are needed
  t.cuts = shape.rows > (act_bf16 ? DW_LEAST : DW_LEAST_F32) * DW_ROWS;
  t.blocks = (int)((t.cuts ? wanted : whole) < most ? (wanted < 1 ? 1 : t.cuts ? wanted : whole) : most);
  // One sum for few tiles: a cluster's two or four pairs to a tile need neither parts in memory nor the second kernel, 7 to 10 us,
  // but leave pairs idle, 0.42 us for each unit that a pair has more than a share: even at 22, by the sum of both.  With clusters and
  // with shares: 577 rows, 1280 x 1280: 14 and 20 us; 3152, 1024 x 2048: 22 and 29; 4000, 1536 x 1280: 25 and 31; 6000, 768 x 768: 24 and
  // 27; 7000, 1280 x 1280: 34 and 37; 8224: 39 and 40; 9000: 43 and 42; 12608, 768 x 768: 33 and 32; 1091, 520 x 776: 19 and 19.  Not every
  // SM finds partners: 14 clusters of eight blocks run at once and 16 do not (2000 rows, 1024 x 1024: 29 us), of four 32 do.
  t.split = 1;
  if (t.cuts && pair && shape.groups == 1 && tiles <= 32) {
    const int split = tiles <= 14 ? 4 : 2, sum = (shape.rows + DW_ROWS - 1) / DW_ROWS, even = (int)(sum * tiles / most);
    if ((sum + split - 1) / split - (even > t.least ? even : t.least) <= 22) {
      t.split = split;
      t.cuts = false;
    }
  }
  return t;
}

}  // namespace

size_t grouped_dw_floats(bool act_bf16, const GroupedShape& shape, int in, int out_features) {
  const DwTiling t = tiling_of(act_bf16, shape, in, out_features);
  return (size_t)64 * ((DW_TABLE + 63) / 64) + (t.cuts ? (size_t)t.blocks : 0) * 2 * ((size_t)t.rows * t.cols + t.rows);
}

GroupedDw grouped_dw_plan(const GroupedCall& c, bool act_bf16) {
  const DwTiling t = tiling_of(act_bf16, c.shape, c.in, c.out_features);
  float* part = c.partial + 64 * ((DW_TABLE + 63) / 64);                        // behind the table
  return GroupedDw{t.rows, t.tiles_in, t.tiles, t.blocks, t.least, t.split, t.cuts, part, part + (size_t)t.blocks * 2 * t.rows * t.cols, reinterpret_cast<int*>(c.partial)};
}

template <int CTAS>
static cudaError_t launch_dw(const DwMaps& m, const DwArgs& p, int units, cudaStream_t s) {
  static PerDeviceFlag configured;
  if (cudaError_t e = ensure_dynamic_smem(configured, grouped_dw_kernel<CTAS>, DwCfg<CTAS>::SMEM_BYTES)) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(units * CTAS));
  cfg.blockDim = dim3(DW_THREADS);
  cfg.dynamicSmemBytes = DwCfg<CTAS>::SMEM_BYTES;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = CTAS;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, grouped_dw_kernel<CTAS>, m, p);
}

cudaError_t launch_grouped_dw_bf16(const GroupedCall& c, cudaStream_t s) {
  const GroupedDw plan = grouped_dw_plan(c, true);
  if (plan.split > 1) return launch_grouped_dw_few(c, plan, s);
  DwMaps m;
  DwArgs p{c.shape, c.in, c.out_features, plan.tiles_in, plan.tiles, plan.least, plan.cuts, c.dbias, plan.part_bias, plan.part, plan.table, c.dev_status};
  // without rows nothing is read, and any map will do
  const int64_t rows = c.shape.rows > 0 ? c.shape.rows : 1;
  const void *dout = c.shape.rows > 0 ? c.dout : c.dw, *x = c.shape.rows > 0 ? c.x : c.dw;
  if (!encode_rows(&m.dout, dout, rows, c.out_features, c.lddout, DW_ROWS) || !encode_rows(&m.x, x, rows, c.in, c.ldx, DW_ROWS) ||
      !encode_weights(&m.dw, c.dw, c.shape.groups, c.out_features, c.in, 32))
    return cudaErrorInvalidValue;
  return plan.rows == 256 ? launch_dw<2>(m, p, plan.blocks, s) : launch_dw<1>(m, p, plan.blocks, s);
}

template <typename T, int ROWS, int COLS>
static cudaError_t launch_join(const GroupedCall& c, const GroupedDw& plan, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(plan.blocks - 1), sizeof(T) == 2 ? ROWS * COLS / (32 * 128) : ROWS / 16);
  cfg.blockDim = dim3(JOIN_THREADS);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, grouped_join_kernel<T, ROWS, COLS>, c.shape, c.in, c.out_features, plan.tiles_in, plan.tiles, plan.blocks,
                            (const int*)plan.table, (const float*)plan.part, (const float*)plan.part_bias, static_cast<T*>(c.dw), c.dbias);
}
cudaError_t launch_grouped_join(const GroupedCall& c, bool act_bf16, cudaStream_t s) {
  const GroupedDw plan = grouped_dw_plan(c, act_bf16);
  if (!act_bf16) return launch_join<float, 128, 128>(c, plan, s);
  return plan.rows == 256 ? launch_join<bf16, 256, TN>(c, plan, s) : launch_join<bf16, 128, TN>(c, plan, s);
}

}  // namespace vit
