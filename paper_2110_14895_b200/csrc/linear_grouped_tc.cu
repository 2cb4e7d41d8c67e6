// Linear layers by group on the 5th-generation tensor cores (bf16): rows times their group's weights, forwards and backwards.
//
//   forward          out[r,:] = f(x[r,:] . W_g^T + b_g),      f: identity, GELU (the argument kept too), + residual
//   input gradient   dx[r,:] = (dout[r,:] . W_g) gelu'(pre[r,:])
//
// Persistent blocks, one per SM: a producer warp (TMA), a warp that issues the products, eight or sixteen epilogue warps,
// two accumulators in tensor memory, so that a tile's epilogue runs beside the next tile's products.  Tiles are numbered group
// after group; each warp finds its tiles in the offsets by itself, 32 groups at a look, so that a call needs neither a
// launch nor a table for them.  A tile begins at its group's first row (TMA copies may begin at any row) and its rows behind
// the group's end are computed and left unwritten: whole pieces of 32 rows leave by TMA, the last one row by row.
//
// The weights are read as they lie, [groups][out][in], for both directions: with the summed index along a row (forwards) or
// across rows (backwards, slabs of 64 columns in the other major order), through a map of three dimensions whose bounds make
// what lies behind a group's weights zero and not the next group's values.
//
// Bound by shared memory and the way out: a stage of a pair takes in and gives out 64 KB in the 512 cycles of its products, 125 of
// the 128 bytes a cycle, and a tile's way out 64 KB twice more for each result; with GELU's argument kept the accumulator and the
// biases are read twice, and a warp's one piece is waited for between its results.  25216 rows of 16 groups, 1024 -> 4096: 156 us
// with a bias (1360 TFLOP/s), 172 with GELU, 195 with its argument kept (tensor pipe active 70 %); the input gradient of the layer
// behind it 160, 196 with GELU's slope (72 %); 4096 -> 1024 with a residual 161.  Results sent straight from registers, rows of 32
// bytes a thread, took 215 us where these took 203.
//
// Every mbarrier wait is bounded; on expiry the block raises the device status word, lets the copies and products in flight
// finish (bounded), frees tensor memory and leaves.
#include "linear_grouped.cuh"
#include "linear_grouped_tc.cuh"

namespace vit {

using namespace grouped;

namespace {

template <int BN, int CTAS, int FINISH> struct Cfg {
  static constexpr int B_ROWS = BN / CTAS;                 // columns of the result whose weights this block loads
  static constexpr int A_BYTES = BM * BK * 2, B_BYTES = B_ROWS * BK * 2, STAGE_BYTES = A_BYTES + B_BYTES;
  // An epilogue warp has 32 rows and 64 columns of a tile at a time, and 4 KB of shared memory for them.  Eight warps are
  // enough to add a bias, and leave room for a stage more (163 against 168 us at 25216 rows of 16 groups, 1024 x 4096);
  // GELU, its slope (213 against 200 us) and what is read besides take sixteen.
  static constexpr int EPI_WARPS = BN == 256 && FINISH != F_BIAS ? 16 : 8, STEPS = BN / 16 / EPI_WARPS, THREADS = (2 + EPI_WARPS) * 32;
  static constexpr int STAGING_BYTES = EPI_WARPS * 4096;
  static constexpr int ROOM = 232448 - 1024 /* alignment */ - 512 /* barriers */ - STAGING_BYTES;
  static constexpr int STAGES = ROOM / STAGE_BYTES < 6 ? ROOM / STAGE_BYTES : 6;
  static constexpr int TMEM_COLS = 2 * BN;
  static constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + STAGING_BYTES + 1024 + 512;
};

struct RowsArgs {
  GroupedShape shape;
  int width, sum;                  // columns of the result; length of the sums
  const float* bias;               // [groups][width] or nullptr
  bf16* out; int64_t ldo;
  bf16* pre; int64_t ldp;          // F_GELU_PRE: written
  int tiles_n;
  int* dev_status;
};
struct RowsMaps { CUtensorMap a, w, out, other; };     // other: the argument written, or the residual / argument read

template <int BN, int CTAS, int FINISH, bool ACROSS>
__global__ void __launch_bounds__(Cfg<BN, CTAS, FINISH>::THREADS, 1)
grouped_rows_kernel(const __grid_constant__ RowsMaps m, const __grid_constant__ RowsArgs p) {
  using C = Cfg<BN, CTAS, FINISH>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t tiles = smem_u32(smem), staging = tiles + C::STAGES * C::STAGE_BYTES;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::STAGES * C::STAGE_BYTES + C::STAGING_BYTES);
  const uint32_t full = smem_u32(bars), empty = full + 8 * C::STAGES, tfull = empty + 8 * C::STAGES, tempty = tfull + 16,
                 landed = tempty + 16 /* [EPI_WARPS] */, drain = landed + 8 * C::EPI_WARPS;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * C::STAGES + 4 + C::EPI_WARPS + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CTAS == 2 ? cluster_ctarank() : 0u;
  const int unit = blockIdx.x / CTAS, units = gridDim.x / CTAS;

  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int i = 0; i < C::STAGES; ++i) {
      mbar_init(full + 8 * i, 1);
      mbar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(tfull + 8 * i, 1);
      mbar_init(tempty + 8 * i, C::EPI_WARPS * CTAS);
    }
    for (int i = 0; i < C::EPI_WARPS; ++i) mbar_init(landed + 8 * i, 1);
    mbar_init(drain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_map(&m.a);
    prefetch_map(&m.w);
    prefetch_map(&m.out);
  }
  if (warp == 1) {
    if (CTAS == 2) tmem_alloc_pair(smem_u32(tmem_slot), (uint32_t)C::TMEM_COLS);
    else tmem_alloc(smem_u32(tmem_slot), (uint32_t)C::TMEM_COLS);
  }
  tc_fence_before();
  __syncthreads();
  if (CTAS == 2) cluster_sync();          // the partner's barriers are initialised before anyone signals them
  tc_fence_after();
  grid_dependency_wait();                 // set-up above overlaps the end of the kernel before this one
  grid_launch_dependents();
  const uint32_t tmem = *tmem_slot;
  const int blocks_k = (p.sum + BK - 1) / BK;
  const TileCount count{BM * CTAS, p.tiles_n};
  GroupAt at;

  if (warp == 0) {
    // ---------------------------------------------------------------- TMA producer
    GroupWalk<TileCount> walk(p.shape, count, lane);
    int stage = 0;
    uint32_t phase = 0;
    long long fills = 0;                           // stages filled so far (this block's share)
    bool ok = true;
    for (int tile = unit; ok && walk.find(tile, at); tile += units) {
      const int local = tile - at.before, mt = local / p.tiles_n;
      const int row = at.begin + mt * (BM * CTAS) + (int)rank * BM, col = (local - mt * p.tiles_n) * BN + (int)rank * C::B_ROWS;
      for (int kb = 0; kb < blocks_k; ++kb) {
        if (!warp_wait(empty + 8 * stage, phase ^ 1, abort_flag)) { ok = false; break; }
        ++fills;
        if (lane == 0) {
          const uint32_t sa = tiles + stage * C::STAGE_BYTES, sb = sa + C::A_BYTES;
          // both blocks' copies of a pair are counted on the even one's barrier, which expects all the bytes
          const uint32_t fb = CTAS == 2 ? map_to_cta(full + 8 * stage, 0) : full + 8 * stage;
          if (rank == 0) mbar_arrive_expect_tx(full + 8 * stage, CTAS * C::STAGE_BYTES);
          load_2d<CTAS>(sa, &m.a, kb * BK, row, fb);
          if (ACROSS) {
#pragma unroll
            for (int s = 0; s < C::B_ROWS / 64; ++s) load_3d<CTAS>(sb + s * SLAB_BYTES, &m.w, col + 64 * s, kb * BK, at.group, fb);
          } else {
            load_3d<CTAS>(sb, &m.w, kb * BK, col, at.group, fb);
          }
        }
        __syncwarp();
        if (++stage == C::STAGES) { stage = 0; phase ^= 1; }
      }
    }
    if (*abort_flag && rank == 0) drain_stages(full, C::STAGES, fills);
  } else if (warp == 1) {
    // ---------------------------------------------------------------- products
    if (rank == 0) {
      GroupWalk<TileCount> walk(p.shape, count, lane);
      constexpr uint32_t id = instr_desc(BM * CTAS, BN, false, ACROSS);
      int stage = 0, buf = 0;
      uint32_t phase = 0, aphase = 0;
      bool ok = true;
      for (int tile = unit; ok && walk.find(tile, at); tile += units) {
        if (!warp_wait(tempty + 8 * buf, aphase ^ 1, abort_flag)) break;
        tc_fence_after();
        const uint32_t d = tmem + (uint32_t)(buf * BN);
        for (int kb = 0; kb < blocks_k; ++kb) {
          if (!warp_wait(full + 8 * stage, phase, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint32_t sa = uniform(tiles + stage * C::STAGE_BYTES);
          const uint64_t ad = smem_desc(sa), bd = smem_desc(sa + C::A_BYTES, ACROSS ? SLAB_BYTES : 16);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < BK / 16; ++k)      // 16 of the summed index: 32 bytes along a row, or 16 rows of 128 bytes
              product<CTAS>(d, ad + (uint64_t)(2 * k), bd + (uint64_t)(ACROSS ? 128 * k : 2 * k), id, (kb > 0 || k > 0) ? 1u : 0u);
            commit<CTAS>(empty + 8 * stage);       // frees the stage when these products are done
          }
          __syncwarp();
          if (++stage == C::STAGES) { stage = 0; phase ^= 1; }
        }
        if (!ok) break;
        if (elect_one()) commit<CTAS>(tfull + 8 * buf);
        __syncwarp();
        if (++buf == 2) { buf = 0; aphase ^= 1; }
      }
      if (*abort_flag) drain_products<CTAS>(drain);
    }
  } else {
    // ---------------------------------------------------------------- epilogue
    if (blockIdx.x == 0 && warp == 2) report_bad_groups(p.shape, p.dev_status, lane);
    GroupWalk<TileCount> walk(p.shape, count, lane);
    const int ew = warp - 2, quarter = warp & 3, column = (ew >> 2) * (64 * C::STEPS);      // lanes of tensor memory it may read; its columns
    const uint32_t piece = staging + ew * 4096, bar = landed + 8 * ew;
    int buf = 0;
    uint32_t aphase = 0, lphase = 0;
    bool ok = true, coming = false;                                     // coming: a copy into the piece that nobody has waited for
    for (int tile = unit; walk.find(tile, at); tile += units) {
      const int local = tile - at.before, mt = local / p.tiles_n;
      const int row0 = at.begin + mt * (BM * CTAS) + (int)rank * BM + quarter * 32, col0 = (local - mt * p.tiles_n) * BN + column;
      const int rows = min(32, at.end - row0);                          // of this warp's 32; none or less: nothing is written
#pragma unroll 1
      for (int step = 0; step < C::STEPS; ++step) {
        const int c0 = col0 + 64 * step;
        const bool some = rows > 0 && c0 < p.width, last = step == C::STEPS - 1;       // the same for the whole warp
        if (some && (FINISH == F_RESIDUAL || FINISH == F_SLOPE)) {
          if (lane == 0) {                                                // comes while the accumulator is awaited
            tma_store_wait_read();
            mbar_arrive_expect_tx(bar, 4096);
            tma_load_2d(piece, &m.other, c0, row0, bar);
          }
          coming = true;
          __syncwarp();
        }
        if (step == 0 && !warp_wait(tfull + 8 * buf, aphase, abort_flag)) { ok = false; break; }
        if (some) {
          tc_fence_after();
          // 32 columns at a time: with sixteen warps a thread has 96 registers
          const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * BN + column + 64 * step);
          const float* bias = FINISH != F_SLOPE && p.bias ? p.bias + (int64_t)at.group * p.width + c0 : nullptr;
          auto sums = [&](float2 (&v)[16], int h) {
            uint32_t r[32];
            tmem_ld32(taddr + 32 * h, r);
            float4 b[8];                                                // under way with the sums
            if (FINISH != F_SLOPE) {
#pragma unroll
              for (int g = 0; g < 8; ++g)
                b[g] = bias && c0 + 32 * h + 4 * g < p.width ? __ldg(reinterpret_cast<const float4*>(bias + 32 * h) + g) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            tmem_ld_wait_for(r);
#pragma unroll
            for (int g = 0; g < 8; ++g) {
              v[2 * g] = make_float2(__uint_as_float(r[4 * g]), __uint_as_float(r[4 * g + 1]));
              v[2 * g + 1] = make_float2(__uint_as_float(r[4 * g + 2]), __uint_as_float(r[4 * g + 3]));
              if (FINISH != F_SLOPE) {
                v[2 * g] = __fadd2_rn(v[2 * g], make_float2(b[g].x, b[g].y));
                v[2 * g + 1] = __fadd2_rn(v[2 * g + 1], make_float2(b[g].z, b[g].w));
              }
            }
          };
          if (FINISH == F_GELU_PRE) {                                     // the argument goes out first
            if (lane == 0) tma_store_wait_read();
            __syncwarp();
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
              float2 v[16];
              sums(v, h);
              put_half(v, piece, lane, h);
            }
            send_rows(&m.other, p.pre, p.ldp, piece, row0, c0, rows, p.width, lane);
          }
          if (FINISH == F_RESIDUAL || FINISH == F_SLOPE) {
            if (!warp_wait(bar, lphase, abort_flag)) { ok = false; break; }
            lphase ^= 1;
            coming = false;
          }
#pragma unroll 1
          for (int h = 0; h < 2; ++h) {
            float2 v[16];
            sums(v, h);
            if (h == 1 && last) {                                         // all of the accumulator has been read
              tc_fence_before();
              __syncwarp();
              if (lane == 0) give_back<CTAS>(tempty + 8 * buf);
            }
            if (FINISH == F_GELU || FINISH == F_GELU_PRE) {
#pragma unroll
              for (int e = 0; e < 16; ++e) v[e] = gelu_2(v[e]);
            }
            if (FINISH == F_RESIDUAL || FINISH == F_SLOPE) {
#pragma unroll
              for (int ck = 0; ck < 4; ++ck) {
                uint32_t w[4];
                read_chunk(w, piece, lane, 4 * h + ck);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const float2 o = make_float2(__uint_as_float(w[e] << 16), __uint_as_float(w[e] & 0xffff0000u));
                  if (FINISH == F_RESIDUAL) v[4 * ck + e] = __fadd2_rn(v[4 * ck + e], o);
                  else v[4 * ck + e] = __fmul2_rn(v[4 * ck + e], gelu_slope_2(o));
                }
              }
            } else if (h == 0) {
              if (lane == 0) tma_store_wait_read();                       // the store before has left the piece
              __syncwarp();
            }
            put_half(v, piece, lane, h);
          }
          send_rows(&m.out, p.out, p.ldo, piece, row0, c0, rows, p.width, lane);
        } else if (last) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) give_back<CTAS>(tempty + 8 * buf);
        }
      }
      if (!ok) break;
      if (++buf == 2) { buf = 0; aphase ^= 1; }
    }
    if (lane == 0) {
      if (coming) {
        volatile int never = 0;
        mbar_wait_limit(bar, lphase, &never, DRAIN_LIMIT_CYCLES);
      }
      tma_store_wait_all();
    }
  }

  // ------------------------------------------------------------------ teardown
  __syncwarp();
  if (CTAS == 2 && *abort_flag)
    // the partner may be in a wait of its own that nothing will satisfy any more
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_to_cta(smem_u32(const_cast<int*>(abort_flag)), rank ^ 1u)), "r"(1) : "memory");
  tc_fence_before();
  __syncthreads();
  if (CTAS == 2) cluster_sync();          // neither block leaves while the other may still touch it
  tc_fence_after();
  if (threadIdx.x == 0 && *abort_flag) atomicExch(p.dev_status, (int)VIT_ERR_TIMEOUT);
  if (warp == 1) {
    __syncwarp();
    if (CTAS == 2) tmem_dealloc_pair(tmem, (uint32_t)C::TMEM_COLS);
    else tmem_dealloc(tmem, (uint32_t)C::TMEM_COLS);
  }
}

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

struct RowsLaunch { RowsMaps m; RowsArgs p; int grid; };

template <int BN, int CTAS, int FINISH, bool ACROSS>
cudaError_t launch_variant(const RowsLaunch& l, cudaStream_t s) {
  using C = Cfg<BN, CTAS, FINISH>;
  static PerDeviceFlag configured;
  auto kernel = grouped_rows_kernel<BN, CTAS, FINISH, ACROSS>;
  if (cudaError_t e = ensure_dynamic_smem(configured, kernel, C::SMEM_BYTES)) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)l.grid);
  cfg.blockDim = dim3(C::THREADS);
  cfg.dynamicSmemBytes = C::SMEM_BYTES;
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
  return cudaLaunchKernelEx(&cfg, kernel, l.m, l.p);
}
template <int BN, int CTAS>
cudaError_t launch_finish(const GroupedCall& c, Finish finish, const RowsLaunch& l, cudaStream_t s) {
  if (c.backward) return finish == F_SLOPE ? launch_variant<BN, CTAS, F_SLOPE, true>(l, s) : launch_variant<BN, CTAS, F_BIAS, true>(l, s);
  switch (finish) {
    case F_GELU: return launch_variant<BN, CTAS, F_GELU, false>(l, s);
    case F_GELU_PRE: return launch_variant<BN, CTAS, F_GELU_PRE, false>(l, s);
    case F_RESIDUAL: return launch_variant<BN, CTAS, F_RESIDUAL, false>(l, s);
    default: return launch_variant<BN, CTAS, F_BIAS, false>(l, s);
  }
}

}  // namespace

namespace grouped {

bool encode_rows(CUtensorMap* tm, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
  const EncodeTiledFn fn = encoder();
  if (!fn || !base) return false;
  // (a map's stride has 40 bits; that of a single row may be anything and is not used)
  const cuuint64_t dim[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, stride[1] = {(cuuint64_t)(rows > 1 ? ld : cols) * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, one[2] = {1, 1};
  return fn(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dim, stride, box, one,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool encode_weights(CUtensorMap* tm, const void* base, int groups, int rows, int cols, int box_rows) {
  const EncodeTiledFn fn = encoder();
  if (!fn || !base) return false;
  const cuuint64_t dim[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)groups};
  const cuuint64_t stride[2] = {(cuuint64_t)cols * 2, (cuuint64_t)cols * rows * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1}, one[3] = {1, 1, 1};
  return fn(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dim, stride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace grouped

// The tiling goes by the sizes alone (the groups' lengths are on the device): rounds of the static schedule, with half a tile
// of rows lost in every group, times the cost of a tile (a pair's 256 x 256, a block's 128 x 256, 128 x 128).
cudaError_t launch_grouped_rows_bf16(const GroupedCall& c, cudaStream_t s) {
  const int width = c.backward ? c.in : c.out_features, sum = c.backward ? c.out_features : c.in;
  const int sms = current_device_sm_count();
  if (sms < 2) return cudaErrorInvalidDevice;
  const Finish finish = c.backward ? (c.pre ? F_SLOPE : F_BIAS) : c.epilogue == 1 ? (c.pre ? F_GELU_PRE : F_GELU) : c.epilogue == 2 ? F_RESIDUAL : F_BIAS;
  const int split = grouped_few_split(c.shape, width, sum);
  if (split > 1) return launch_grouped_few_bf16(c, finish, split, s);
  auto tiles = [&](int span) { return c.shape.groups == 1 ? (double)((c.shape.rows + (int64_t)span - 1) / span) : (double)c.shape.rows / span + 0.5 * c.shape.groups; };
  auto rounds = [](double n, int units) { return n <= units ? 1.0 : n / units < 8 ? (double)(int64_t)(n / units + 0.999) : n / units; };
  const double n256 = (width + 255) / 256, n128 = (width + 127) / 128;
  const double pair = 0.92 * rounds(tiles(2 * BM) * n256, sms / 2), wide = rounds(tiles(BM) * n256, sms), narrow = 0.75 * rounds(tiles(BM) * n128, sms);
  const bool two = pair <= wide && pair <= narrow, broad = two || wide <= narrow;
  const int bn = broad ? 256 : 128, span = two ? 2 * BM : BM;
  RowsLaunch l;
  l.p = RowsArgs{c.shape, width, sum, c.backward ? nullptr : c.bias, static_cast<bf16*>(c.y), c.ldy, static_cast<bf16*>(c.pre), c.ldp,
                 (width + bn - 1) / bn, c.dev_status};
  const int64_t most = ((int64_t)c.shape.rows / span + c.shape.groups) * l.p.tiles_n;       // tiles there can be
  const int units = two ? sms / 2 : sms;
  l.grid = (int)(most < units ? most : units) * (two ? 2 : 1);
  if (!encode_rows(&l.m.a, c.x, c.shape.rows, sum, c.ldx, BM) || !encode_rows(&l.m.out, c.y, c.shape.rows, width, c.ldy, 32)) return cudaErrorInvalidValue;
  if (!encode_weights(&l.m.w, c.w, c.shape.groups, c.out_features, c.in, c.backward ? BK : bn / (two ? 2 : 1))) return cudaErrorInvalidValue;
  l.m.other = l.m.out;
  if (finish == F_GELU_PRE || finish == F_SLOPE) {
    if (!encode_rows(&l.m.other, c.pre, c.shape.rows, width, c.ldp, 32)) return cudaErrorInvalidValue;
  } else if (finish == F_RESIDUAL) {
    if (!encode_rows(&l.m.other, c.residual, c.shape.rows, width, c.ldr, 32)) return cudaErrorInvalidValue;
  }
  return two ? launch_finish<256, 2>(c, finish, l, s) : broad ? launch_finish<256, 1>(c, finish, l, s) : launch_finish<128, 1>(c, finish, l, s);
}

}  // namespace vit
