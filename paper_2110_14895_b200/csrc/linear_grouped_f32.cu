// Linear layers by group in the fp32 mode, on the fp32 pipes: rows times their group's weights forwards and backwards, and the
// weights' gradients.  Tiles of the result in registers, 16 of the summed index at a time through shared memory, the next
// pieces under way while these are multiplied; two products to an instruction (packed fp32).
// Tiles of 128 x 128 or 64 x 64, whose sums can be shared by a cluster of blocks and are joined in its shared memory (cycles_of).
// 8224 rows, 1280 x 1280: 606 us (44 TFLOP/s), the fp32 pipe active 70 % of the time and issue limited by it; 577 rows of 4 groups,
// 768 to 192: 14 us.  Weights' gradients of 25216 rows, 768 x 192: 215 us, the pipe active 75 %.
#include "linear_grouped.cuh"

namespace vit {

namespace {

constexpr int KS = 16, THREADS = 256, WIDE = 128, SMALL = 64;

// T x 16 pieces of both operands, the summed index across rows, in a ring in shared memory.
template <int T> struct Ring {
  static constexpr int STAGES = T == WIDE ? 4 : 6, LD = T + 4, PIECE = KS * LD, BYTES = STAGES * 2 * PIECE * 4;
};
__device__ __forceinline__ void cp_async_4(uint32_t dst, const void* src, uint32_t src_bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(src_bytes) : "memory");
}
// A thread's copies of a piece.  `base` is the operand's first value of it; valid: the tile's rows (or, ACROSS, columns) that
// exist; left: of the summed index; what does not exist is zero.  ACROSS: the summed index runs over rows of memory.  Else values
// are copied one by one, by a warp 4 rows of 8, which meet all banks.
template <int T, bool ACROSS>
__device__ __forceinline__ void fetch(float* to, const float* base, int64_t ld, int valid, int left) {
  const uint32_t piece = ptx::smem_u32(to);
  if (ACROSS) {
#pragma unroll
    for (int i = 0; i < T / 64; ++i) {
      const int at = (int)threadIdx.x + THREADS * i, t = at % (T / 4) * 4, k = at / (T / 4);
      const bool there = t < valid && k < left;
      ptx::cp_async_16(piece + (uint32_t)(k * Ring<T>::LD + t) * 4, there ? base + (int64_t)k * ld + t : base, there ? 16u : 0u);
    }
  } else {
    const int t0 = (int)threadIdx.x / 8, k0 = (int)threadIdx.x % 8;
#pragma unroll
    for (int i = 0; i < T / 32; ++i)
#pragma unroll
      for (int j = 0; j < KS / 8; ++j) {
        const int t = t0 + 32 * i, k = k0 + 8 * j;
        const bool there = t < valid && k < left;
        cp_async_4(piece + (uint32_t)(k * Ring<T>::LD + t) * 4, there ? base + (int64_t)t * ld + k : base, there ? 4u : 0u);
      }
  }
}

// Where a thread's values of a tile lie.  A warp has 8 by 4 threads, and neighbouring lanes share columns: its reads of 16 bytes
// are then served for half a warp at a time (64 x 64 tiles take 0.86 of the time of rows of 16 threads).
__device__ __forceinline__ int thread_x() { return (threadIdx.x >> 5 & 1) * 8 + (threadIdx.x >> 1 & 7); }
__device__ __forceinline__ int thread_y() { return (threadIdx.x >> 6) * 4 + (threadIdx.x >> 4 & 1) * 2 + (threadIdx.x & 1); }
// A thread's values of a tile: rows 4 ty + r and T / 2 + 4 ty + r, columns alike (T = 128); 4 by 4 of them (T = 64).
template <int T> struct Tile { float2 v[T / 16][T / 32]; };
template <int T> __device__ __forceinline__ int part_at(int i, int t) { return T == WIDE ? (i / 4) * 64 + 4 * t + i % 4 : 4 * t + i; }

// what the next of the summed index needs is read while this one's is multiplied
template <int T>
__device__ __forceinline__ void multiply(Tile<T>& acc, const float (*a)[T + 4], const float (*b)[T + 4]) {
  const int tx = thread_x(), ty = thread_y();
  float4 x[2][T / 64], y[2][T / 64];
  auto read = [&](int k) {
#pragma unroll
    for (int h = 0; h < T / 64; ++h) {
      x[k & 1][h] = *reinterpret_cast<const float4*>(&a[k][64 * h + 4 * ty]);
      y[k & 1][h] = *reinterpret_cast<const float4*>(&b[k][64 * h + 4 * tx]);
    }
  };
  read(0);
#pragma unroll
  for (int k = 0; k < KS; ++k) {
    if (k + 1 < KS) read(k + 1);
#pragma unroll
    for (int i = 0; i < T / 16; ++i) {
      const float4 f = x[k & 1][i / 4];
      const float v = i % 4 == 0 ? f.x : i % 4 == 1 ? f.y : i % 4 == 2 ? f.z : f.w;
#pragma unroll
      for (int h = 0; h < T / 64; ++h) {
        acc.v[i][2 * h] = __ffma2_rn(make_float2(v, v), make_float2(y[k & 1][h].x, y[k & 1][h].y), acc.v[i][2 * h]);
        acc.v[i][2 * h + 1] = __ffma2_rn(make_float2(v, v), make_float2(y[k & 1][h].z, y[k & 1][h].w), acc.v[i][2 * h + 1]);
      }
    }
  }
}

// A tile's sum over `steps` pieces.  get(s, a, b): the copies of piece s; also(a): what else is done with it.
template <int T, typename Get, typename Also>
__device__ __forceinline__ void sum_pieces(Tile<T>& acc, float* ring, int steps, Get get, Also also) {
  using R = Ring<T>;
  __syncthreads();                                     // nobody reads the ring any more
#pragma unroll
  for (int s = 0; s < R::STAGES - 1; ++s) {
    if (s < steps) get(s, ring + s * 2 * R::PIECE, ring + (s * 2 + 1) * R::PIECE);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  int now = 0, next = R::STAGES - 1;
  for (int s = 0; s < steps; ++s) {
    asm volatile("cp.async.wait_group %0;" ::"n"(R::STAGES - 2) : "memory");
    __syncthreads();                                   // all threads' copies have landed, and piece s - 1 has been multiplied
    if (s + R::STAGES - 1 < steps) get(s + R::STAGES - 1, ring + next * 2 * R::PIECE, ring + (next * 2 + 1) * R::PIECE);
    asm volatile("cp.async.commit_group;" ::: "memory");
    const auto a = reinterpret_cast<const float(*)[R::LD]>(ring + now * 2 * R::PIECE), b = a + KS;
    multiply<T>(acc, a, b);
    also(a);
    if (++now == R::STAGES) now = 0;
    if (++next == R::STAGES) next = 0;
  }
}

struct RowsArgs {
  GroupedShape shape;
  int width, sum, epilogue, tiles_n, split;
  bool early;                          // the next kernel may be launched at once
  const float *x, *w, *bias, *residual;
  float *pre, *y;
  int64_t ldx, ldr, ldp, ldy;
  int* dev_status;
};

// four values of a row of the result: bias, GELU, residual or GELU's slope, and out
template <bool BACKWARD>
__device__ __forceinline__ void finish(const RowsArgs& p, int group, int64_t row, int c, float4 sum) {
  float v[4] = {sum.x, sum.y, sum.z, sum.w};
  if (BACKWARD) {
    if (p.pre) {
      const float4 o = *reinterpret_cast<const float4*>(p.pre + row * p.ldp + c);
      const float f[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] *= gelu_slope_f32(f[e]);
    }
  } else {
    if (p.bias) {
      const float4 o = *reinterpret_cast<const float4*>(p.bias + (int64_t)group * p.width + c);
      v[0] += o.x; v[1] += o.y; v[2] += o.z; v[3] += o.w;
    }
    if (p.epilogue == 1) {
      if (p.pre) *reinterpret_cast<float4*>(p.pre + row * p.ldp + c) = make_float4(v[0], v[1], v[2], v[3]);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = gelu_f32(v[e]);
    } else if (p.epilogue == 2) {
      const float4 o = *reinterpret_cast<const float4*>(p.residual + row * p.ldr + c);
      v[0] += o.x; v[1] += o.y; v[2] += o.z; v[3] += o.w;
    }
  }
  *reinterpret_cast<float4*>(p.y + row * p.ldy + c) = make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ float4 read_cluster(const float* here, uint32_t rank) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(ptx::map_to_cta(ptx::smem_u32(here), rank)) : "memory");
  return v;
}

template <int T, bool BACKWARD>
__global__ void __launch_bounds__(THREADS, T == WIDE ? 2 : 4)
grouped_rows_f32_kernel(const RowsArgs p) {
  extern __shared__ __align__(16) float ring[];         // and a block's part of a tile whose sums are shared
  const int lane = threadIdx.x & 31, tx = thread_x(), ty = thread_y();
  const int split = p.split, self = (int)blockIdx.x / split, units = (int)gridDim.x / split;
  const uint32_t rank = blockIdx.x % split;            // in the cluster that shares a tile's sums
  const int share = (p.sum + KS * split - 1) / (KS * split) * KS, k_begin = (int)rank * share, k_end = min(p.sum, k_begin + share);
  ptx::grid_dependency_wait();
  // The next kernel's blocks take the places that are left: where there are some, or come one by one, the first to come would
  // crowd on a few SMs (kernels of their kind one after the other: 2000 rows, 768 x 768, 84 us, 108 if launched at once; 5300
  // rows, 576 x 520, 90 and 121).  Whole sums on all places are better off (4000 rows, 1024 x 4096: 759 us, 855 launched late).
  if (p.early) ptx::grid_launch_dependents();
  if (blockIdx.x == 0 && threadIdx.x < 32) report_bad_groups(p.shape, p.dev_status, lane);
  GroupWalk<TileCount> walk(p.shape, TileCount{T, p.tiles_n}, lane);
  GroupAt at;
  for (int tile = self; walk.find(tile, at); tile += units) {
    const int local = tile - at.before, row0 = at.begin + local / p.tiles_n * T, col0 = local % p.tiles_n * T;
    const int rows = min(T, at.end - row0), cols = min(T, p.width - col0);
    const float* x = p.x + (int64_t)row0 * p.ldx;
    // weights [out][in]: forwards a column of the result is a row of them, backwards a column
    const float* w = p.w + (int64_t)at.group * p.width * p.sum + (BACKWARD ? (int64_t)col0 : (int64_t)col0 * p.sum);
    const int64_t ldw = BACKWARD ? p.width : p.sum;
    Tile<T> acc = {};
    sum_pieces<T>(acc, ring, (k_end - k_begin + KS - 1) / KS,
                  [&](int s, float* a, float* b) {
                    const int k = k_begin + s * KS;
                    fetch<T, false>(a, x + k, p.ldx, rows, k_end - k);
                    fetch<T, BACKWARD>(b, w + (BACKWARD ? (int64_t)k * ldw : (int64_t)k), ldw, cols, k_end - k);
                  },
                  [](const float(*)[T + 4]) {});
    if (split == 1) {
#pragma unroll
      for (int i = 0; i < T / 16; ++i) {
        const int row = row0 + part_at<T>(i, ty);
        if (row >= at.end) continue;
#pragma unroll
        for (int h = 0; h < T / 64; ++h) {
          const int c = col0 + 64 * h + 4 * tx;
          if (c < p.width)
            finish<BACKWARD>(p, at.group, row, c, make_float4(acc.v[i][2 * h].x, acc.v[i][2 * h].y, acc.v[i][2 * h + 1].x, acc.v[i][2 * h + 1].y));
        }
      }
    } else {
      // every block leaves its part where the others can read it, and finishes some of the rows
      __syncthreads();
#pragma unroll
      for (int i = 0; i < T / 16; ++i)
#pragma unroll
        for (int h = 0; h < T / 64; ++h)
          *reinterpret_cast<float4*>(&ring[part_at<T>(i, ty) * (T + 4) + 64 * h + 4 * tx]) =
              make_float4(acc.v[i][2 * h].x, acc.v[i][2 * h].y, acc.v[i][2 * h + 1].x, acc.v[i][2 * h + 1].y);
      ptx::cluster_sync();
      const int first = (int)rank * T / split, count = ((int)rank + 1) * T / split - first;
      for (int i = threadIdx.x; i < count * (T / 4); i += THREADS) {
        const int r = first + i / (T / 4), c = i % (T / 4) * 4;
        if (row0 + r >= at.end || col0 + c >= p.width) continue;
        const float* from = &ring[r * (T + 4) + c];
        float4 sum = read_cluster(from, 0);
        for (int k = 1; k < split; ++k) {
          const float4 v = read_cluster(from, (uint32_t)k);
          sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
        }
        finish<BACKWARD>(p, at.group, row0 + r, col0 + c, sum);
      }
      ptx::cluster_sync();                              // nobody reads there any more
    }
  }
}

struct DwArgs {
  GroupedShape shape;
  int in, out, tiles_in, tiles, least, cuts;
  const float *x, *dout;
  int64_t ldx, lddout;
  float *dw, *dbias, *part, *part_bias;
  int* table;
  int* dev_status;
};

__global__ void __launch_bounds__(THREADS, 2)
grouped_dw_f32_kernel(const DwArgs p) {
  constexpr int T = WIDE;
  extern __shared__ __align__(16) float ring[];
  const int lane = threadIdx.x & 31, tx = thread_x(), ty = thread_y();
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  if (blockIdx.x == 0 && threadIdx.x < 32) report_bad_groups(p.shape, p.dev_status, lane);
  const Share share = find_share(p.shape, p.tiles, (int)gridDim.x, (int)blockIdx.x, p.least, p.cuts, reinterpret_cast<int*>(ring), p.table);
  __syncthreads();
  PartWalk work(p.shape, p.tiles, lane, share, (int)blockIdx.x, (int)gridDim.x);
  Part part;
  while (work.next(part)) {
    const int n0 = part.tile / p.tiles_in * T, k0 = part.tile % p.tiles_in * T;
    const int64_t r0 = part.begin + (int64_t)part.from * DW_ROWS;
    const int rows = (int)(min((int64_t)part.end, part.begin + (int64_t)part.to * DW_ROWS) - r0);      // none for an empty group
    const float *d = p.dout + r0 * p.lddout + n0, *x = p.x + r0 * p.ldx + k0;
    Tile<T> acc = {};
    float bias = 0.f;
    const bool sums = p.dbias && k0 == 0 && threadIdx.x < T;
    sum_pieces<T>(acc, ring, (rows + KS - 1) / KS,
                  [&](int s, float* a, float* b) {
                    const int r = s * KS;
                    fetch<T, true>(a, d + (int64_t)r * p.lddout, p.lddout, p.out - n0, rows - r);
                    fetch<T, true>(b, x + (int64_t)r * p.ldx, p.ldx, p.in - k0, rows - r);
                  },
                  [&](const float(*a)[T + 4]) {
                    if (!sums) return;
                    float some = 0.f;
#pragma unroll
                    for (int k = 0; k < KS; ++k) some += a[k][threadIdx.x];
                    bias += some;
                  });
    const bool whole = part.whole();
    const int64_t slot = (int64_t)blockIdx.x * 2 + part.slot();
#pragma unroll
    for (int i = 0; i < T / 16; ++i) {
      const int n = part_at<T>(i, ty);
#pragma unroll
      for (int h = 0; h < T / 64; ++h) {
        const int k = 64 * h + 4 * tx;
        if (n0 + n >= p.out || k0 + k >= p.in) continue;
        float* to = whole ? p.dw + ((int64_t)part.group * p.out + n0 + n) * p.in + k0 + k : p.part + (slot * T + n) * T + k;
        *reinterpret_cast<float4*>(to) = make_float4(acc.v[i][2 * h].x, acc.v[i][2 * h].y, acc.v[i][2 * h + 1].x, acc.v[i][2 * h + 1].y);
      }
    }
    if (sums && n0 + (int)threadIdx.x < p.out) *(whole ? p.dbias + (int64_t)part.group * p.out + n0 + threadIdx.x : p.part_bias + slot * T + threadIdx.x) = bias;
  }
}

template <int T, typename Kernel, typename Args>
cudaError_t launch_after(PerDeviceFlag& configured, Kernel kernel, int grid, const Args& args, cudaStream_t s, int cluster = 1) {
  if (cudaError_t e = ensure_dynamic_smem(configured, kernel, Ring<T>::BYTES)) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.dynamicSmemBytes = Ring<T>::BYTES;
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(THREADS);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, args);
}

}  // namespace

namespace {
__global__ void check_groups_kernel(const GroupedShape shape, int* dev_status) { report_bad_groups(shape, dev_status, (int)threadIdx.x); }
}  // namespace
cudaError_t launch_check_groups(const GroupedCall& c, cudaStream_t s) {
  check_groups_kernel<<<1, 32, 0, s>>>(c.shape, c.dev_status);
  return cudaGetLastError();
}

// Tiles at a time: two or four blocks to an SM; clusters do not find all places (71 of four and 33 of eight blocks of 128 x 128, 142
// and 71 of 64 x 64, by the occupancy calculator).
static int units_of(bool wide, int split, int sms) {
  const int all = sms * (wide ? 2 : 4) / split;
  return split < 4 ? all : split == 8 && wide ? all * 9 / 10 : all * 24 / 25;
}
// About what the products of rows take, in cycles.  A round of blocks takes, for 16 of the sum, `piece` with one to four of them
// on an SM, and what starts and ends a tile, more so between rounds.  Measured with either tile and 1 to 8 blocks to a sum at 23
// shapes: the choice is the best or within 7 % of it (577 rows, 768 x 768: 28 us with 128 x 128 tiles in eighths, 33 with 64 x 64;
// 197 rows, 768 x 192: 9 us with 64 x 64 in eighths, 17 with 128 x 128; 8224 rows, 1280 x 1280: 606 us in halves, 652 whole).
static double cycles_of(bool wide, int split, const GroupedShape& shape, int width, int sum, int sms) {
  constexpr double PIECE[2][4] = {{1085., 1900., 2900., 3900.}, {2950., 5330., 0., 0.}};
  const int t = wide ? WIDE : SMALL, places = wide ? 2 : 4;
  // groups end somewhere in a tile, and those with rows have one
  const int64_t some = shape.groups < shape.rows ? shape.groups : shape.rows, row_tiles = (2 * (int64_t)shape.rows + some * t) / (2 * t);
  const int64_t down = some == 1 ? (shape.rows + t - 1) / t : row_tiles > some ? row_tiles : some, tiles = down * ((width + t - 1) / t);
  const int64_t units = units_of(wide, split, sms), rounds = tiles / units, last = tiles - rounds * units;
  const double pieces = (sum + KS * split - 1) / (KS * split);
  const double end = wide ? (split == 1 ? 9000. : 11500.) : 5500. + 600. * split;
  const double between = !wide ? end : split == 1 ? 12000. : split == 2 ? 15000. : split == 4 ? 28000. : 50000.;
  double cycles = rounds * (pieces * PIECE[wide][places - 1] + between);
  if (last == 0) return cycles - (rounds > 0 ? between - end : 0.);
  // clusters do not spread evenly over the SMs by themselves
  const int64_t blocks = last * split * (rounds == 0 && split > 1 ? 23 : 20) / 20, on_sm = (blocks + sms - 1) / sms;
  return cycles + pieces * PIECE[wide][(on_sm < places ? on_sm : places) - 1] + end;
}
cudaError_t launch_grouped_rows_f32(const GroupedCall& c, cudaStream_t s) {
  RowsArgs p{c.shape, c.backward ? c.in : c.out_features, c.backward ? c.out_features : c.in, c.epilogue, 0, 1, false, static_cast<const float*>(c.x),
             static_cast<const float*>(c.w), c.bias, static_cast<const float*>(c.residual), static_cast<float*>(c.pre), static_cast<float*>(c.y),
             c.ldx, c.ldr, c.ldp, c.ldy, c.dev_status};
  const int sms = current_device_sm_count();
  if (sms < 1) return cudaErrorInvalidDevice;
  bool wide = false;
  double best = 0.;
  for (int t = SMALL; t <= WIDE; t += SMALL)
    for (int split = 1; split <= 8 && (split == 1 || p.sum >= 2 * KS * split); split *= 2) {
      const double cycles = cycles_of(t == WIDE, split, c.shape, p.width, p.sum, sms);
      if (best > 0. && cycles >= best) continue;
      best = cycles;
      wide = t == WIDE;
      p.split = split;
    }
  const int t = wide ? WIDE : SMALL, units = units_of(wide, p.split, sms);
  p.tiles_n = (p.width + t - 1) / t;
  const int64_t most = ((int64_t)c.shape.rows / t + c.shape.groups) * p.tiles_n;      // tiles
  p.early = wide && p.split == 1 && most >= units;
  const int grid = (int)(most < units ? most : units) * p.split;
  static PerDeviceFlag configured[4];
  if (c.backward)
    return wide ? launch_after<WIDE>(configured[0], grouped_rows_f32_kernel<WIDE, true>, grid, p, s, p.split)
                : launch_after<SMALL>(configured[1], grouped_rows_f32_kernel<SMALL, true>, grid, p, s, p.split);
  return wide ? launch_after<WIDE>(configured[2], grouped_rows_f32_kernel<WIDE, false>, grid, p, s, p.split)
              : launch_after<SMALL>(configured[3], grouped_rows_f32_kernel<SMALL, false>, grid, p, s, p.split);
}

cudaError_t launch_grouped_dw_f32(const GroupedCall& c, cudaStream_t s) {
  const GroupedDw plan = grouped_dw_plan(c, false);
  const DwArgs p{c.shape, c.in, c.out_features, plan.tiles_in, plan.tiles, plan.least, plan.cuts, static_cast<const float*>(c.x), static_cast<const float*>(c.dout),
                 c.ldx, c.lddout, static_cast<float*>(c.dw), c.dbias, plan.part, plan.part_bias, plan.table, c.dev_status};
  static PerDeviceFlag configured;
  return launch_after<WIDE>(configured, grouped_dw_f32_kernel, plan.blocks, p, s);
}

}  // namespace vit
