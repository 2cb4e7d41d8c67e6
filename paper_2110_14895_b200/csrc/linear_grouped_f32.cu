// Linear layers by group in the fp32 mode, on the fp32 pipes: rows times their group's weights forwards and backwards, and the
// weights' gradients.  Tiles of the result in registers, 16 of the summed index at a time through shared memory, the next 16
// under way while these are multiplied; two products to an instruction (packed fp32).
// 128 x 128 tiles where there are enough of them to go round, else 64 x 64, whose sums are shared by a cluster of blocks and
// joined in its shared memory as long as blocks are left over.
#include "linear_grouped.cuh"

namespace vit {

namespace {

constexpr int KS = 16, THREADS = 256, WIDE = 128, SMALL = 64;

// A T x 16 piece of an operand in registers: float4 i of a thread.  `base` is the operand's first value of the tile; valid: its
// rows (or, ACROSS, columns) that exist; left: of the summed index.  ACROSS: the summed index runs over rows of memory.
template <int T, bool ACROSS>
__device__ __forceinline__ void fetch(float4 (&v)[T / 64], const float* base, int64_t ld, int valid, int left) {
#pragma unroll
  for (int i = 0; i < T / 64; ++i) {
    const int at = (int)threadIdx.x + THREADS * i;
    const int t = ACROSS ? at % (T / 4) * 4 : at / 4, k = ACROSS ? at / (T / 4) : at % 4 * 4;
    v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (t < valid && k < left) v[i] = *reinterpret_cast<const float4*>(base + (ACROSS ? k * ld + t : t * ld + k));
  }
}
template <int T, bool ACROSS>
__device__ __forceinline__ void keep(const float4 (&v)[T / 64], float (*to)[T + 4]) {
#pragma unroll
  for (int i = 0; i < T / 64; ++i) {
    const int at = (int)threadIdx.x + THREADS * i;
    if (ACROSS) *reinterpret_cast<float4*>(&to[at / (T / 4)][at % (T / 4) * 4]) = v[i];
    else {
      const int t = at / 4, k = at % 4 * 4;
      to[k][t] = v[i].x;
      to[k + 1][t] = v[i].y;
      to[k + 2][t] = v[i].z;
      to[k + 3][t] = v[i].w;
    }
  }
}

// A thread's values of a tile: rows 4 ty + r and T / 2 + 4 ty + r, columns alike (T = 128); 4 by 4 of them (T = 64).
template <int T> struct Tile { float2 v[T / 16][T / 32]; };
template <int T> __device__ __forceinline__ int part_at(int i, int t) { return T == WIDE ? (i / 4) * 64 + 4 * t + i % 4 : 4 * t + i; }

template <int T>
__device__ __forceinline__ void multiply(Tile<T>& acc, const float (*a)[T + 4], const float (*b)[T + 4]) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
  for (int k = 0; k < KS; ++k) {
    float x[T / 16];
    float2 y[T / 32];
#pragma unroll
    for (int h = 0; h < T / 64; ++h) {
      const float4 f = *reinterpret_cast<const float4*>(&a[k][64 * h + 4 * ty]), g = *reinterpret_cast<const float4*>(&b[k][64 * h + 4 * tx]);
      x[4 * h] = f.x; x[4 * h + 1] = f.y; x[4 * h + 2] = f.z; x[4 * h + 3] = f.w;
      y[2 * h] = make_float2(g.x, g.y); y[2 * h + 1] = make_float2(g.z, g.w);
    }
#pragma unroll
    for (int i = 0; i < T / 16; ++i)
#pragma unroll
      for (int j = 0; j < T / 32; ++j) acc.v[i][j] = __ffma2_rn(make_float2(x[i], x[i]), y[j], acc.v[i][j]);
  }
}

struct RowsArgs {
  GroupedShape shape;
  int width, sum, epilogue, tiles_n, split;
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

template <int T> union Stages {
  struct { float a[2][KS][T + 4], b[2][KS][T + 4]; } s;
  float sums[T == SMALL ? T : 1][T + 4];               // a block's part of a tile whose sums are shared
};

template <int T, bool BACKWARD>
__global__ void __launch_bounds__(THREADS, T == WIDE ? 2 : 4)
grouped_rows_f32_kernel(const RowsArgs p) {
  __shared__ __align__(16) Stages<T> mem;
  auto &a = mem.s.a, &b = mem.s.b;
  const int lane = threadIdx.x & 31, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int split = T == SMALL ? p.split : 1, self = (int)blockIdx.x / split, units = (int)gridDim.x / split;
  const uint32_t rank = blockIdx.x % split;            // in the cluster that shares a tile's sums
  const int share = (p.sum + KS * split - 1) / (KS * split) * KS, k_begin = (int)rank * share, k_end = min(p.sum, k_begin + share);
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
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
    float4 va[T / 64], vb[T / 64];
    auto get = [&](int k) {
      fetch<T, false>(va, x + k, p.ldx, rows, k_end - k);
      fetch<T, BACKWARD>(vb, w + (BACKWARD ? (int64_t)k * ldw : (int64_t)k), ldw, cols, k_end - k);
    };
    get(k_begin);
    __syncthreads();                                    // the tile before has been multiplied
    keep<T, false>(va, a[0]);
    keep<T, BACKWARD>(vb, b[0]);
    __syncthreads();
    int now = 0;
    for (int k = k_begin; k < k_end; k += KS, now ^= 1) {
      const bool more = k + KS < k_end;
      if (more) get(k + KS);
      multiply<T>(acc, a[now], b[now]);
      if (more) {
        keep<T, false>(va, a[now ^ 1]);
        keep<T, BACKWARD>(vb, b[now ^ 1]);
      }
      __syncthreads();
    }
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
    } else if (T == SMALL) {
      // every block leaves its part where the others can read it, and finishes some of the rows
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(&mem.sums[(4 * ty + i) % (T == SMALL ? T : 1)][4 * tx]) = make_float4(acc.v[i][0].x, acc.v[i][0].y, acc.v[i][1].x, acc.v[i][1].y);
      ptx::cluster_sync();
      for (int i = threadIdx.x; i < T / split * 16; i += THREADS) {
        const int r = (int)rank * (T / split) + i / 16, c = i % 16 * 4;
        if (row0 + r >= at.end || col0 + c >= p.width) continue;
        const float* from = &mem.sums[r % (T == SMALL ? T : 1)][c];
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
  __shared__ __align__(16) float a[2][KS][T + 4], b[2][KS][T + 4];
  const int lane = threadIdx.x & 31, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  if (blockIdx.x == 0 && threadIdx.x < 32) report_bad_groups(p.shape, p.dev_status, lane);
  const Share share = find_share(p.shape, p.tiles, (int)gridDim.x, (int)blockIdx.x, p.least, p.cuts, reinterpret_cast<int*>(&a[0][0][0]), p.table);
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
    float4 va[2], vb[2];
    fetch<T, true>(va, d, p.lddout, p.out - n0, rows);
    fetch<T, true>(vb, x, p.ldx, p.in - k0, rows);
    __syncthreads();
    keep<T, true>(va, a[0]);
    keep<T, true>(vb, b[0]);
    __syncthreads();
    int now = 0;
    for (int r = 0; r < rows; r += KS, now ^= 1) {
      const bool more = r + KS < rows;
      if (more) {
        fetch<T, true>(va, d + (int64_t)(r + KS) * p.lddout, p.lddout, p.out - n0, rows - r - KS);
        fetch<T, true>(vb, x + (int64_t)(r + KS) * p.ldx, p.ldx, p.in - k0, rows - r - KS);
      }
      multiply<T>(acc, a[now], b[now]);
      if (sums) {
        float some = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) some += a[now][k][threadIdx.x];
        bias += some;
      }
      if (more) {
        keep<T, true>(va, a[now ^ 1]);
        keep<T, true>(vb, b[now ^ 1]);
      }
      __syncthreads();
    }
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

template <typename Kernel, typename Args>
cudaError_t launch_after(Kernel kernel, int grid, const Args& args, cudaStream_t s, int cluster = 1) {
  cudaLaunchConfig_t cfg = {};
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

cudaError_t launch_grouped_rows_f32(const GroupedCall& c, cudaStream_t s) {
  RowsArgs p{c.shape, c.backward ? c.in : c.out_features, c.backward ? c.out_features : c.in, c.epilogue, 0, 1, static_cast<const float*>(c.x),
             static_cast<const float*>(c.w), c.bias, static_cast<const float*>(c.residual), static_cast<float*>(c.pre), static_cast<float*>(c.y),
             c.ldx, c.ldr, c.ldp, c.ldy, c.dev_status};
  const int sms = current_device_sm_count();
  auto tiles = [&](int t) { return ((int64_t)c.shape.rows / t + c.shape.groups) * ((p.width + t - 1) / t); };
  const bool wide = tiles(WIDE) >= 2 * (int64_t)sms;
  const int t = wide ? WIDE : SMALL;
  p.tiles_n = (p.width + t - 1) / t;
  // at least 64 of a sum to a block, and no more blocks than run at once
  if (!wide)
    while (p.split < 8 && tiles(t) * p.split * 2 <= (int64_t)sms * 2 && p.sum >= 128 * p.split) p.split *= 2;
  const int64_t most = (int64_t)sms * (wide ? 2 : 4);
  const int grid = (int)(tiles(t) < most ? tiles(t) : most) * p.split;
  if (c.backward) return wide ? launch_after(grouped_rows_f32_kernel<WIDE, true>, grid, p, s) : launch_after(grouped_rows_f32_kernel<SMALL, true>, grid, p, s, p.split);
  return wide ? launch_after(grouped_rows_f32_kernel<WIDE, false>, grid, p, s) : launch_after(grouped_rows_f32_kernel<SMALL, false>, grid, p, s, p.split);
}

cudaError_t launch_grouped_dw_f32(const GroupedCall& c, cudaStream_t s) {
  const GroupedDw plan = grouped_dw_plan(c, false);
  const DwArgs p{c.shape, c.in, c.out_features, plan.tiles_in, plan.tiles, plan.least, plan.cuts, static_cast<const float*>(c.x), static_cast<const float*>(c.dout),
                 c.ldx, c.lddout, static_cast<float*>(c.dw), c.dbias, plan.part, plan.part_bias, plan.table, c.dev_status};
  return launch_after(grouped_dw_f32_kernel, plan.blocks, p, s);
}

}  // namespace vit
