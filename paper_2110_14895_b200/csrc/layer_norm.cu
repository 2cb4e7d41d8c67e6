// Layer norm of every row with the statistics that its gradients need, and the gradients.
//
//   forward   y = (x - m) r g + b,  m = mean(x),  r = 1 / sqrt(mean((x - m)^2) + eps)
//   backward  z = (x - m) r,  w = g dy:   dx = r (w - mean(w) - z mean(w z)) + dres,  dg = sum dy z,  db = sum dy
//
// Both are bound by memory: a row is read and written once.  One warp owns a row (four warps beyond 2048 columns) and a
// lane the same columns of every row, eight at a time, so that the sums over rows for dg and db stay in registers.
#include "vit_internal.h"
#include "sm100_ptx.cuh"

namespace vit {

namespace {

constexpr int CH = 8;                          // columns of a lane's piece: one 16-byte load in bf16, two in fp32
constexpr int NARROW = 2048;                   // columns that one warp holds

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float2 twice(float v) { return make_float2(v, v); }

// a piece as it lies in memory
template <typename T> struct Raw;
template <> struct Raw<bf16> { uint4 u; };
template <> struct Raw<float> { float4 a, b; };

__device__ __forceinline__ Raw<bf16> load_raw(const bf16* p) { return {*reinterpret_cast<const uint4*>(p)}; }
__device__ __forceinline__ Raw<float> load_raw(const float* p) { return {reinterpret_cast<const float4*>(p)[0], reinterpret_cast<const float4*>(p)[1]}; }
// bf16 -> fp32 is a shift (low half) or a mask (high half) of the 32-bit word
__device__ __forceinline__ void open(const Raw<bf16>& r, float2 (&v)[4]) {
  const uint32_t w[4] = {r.u.x, r.u.y, r.u.z, r.u.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = make_float2(__uint_as_float(w[e] << 16), __uint_as_float(w[e] & 0xffff0000u));
}
__device__ __forceinline__ void open(const Raw<float>& r, float2 (&v)[4]) {
  v[0] = make_float2(r.a.x, r.a.y); v[1] = make_float2(r.a.z, r.a.w);
  v[2] = make_float2(r.b.x, r.b.y); v[3] = make_float2(r.b.z, r.b.w);
}
__device__ __forceinline__ void store_piece(bf16* p, const float2 (&v)[4]) {
  uint4 o;
  __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&o);
#pragma unroll
  for (int e = 0; e < 4; ++e) h[e] = __floats2bfloat162_rn(v[e].x, v[e].y);
  *reinterpret_cast<uint4*>(p) = o;
}
__device__ __forceinline__ void store_piece(float* p, const float2 (&v)[4]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
}

// One or two sums (N) over a row's warps: one, or the four of a group of 128 threads, which meet at a barrier of their own.  Two slots,
// used in turn, keep a late reader from the next sum's writers.
template <int WPR, int N>
__device__ __forceinline__ float2 row_sums(float2 v, float2 (*slots)[4], int& turn) {
  v.x = warp_sum(v.x);
  if (N == 2) v.y = warp_sum(v.y);
  if (WPR == 1) return v;
  const int warp = threadIdx.x >> 5, group = warp / WPR;
  float2* s = slots[2 * group + turn];
  turn ^= 1;
  if ((threadIdx.x & 31) == 0) s[warp % WPR] = v;
  asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(WPR * 32) : "memory");
  float2 t = s[0];
#pragma unroll
  for (int i = 1; i < WPR; ++i) t = make_float2(t.x + s[i].x, t.y + s[i].y);
  return t;
}

struct ForwardArgs {
  const void* x; int64_t ldx;
  const float *gain, *shift;
  float eps;
  void* y; int64_t ldy;
  float2* stats;
  int rows, cols;
};

// R rows at a time share the loads of gain and shift, which are four times a bf16 row's own: 32896 rows of 1280 columns take 36
// us one at a time (whatever the number of warps, with or without rows fetched ahead), 31 with two, 32 with three or four.
constexpr int FORWARD_THREADS = 128;
template <typename T, int NCH, int WPR, int R>            // R: 1 or 2
__global__ void __launch_bounds__(FORWARD_THREADS)
layer_norm_kernel(const ForwardArgs p) {
  __shared__ float2 slots[2][4];
  const int warp = threadIdx.x >> 5, at = (warp % WPR) * 32 + (threadIdx.x & 31);
  const int64_t row = ((int64_t)blockIdx.x * (FORWARD_THREADS / 32 / WPR) + warp / WPR) * R;
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  if (row >= p.rows) return;                    // all warps of a row together
  const T* x = static_cast<const T*>(p.x) + row * p.ldx;
  Raw<T> raw[R][NCH];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < NCH; ++i) {             // all loads in flight before the first use
      const int c = (at + 32 * WPR * i) * CH;
      if (c < p.cols && row + r < p.rows) raw[r][i] = load_raw(x + r * p.ldx + c);
    }
  int turn = 0;
  float mean[R], rstd[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < NCH; ++i)
      if ((at + 32 * WPR * i) * CH < p.cols) {
        float2 v[4];
        open(raw[r][i], v);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum = __fadd2_rn(sum, v[e]);
      }
    mean[r] = sum.x + sum.y;
  }
  float2 both = row_sums<WPR, R>(make_float2(mean[0], mean[R - 1]), slots, turn);
  mean[0] = both.x / (float)p.cols;
  if (R == 2) mean[R - 1] = both.y / (float)p.cols;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < NCH; ++i)
      if ((at + 32 * WPR * i) * CH < p.cols) {
        float2 v[4];
        open(raw[r][i], v);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] = __fadd2_rn(v[e], twice(-mean[r]));
          sum = __ffma2_rn(v[e], v[e], sum);
        }
      }
    rstd[r] = sum.x + sum.y;
  }
  both = row_sums<WPR, R>(make_float2(rstd[0], rstd[R - 1]), slots, turn);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    rstd[r] = 1.0f / sqrtf((r == 0 ? both.x : both.y) / (float)p.cols + p.eps);
    if (at == 0 && p.stats && row + r < p.rows) p.stats[row + r] = make_float2(mean[r], rstd[r]);
  }
  T* y = static_cast<T*>(p.y) + row * p.ldy;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = (at + 32 * WPR * i) * CH;
    if (c < p.cols) {
      float2 g[4], b[4];
      open(load_raw(p.gain + c), g);
      open(load_raw(p.shift + c), b);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float2 v[4];
        open(raw[r][i], v);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __ffma2_rn(__fmul2_rn(__fadd2_rn(v[e], twice(-mean[r])), twice(rstd[r])), g[e], b[e]);
        if (row + r < p.rows) store_piece(y + r * p.ldy + c, v);
      }
    }
  }
}

struct BackwardArgs {
  const void* x; int64_t ldx;
  const float* gain;
  const float2* stats;
  const void* dy; int64_t lddy;
  const void* dres; int64_t lddres;
  void* dx; int64_t lddx;
  float* partial;                               // [blocks][2][cols]
  int rows, cols, stages;
};

// A warp's rows come through a ring in shared memory, `stages` rows ahead.  A lane copies what it will read itself, so that
// no two threads have to meet over it, and the registers are left to the sums of dg and db.
template <typename T, int NCH, int WPR, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, 1)
layer_norm_backward_kernel(const BackwardArgs p) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float2 slots[2 * WARPS / WPR][4];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, at = (warp % WPR) * 32 + lane;
  const int64_t step = (int64_t)gridDim.x * (WARPS / WPR);
  float* gain = reinterpret_cast<float*>(smem);                            // [cols]
  const int arrays = p.dres ? 3 : 2;
  const uint32_t row_bytes = (uint32_t)p.cols * sizeof(T), stage_bytes = row_bytes * arrays;
  uint8_t* ring = smem + (size_t)p.cols * 4 + (size_t)(warp / WPR) * p.stages * stage_bytes;
  auto fetch = [&](int64_t row, int stage) {
    if (row < p.rows) {
      const uint32_t to = ptx::smem_u32(ring + stage * stage_bytes);
      const T* x = static_cast<const T*>(p.x) + row * p.ldx;
      const T* dy = static_cast<const T*>(p.dy) + row * p.lddy;
      const T* dres = static_cast<const T*>(p.dres) + row * p.lddres;
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int c = (at + 32 * WPR * i) * CH;
        if (c < p.cols) {
#pragma unroll
          for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
            const int e = c + h * (16 / (int)sizeof(T));
            const uint32_t off = to + (uint32_t)e * sizeof(T);
            ptx::cp_async_16(off, x + e, 16);
            ptx::cp_async_16(off + row_bytes, dy + e, 16);
            if (p.dres) ptx::cp_async_16(off + 2 * row_bytes, dres + e, 16);
          }
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");      // an empty group where there is no row
  };
  float2 dg[NCH][4], db[NCH][4];
#pragma unroll
  for (int i = 0; i < NCH; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) dg[i][e] = db[i][e] = make_float2(0.f, 0.f);
  const float inv = 1.0f / (float)p.cols;
  int64_t row = (int64_t)blockIdx.x * (WARPS / WPR) + warp / WPR;
  // (the next kernel launched at once would crowd here: 3152 rows of 768, both kernels, 8.7 us for 7.9)
  ptx::grid_dependency_wait();
  for (int s = 0; s < p.stages - 1; ++s) fetch(row + s * step, s);
  for (int i = 4 * threadIdx.x; i < p.cols; i += WARPS * 128) *reinterpret_cast<float4*>(gain + i) = *reinterpret_cast<const float4*>(p.gain + i);
  __syncthreads();
  float2 st = row < p.rows ? p.stats[row] : make_float2(0.f, 0.f);
  int stage = 0, turn = 0;
  for (; row < p.rows; row += step) {
    int ahead = stage + p.stages - 1;
    if (ahead >= p.stages) ahead -= p.stages;
    fetch(row + (p.stages - 1) * step, ahead);
    const float2 st_next = row + step < p.rows ? p.stats[row + step] : st;
    if (p.stages == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else asm volatile("cp.async.wait_group 1;" ::: "memory");
    const T* xs = reinterpret_cast<const T*>(ring + stage * stage_bytes);
    const T* ds = reinterpret_cast<const T*>(ring + stage * stage_bytes + row_bytes);
    const float2 nm = twice(-st.x), r = twice(st.y);
    float2 s1 = make_float2(0.f, 0.f), s2 = s1;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = (at + 32 * WPR * i) * CH;
      if (c < p.cols) {
        float2 z[4], d[4], g[4];
        open(load_raw(xs + c), z);
        open(load_raw(ds + c), d);
        open(load_raw(gain + c), g);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          z[e] = __fmul2_rn(__fadd2_rn(z[e], nm), r);
          dg[i][e] = __ffma2_rn(d[e], z[e], dg[i][e]);
          db[i][e] = __fadd2_rn(d[e], db[i][e]);
          d[e] = __fmul2_rn(d[e], g[e]);
          s1 = __fadd2_rn(s1, d[e]);
          s2 = __ffma2_rn(d[e], z[e], s2);
        }
      }
    }
    const float2 sums = row_sums<WPR, 2>(make_float2(s1.x + s1.y, s2.x + s2.y), slots, turn);
    const float2 c1 = twice(-sums.x * inv), c2 = twice(-sums.y * inv);
    T* dx = static_cast<T*>(p.dx) + row * p.lddx;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = (at + 32 * WPR * i) * CH;
      if (c < p.cols) {
        float2 z[4], d[4], g[4];
        open(load_raw(xs + c), z);
        open(load_raw(ds + c), d);
        open(load_raw(gain + c), g);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          z[e] = __fmul2_rn(__fadd2_rn(z[e], nm), r);
          d[e] = __fmul2_rn(r, __ffma2_rn(z[e], c2, __ffma2_rn(d[e], g[e], c1)));
        }
        if (p.dres) {
          open(load_raw(ds + p.cols + c), g);
#pragma unroll
          for (int e = 0; e < 4; ++e) d[e] = __fadd2_rn(d[e], g[e]);
        }
        store_piece(dx + c, d);
      }
    }
    st = st_next;
    if (++stage == p.stages) stage = 0;
  }
  // this block's share of dg and db: its rows' warps are added in a fixed order
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  float* share = reinterpret_cast<float*>(smem + (size_t)p.cols * 4);      // [WARPS / WPR][2][cols]
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = (at + 32 * WPR * i) * CH;
    if (c < p.cols) {
      store_piece(share + (size_t)(warp / WPR) * 2 * p.cols + c, dg[i]);
      store_piece(share + (size_t)(warp / WPR) * 2 * p.cols + p.cols + c, db[i]);
    }
  }
  __syncthreads();
  for (int i = 4 * threadIdx.x; i < 2 * p.cols; i += WARPS * 128) {
    float4 sum = *reinterpret_cast<const float4*>(share + i);
#pragma unroll
    for (int w = 1; w < WARPS / WPR; ++w) {
      const float4 v = *reinterpret_cast<const float4*>(share + (size_t)w * 2 * p.cols + i);
      sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
    }
    *reinterpret_cast<float4*>(p.partial + (int64_t)blockIdx.x * 2 * p.cols + i) = sum;
  }
}

// dgain[c], dshift[c] = sum of the blocks' shares, in a fixed order: 8 columns (a sector) to a block, 32 threads to a column, all
// loads of a thread in flight together (one after the other they took 8 us for 148 shares of 1024 columns, now 4)
constexpr int COLUMN_THREADS = 256;
__global__ void __launch_bounds__(COLUMN_THREADS)
column_grad_kernel(const float* __restrict__ partial, int blocks, int cols, float* __restrict__ dgain, float* __restrict__ dshift) {
  __shared__ float sums[COLUMN_THREADS / 32][8];
  const int column = threadIdx.x & 7, part = threadIdx.x >> 3, i = blockIdx.x * 8 + column;
  ptx::grid_dependency_wait();                           // the shares are written by the kernel before this one
  ptx::grid_launch_dependents();
  constexpr int N = LAYER_NORM_MAX_BLOCKS / (COLUMN_THREADS / 8);
  float v[N], sum = 0.f;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int b = part + k * (COLUMN_THREADS / 8);
    v[k] = b < blocks ? partial[(int64_t)b * 2 * cols + i] : 0.f;
  }
#pragma unroll
  for (int k = 0; k < N; ++k) sum += v[k];
  sum += __shfl_xor_sync(0xffffffffu, sum, 8);
  sum += __shfl_xor_sync(0xffffffffu, sum, 16);
  if ((threadIdx.x & 31) < 8) sums[threadIdx.x >> 5][column] = sum;
  __syncthreads();
  if (threadIdx.x < 8) {
    sum = 0.f;
#pragma unroll
    for (int b = 0; b < COLUMN_THREADS / 32; ++b) sum += sums[b][column];
    (i < cols ? dgain : dshift)[i < cols ? i : i - cols] = sum;
  }
}

template <typename Kernel, typename... Args>
cudaError_t launch_after(Kernel kernel, int grid, int threads, size_t smem, cudaStream_t s, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <typename T, int NCH, int WPR, int R>
cudaError_t launch_forward(const ForwardArgs& a, cudaStream_t s) {
  constexpr int ROWS = FORWARD_THREADS / 32 / WPR * R;
  return launch_after(layer_norm_kernel<T, NCH, WPR, R>, (int)(((int64_t)a.rows + ROWS - 1) / ROWS), FORWARD_THREADS, 0, s, a);
}
// two rows to a warp where there are rows enough for 16 warps an SM, and registers for them
template <typename T, int NCH>
cudaError_t launch_narrow(const ForwardArgs& a, cudaStream_t s) {
  if constexpr (NCH * sizeof(T) <= 12)
    if (a.rows >= 32 * current_device_sm_count()) return launch_forward<T, NCH, 1, 2>(a, s);
  return launch_forward<T, NCH, 1, 1>(a, s);
}
template <typename T>
cudaError_t dispatch_forward(const ForwardArgs& a, cudaStream_t s) {
  const int per_warp = (a.cols + 32 * CH - 1) / (32 * CH);
  if (a.cols <= NARROW) switch (per_warp) {
    case 1: return launch_narrow<T, 1>(a, s);
    case 2: return launch_narrow<T, 2>(a, s);
    case 3: return launch_narrow<T, 3>(a, s);
    case 4: return launch_narrow<T, 4>(a, s);
    case 5: return launch_narrow<T, 5>(a, s);
    case 6: return launch_narrow<T, 6>(a, s);
    default: return launch_narrow<T, 8>(a, s);
  }
  if (per_warp <= 16) return launch_forward<T, 4, 4, sizeof(T) == 2 ? 2 : 1>(a, s);
  return launch_forward<T, 8, 4, 1>(a, s);
}

constexpr size_t SHARED_BYTES = 225 * 1024;

template <typename T, int NCH, int WPR, int WARPS>
cudaError_t launch_backward(BackwardArgs a, cudaStream_t s, int* blocks) {
  static PerDeviceFlag done;
  auto kernel = layer_norm_backward_kernel<T, NCH, WPR, WARPS>;
  if (cudaError_t e = ensure_dynamic_smem(done, kernel, (int)SHARED_BYTES)) return e;
  const size_t stage = (size_t)(WARPS / WPR) * a.cols * sizeof(T) * (a.dres ? 3 : 2);
  a.stages = 3 * stage + (size_t)a.cols * sizeof(float) <= SHARED_BYTES ? 3 : 2;
  size_t smem = a.stages * stage;
  const size_t share = (size_t)(WARPS / WPR) * 2 * a.cols * sizeof(float);
  if (smem < share) smem = share;
  smem += (size_t)a.cols * sizeof(float);
  const int64_t want = ((int64_t)a.rows + WARPS / WPR - 1) / (WARPS / WPR);
  const int sms = current_device_sm_count();
  *blocks = (int)(want < sms ? want : sms);
  if (*blocks > LAYER_NORM_MAX_BLOCKS) *blocks = LAYER_NORM_MAX_BLOCKS;
  return launch_after(kernel, *blocks, WARPS * 32, smem, s, a);
}
// The sums of dg and db are what a thread needs registers for: a warp to a row of 1280 columns leaves room for eight warps an SM
// (60.5 us at 32896 rows), two warps to a row for sixteen (58 us); at 1024 columns twelve and twenty (24.2, 23.9 us at 12608
// rows; all with some of the inputs still in L2).  On inputs that L2 does not hold, bf16 and with the residual's gradient, calls take
// 9 us for the start, the end and the second kernel, and their bytes at 6.6 TB/s: 3152 rows of 768 columns 11 us, 12608 of 768
// 21, 12608 of 1024 25, 32896 of 1280 60.  fp32 rows are twice as long in the ring.
template <typename T>
cudaError_t dispatch_backward(const BackwardArgs& a, cudaStream_t s, int* blocks) {
  constexpr bool F = sizeof(T) == 4;
  if (a.cols <= 256) return launch_backward<T, 1, 1, 16>(a, s, blocks);
  if (a.cols <= 512) return launch_backward<T, 2, 1, 16>(a, s, blocks);
  if (a.cols <= 768) return launch_backward<T, 3, 1, 12>(a, s, blocks);
  if (a.cols <= 1024) return launch_backward<T, 2, 2, F ? 16 : 20>(a, s, blocks);
  if (a.cols <= 1536) return launch_backward<T, 3, 2, F ? 12 : 16>(a, s, blocks);
  if (a.cols <= 2048) return launch_backward<T, 2, 4, F ? 16 : 20>(a, s, blocks);
  if (a.cols <= 4096) return launch_backward<T, 4, 4, F ? 8 : 12>(a, s, blocks);
  return launch_backward<T, 8, 4, F ? 4 : 8>(a, s, blocks);
}

}  // namespace

cudaError_t launch_layer_norm(const LayerNormCall& c, cudaStream_t s) {
  const ForwardArgs a{c.x, c.ldx, c.gain, c.shift, c.eps, c.y, c.ldy, c.stats, c.rows, c.cols};
  return c.act_bf16 ? dispatch_forward<bf16>(a, s) : dispatch_forward<float>(a, s);
}

cudaError_t launch_layer_norm_backward(const LayerNormCall& c, float* partial, int* blocks, cudaStream_t s) {
  const BackwardArgs a{c.x, c.ldx, c.gain, c.stats, c.dy, c.lddy, c.dres, c.lddres, c.dx, c.lddx, partial, c.rows, c.cols, 0};
  return c.act_bf16 ? dispatch_backward<bf16>(a, s, blocks) : dispatch_backward<float>(a, s, blocks);
}

cudaError_t launch_column_grad(const float* partial, int blocks, int cols, float* dgain, float* dshift, cudaStream_t s) {
  return launch_after(column_grad_kernel, 2 * cols / 8, COLUMN_THREADS, 0, s, partial, blocks, cols, dgain, dshift);
}

}  // namespace vit
