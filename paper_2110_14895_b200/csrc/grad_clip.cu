// The common norm of many tensors, and the tensors scaled down to a bound:
//   n = sqrt(sum over all tensors of x^2),  dst = x min(1, bound / n)
//
// Bound by memory: every value is read twice (the factor is known only when all have been seen) and written once.  The list
// of tensors travels in the kernels' parameters, so that a call needs no copy and a captured graph keeps its own list.
// A block owns a run of neighbouring pieces.  All gradients of ViT-H/14, 1.26 GB: 186 us for the sums (6.8 TB/s) and 420 for the
// scaling (6.0 TB/s); backwards, the second kernel would not find what the first read last in L2 either.
#include "vit_internal.h"
#include "sm100_ptx.cuh"

namespace vit {

namespace {

// Values of a piece, and threads of a block: 32 values to a thread are enough loads in flight (all gradients of ViT-H/14: 675 us
// with 16 and 256 threads, 632 with 32, 618 with 512 threads; four blocks an SM of 64 to a thread 759).
constexpr int PIECE = 16384;
constexpr int THREADS = 512;
constexpr int PER = PIECE / THREADS;           // values of a thread

struct Entry { const void* src; void* dst; int64_t count; int32_t first_piece; int32_t is_bf16; };
template <int CAP> struct List { int n, pieces; Entry e[CAP]; };

__device__ __forceinline__ float2 lo_hi(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }

// this thread's values of a piece, zeros behind the end of the tensor.  Vectors of 16 bytes, neighbouring threads side by side.
__device__ __forceinline__ void load_piece(const Entry& e, int64_t at, float (&v)[PER]) {
  const int left = (int)(e.count - at < PIECE ? e.count - at : PIECE);
  if (e.is_bf16) {
    const bf16* p = static_cast<const bf16*>(e.src) + at;
    uint4 u[PER / 8];
#pragma unroll
    for (int i = 0; i < PER / 8; ++i) {
      const int c = (i * THREADS + (int)threadIdx.x) * 8;
      u[i] = make_uint4(0, 0, 0, 0);
      if (c + 8 <= left) u[i] = *reinterpret_cast<const uint4*>(p + c);
      else if (c < left) {
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (c + k < left) w[k >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[c + k] << (16 * (k & 1));
        u[i] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
#pragma unroll
    for (int i = 0; i < PER / 8; ++i) {
      const uint32_t w[4] = {u[i].x, u[i].y, u[i].z, u[i].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 f = lo_hi(w[k]);
        v[8 * i + 2 * k] = f.x;
        v[8 * i + 2 * k + 1] = f.y;
      }
    }
  } else {
    const float* p = static_cast<const float*>(e.src) + at;
#pragma unroll
    for (int i = 0; i < PER / 4; ++i) {
      const int c = (i * THREADS + (int)threadIdx.x) * 4;
      float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
      if (c + 4 <= left) f = *reinterpret_cast<const float4*>(p + c);
      else {
        if (c < left) f.x = p[c];
        if (c + 1 < left) f.y = p[c + 1];
        if (c + 2 < left) f.z = p[c + 2];
      }
      v[4 * i] = f.x; v[4 * i + 1] = f.y; v[4 * i + 2] = f.z; v[4 * i + 3] = f.w;
    }
  }
}
__device__ __forceinline__ void store_piece(const Entry& e, int64_t at, const float (&v)[PER]) {
  const int left = (int)(e.count - at < PIECE ? e.count - at : PIECE);
  if (e.is_bf16) {
    bf16* p = static_cast<bf16*>(e.dst) + at;
#pragma unroll
    for (int i = 0; i < PER / 8; ++i) {
      const int c = (i * THREADS + (int)threadIdx.x) * 8;
      if (c + 8 <= left) {
        uint4 o;
        __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&o);
#pragma unroll
        for (int k = 0; k < 4; ++k) h[k] = __floats2bfloat162_rn(v[8 * i + 2 * k], v[8 * i + 2 * k + 1]);
        *reinterpret_cast<uint4*>(p + c) = o;
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (c + k < left) p[c + k] = __float2bfloat16_rn(v[8 * i + k]);
      }
    }
  } else {
    float* p = static_cast<float*>(e.dst) + at;
#pragma unroll
    for (int i = 0; i < PER / 4; ++i) {
      const int c = (i * THREADS + (int)threadIdx.x) * 4;
      if (c + 4 <= left) *reinterpret_cast<float4*>(p + c) = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
      else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (c + k < left) p[c + k] = v[4 * i + k];
      }
    }
  }
}

// the sum of a block's values, the same for all threads and in the same order every time
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double warps[THREADS / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int i = 0; i < THREADS / 32; ++i) v += warps[i];
  return v;
}

template <int CAP>
__device__ __forceinline__ int entry_of(const List<CAP>& list, int piece) {
  int lo = 0, hi = list.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (list.e[mid].first_piece <= piece) lo = mid;
    else hi = mid;
  }
  return lo;
}
__device__ __forceinline__ int share_begin(int total, int block, int blocks) { return (int)((int64_t)total * block / blocks); }

template <int CAP>
__global__ void __launch_bounds__(THREADS)
square_sum_kernel(const __grid_constant__ List<CAP> list, double* __restrict__ partial) {
  const int begin = share_begin(list.pieces, (int)blockIdx.x, (int)gridDim.x), end = share_begin(list.pieces, (int)blockIdx.x + 1, (int)gridDim.x);
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  double sum = 0.0;
  int at = begin < end ? entry_of(list, begin) : 0;
  for (int piece = begin; piece < end; ++piece) {
    while (at + 1 < list.n && list.e[at + 1].first_piece <= piece) ++at;      // tensors without values have no piece
    float v[PER];
    load_piece(list.e[at], (int64_t)(piece - list.e[at].first_piece) * PIECE, v);
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < PER; i += 2) s = __ffma2_rn(make_float2(v[i], v[i + 1]), make_float2(v[i], v[i + 1]), s);
    const float some = s.x + s.y;
    // 16 squares in 32 bits, all others in 64: what overflows there, or loses bits below the normal numbers, is squared in 64
    if (some < 1e30f && some > 1e-30f) sum += (double)some;
    else {
#pragma unroll
      for (int i = 0; i < PER; ++i) sum = fma((double)v[i], (double)v[i], sum);
    }
  }
  sum = block_sum(sum);
  if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

template <int CAP>
__global__ void __launch_bounds__(THREADS)
clip_kernel(const __grid_constant__ List<CAP> list, const double* __restrict__ partial, int partials, float bound, float* norm) {
  const int begin = share_begin(list.pieces, (int)blockIdx.x, (int)gridDim.x), end = share_begin(list.pieces, (int)blockIdx.x + 1, (int)gridDim.x);
  int at = begin < end ? entry_of(list, begin) : 0;
  // The first piece is fetched while the kernel before this one ends: that one, too, has only begun when nobody wrote the
  // tensors any more, and does not write them itself.
  float v[PER];
  if (begin < end && list.e[at].dst) load_piece(list.e[at], (int64_t)(begin - list.e[at].first_piece) * PIECE, v);
  ptx::grid_dependency_wait();
  double sum = 0.0;
  for (int i = threadIdx.x; i < partials; i += THREADS) sum += partial[i];
  const double n = sqrt(block_sum(sum));
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
  // not a number: so is the factor.  Infinite: zero, for any bound, and the infinite values themselves become not a number.  A factor
  // that would lose bits below the normal numbers of 32 bits, or has none left there, is applied in 64.
  const double by64 = isinf(n) ? 0.0 : n <= (double)bound ? 1.0 : (double)bound / n;
  const bool tiny = by64 > 0.0 && by64 < 0x1p-100;
  const float by = (float)by64;
  for (int piece = begin; piece < end; ++piece) {
    while (at + 1 < list.n && list.e[at + 1].first_piece <= piece) ++at;
    const Entry& e = list.e[at];
    if (!e.dst || (e.dst == e.src && by == 1.0f)) continue;
    const int64_t from = (int64_t)(piece - e.first_piece) * PIECE;
    if (piece != begin) load_piece(e, from, v);
    if (tiny) {
#pragma unroll
      for (int i = 0; i < PER; ++i) v[i] = (float)((double)v[i] * by64);
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) v[i] *= by;
    }
    store_piece(e, from, v);
  }
}

template <typename Kernel, typename... Args>
cudaError_t launch_after(Kernel kernel, int grid, cudaStream_t s, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(THREADS);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

constexpr int MOST = 960;                      // tensors of a launch: 30 KB of the 32 that parameters may have

int grid_of(int pieces) {
  const int most = current_device_sm_count() * 4;
  const int grid = pieces < most ? pieces : most;
  return grid < 1 ? 1 : grid > GRAD_CLIP_MAX_BLOCKS ? GRAD_CLIP_MAX_BLOCKS : grid;
}

template <int CAP>
void fill(List<CAP>& list, const vit_tensor* t, int n) {
  list.n = n;
  int pieces = 0;
  for (int i = 0; i < n; ++i) {
    list.e[i] = Entry{t[i].src, t[i].dst, t[i].count, pieces, t[i].dtype == VIT_BF16};
    pieces += (int)((t[i].count + PIECE - 1) / PIECE);
  }
  list.pieces = pieces;
}
template <int CAP>
cudaError_t launch_list(const vit_tensor* t, int n, bool clip, double* partial, int* partials, float bound, float* norm, cudaStream_t s) {
  List<CAP> list;
  fill(list, t, n);
  const int grid = grid_of(list.pieces);
  if (clip) return launch_after(clip_kernel<CAP>, grid, s, list, partial, *partials, bound, norm);
  *partials = grid;
  return launch_after(square_sum_kernel<CAP>, grid, s, list, partial);
}

}  // namespace

int grad_clip_lists(int tensors) { return tensors <= MOST ? 1 : (tensors - 1) / MOST + 1; }

// list number `index` of the call's: its sum of squares (clip == false; *partials: how many parts it leaves) or its scaling
cudaError_t launch_grad_clip(const vit_tensor* tensors, int count, int index, bool clip, double* partial, int* partials, float bound,
                             float* norm, cudaStream_t s) {
  const vit_tensor* t = tensors + (size_t)index * MOST;
  const int n = count - index * MOST < MOST ? count - index * MOST : MOST;
  if (n <= 32) return launch_list<32>(t, n, clip, partial, partials, bound, norm, s);
  if (n <= 192) return launch_list<192>(t, n, clip, partial, partials, bound, norm, s);
  if (n <= 480) return launch_list<480>(t, n, clip, partial, partials, bound, norm, s);
  return launch_list<MOST>(t, n, clip, partial, partials, bound, norm, s);
}

}  // namespace vit
