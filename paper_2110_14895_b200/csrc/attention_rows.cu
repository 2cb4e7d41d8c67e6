// Attention of few queries over many keys (attention pooling: one learned query per image; single tokens when
// served).  Nothing is reused but the queries, so what bounds it is the bytes of K and V, and with the usual few
// thousand keys the latency of fetching them.
//
// The keys of a (sequence, key head) are shared by the blocks of a cluster; a block takes up to four rows (queries
// of the heads that share the key head) along, so that K and V are read once for them.  A key belongs to d / 8
// lanes, eight channels to a lane; as many keys side by side in a warp as fit, four of them one after the other in
// flight.  Every group of lanes keeps its own running maximum, sum and weighted values; they are joined in shared
// memory, and the blocks' results through the cluster's shared memory, in a fixed order, in the same launch.
#include "vit_internal.h"
#include "attention_packed.cuh"
#include "lane_groups.cuh"
#include "sm100_ptx.cuh"

namespace vit {

namespace {

constexpr int WARPS = 4, THREADS = 32 * WARPS, UNROLL = 4;

struct Eight { float v[8]; };
template <typename T> struct Raw;                          // eight channels as they lie in memory
template <> struct Raw<bf16> { uint4 v; };
template <> struct Raw<float> { float4 v[2]; };
__device__ __forceinline__ Raw<float> load8(const float* a) {
  return Raw<float>{{reinterpret_cast<const float4*>(a)[0], reinterpret_cast<const float4*>(a)[1]}};
}
__device__ __forceinline__ Raw<bf16> load8(const bf16* a) { return Raw<bf16>{*reinterpret_cast<const uint4*>(a)}; }
__device__ __forceinline__ Eight open8(const Raw<float>& r) {
  return Eight{{r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w, r.v[1].x, r.v[1].y, r.v[1].z, r.v[1].w}};
}
__device__ __forceinline__ Eight open8(const Raw<bf16>& r) {
  const uint4 u = r.v;
  return Eight{{__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u),
                __uint_as_float(u.z << 16), __uint_as_float(u.z & 0xffff0000u), __uint_as_float(u.w << 16), __uint_as_float(u.w & 0xffff0000u)}};
}
__device__ __forceinline__ void store1(float* a, float v) { *a = v; }
__device__ __forceinline__ void store1(bf16* a, float v) { *a = __float2bfloat16_rn(v); }

__device__ __forceinline__ void peer_store(uint32_t own_addr, uint32_t rank, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(ptx::map_to_cta(own_addr, rank)), "f"(v) : "memory");
}

// grid: clusters of `splits` blocks, one per (sequence, key head, ROWS rows)
template <typename T, int ROWS>
__global__ void __launch_bounds__(THREADS)
packed_rows_kernel(const PackedCall c, int row_blocks, int splits) {
  // [groups][ROWS][d + 2]: weighted values, maximum, sum; then the same of the cluster's blocks, in its first one: [splits][ROWS][d + 2]
  extern __shared__ __align__(16) float sm[];
  const int d = c.p.d, lanes = d / 8, side = 32 / lanes, groups = WARPS * side, width = d + 2;
  const int item = blockIdx.x / splits, rank = blockIdx.x % splits;
  const int rb = item % row_blocks, kv = item / row_blocks % c.p.kv_heads, seq = item / row_blocks / c.p.kv_heads;
  const int group = c.p.heads / c.p.kv_heads;
  SeqRange r;
  if (!seq_range(c.p, seq, r, c.dev_status, threadIdx.x == 0)) return;       // the whole cluster leaves
  const int row0 = rb * ROWS, rows = min(ROWS, r.q_len * group - row0);   // row = query * group + head of the group
  if (rows <= 0) return;
  if (splits > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");      // this block runs
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, slot = lane / lanes, at = lane - slot * lanes;
  const bool active = slot < side;
  const HeadSum sums = head_sum_plan(lanes, at, active ? slot * lanes : 0);
  const int c0 = active ? at * 8 : 0;
  const float sl2 = c.p.scale * 1.4426950408889634f;

  Eight q[ROWS];
  float m[ROWS], l[ROWS], acc[ROWS][8];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int row = row0 + min(i, rows - 1);
    q[i] = open8(load8(static_cast<const T*>(c.q) + ((int64_t)r.q_begin + row / group) * c.ldq + (int64_t)(kv * group + row % group) * d + c0));
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      q[i].v[e] = active ? q[i].v[e] * sl2 : 0.f;          // scores in units of log2
      acc[i][e] = 0.f;
    }
  }
  const int chunk = (r.k_len + splits - 1) / splits, begin = min(r.k_len, rank * chunk), end = min(r.k_len, begin + chunk);
  const T* kp = static_cast<const T*>(c.k) + (int64_t)kv * d + c0;
  const T* vp = static_cast<const T*>(c.v) + (int64_t)kv * d + c0;
  // the keys of the next round are on their way while this one's are worked on; keys that are not there are zero
  // (nothing of what lies behind them is looked at) and get probabilities of zero
  Raw<T> kn[UNROLL], vn[UNROLL];
  auto fetch = [&](int k0) {
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int key = k0 + u * groups + slot;
      kn[u] = Raw<T>{};
      vn[u] = Raw<T>{};
      if (active && key < end) {
        kn[u] = load8(kp + ((int64_t)r.k_begin + key) * c.ldk);
        vn[u] = load8(vp + ((int64_t)r.k_begin + key) * c.ldv);
      }
    }
  };
  fetch(begin + warp * side);
  for (int k0 = begin + warp * side; k0 < end; k0 += groups * UNROLL) {
    Eight kk[UNROLL], vv[UNROLL];
    bool there[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      there[u] = active && k0 + u * groups + slot < end;
      kk[u] = open8(kn[u]);
      vv[u] = open8(vn[u]);
    }
    if (k0 + groups * UNROLL < end) fetch(k0 + groups * UNROLL);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      float s[UNROLL];
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        s[u] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) s[u] = fmaf(q[i].v[e], kk[u].v[e], s[u]);
      }
      head_sums(s, sums);
      float top = m[i];
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        if (!there[u]) s[u] = -INFINITY;
        top = fmaxf(top, s[u]);
      }
      const float ref = top == -INFINITY ? 0.f : top, keep = exp2f(m[i] - ref);
      m[i] = top;
      l[i] *= keep;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[i][e] *= keep;
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        const float p = exp2f(s[u] - ref);
        l[i] += p;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[i][e] = fmaf(p, vv[u].v[e], acc[i][e]);
      }
    }
  }
  if (active) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      float* to = sm + ((warp * side + slot) * ROWS + i) * width;
#pragma unroll
      for (int e = 0; e < 8; ++e) to[c0 + e] = acc[i][e];
      if (at == 0) {
        to[d] = m[i];
        to[d + 1] = l[i];
      }
    }
  }
  __syncthreads();
  // the block's groups of lanes, in order: every channel gathers the common maximum for itself
  float* joined = sm + groups * ROWS * width;
  const uint32_t mine = ptx::smem_u32(joined + rank * ROWS * width);
  if (splits > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");                // the first block runs
  for (int e = threadIdx.x; e < ROWS * d; e += THREADS) {
    const int i = e / d, ch = e - i * d;
    float top = -INFINITY, sum = 0.f, o = 0.f;
    for (int g = 0; g < groups; ++g) top = fmaxf(top, sm[(g * ROWS + i) * width + d]);
    const float ref = top == -INFINITY ? 0.f : top;
    for (int g = 0; g < groups; ++g) {
      const float* from = sm + (g * ROWS + i) * width;
      const float f = exp2f(from[d] - ref);
      sum = fmaf(f, from[d + 1], sum);
      o = fmaf(f, from[ch], o);
    }
    peer_store(mine + (uint32_t)(i * width + ch) * 4, 0, o);
    if (ch == 0) {
      peer_store(mine + (uint32_t)(i * width + d) * 4, 0, top);
      peer_store(mine + (uint32_t)(i * width + d + 1) * 4, 0, sum);
    }
  }
  if (splits > 1) ptx::cluster_sync();
  else __syncthreads();
  if (rank != 0) return;
  // the blocks, in order
  for (int e = threadIdx.x; e < rows * d; e += THREADS) {
    const int i = e / d, ch = e - i * d;
    float top = -INFINITY, sum = 0.f, o = 0.f;
    for (int b = 0; b < splits; ++b) top = fmaxf(top, joined[(b * ROWS + i) * width + d]);
    const float ref = top == -INFINITY ? 0.f : top;
    for (int b = 0; b < splits; ++b) {
      const float* from = joined + (b * ROWS + i) * width;
      const float f = exp2f(from[d] - ref);
      sum = fmaf(f, from[d + 1], sum);
      o = fmaf(f, from[ch], o);
    }
    const int row = row0 + i, head = kv * group + row % group;
    const int64_t to = (int64_t)r.q_begin + row / group;
    store1(static_cast<T*>(c.out) + to * c.ldo + (int64_t)head * d + ch, sum == 0.f ? 0.f : o / sum);      // no keys: zero
    if (ch == 0) c.lse[(int64_t)head * c.p.q_rows + to] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.69314718055994531f;
  }
}

template <typename T, int ROWS>
cudaError_t launch_variant(const PackedCall& c, cudaStream_t s) {
  const int sms = current_device_sm_count();
  if (sms < 1) return cudaErrorInvalidDevice;
  const int group = c.p.heads / c.p.kv_heads, row_blocks = (c.p.max_q * group + ROWS - 1) / ROWS;
  const int64_t items = (int64_t)c.p.sequences * c.p.kv_heads * row_blocks;
  // as many blocks to a (sequence, key head) as fill the device twice, of 64 keys at least, eight at most
  int splits = 1;
  while (splits < 8 && items * splits < 2 * sms && c.p.max_k > 64 * splits) splits *= 2;
  const int lanes = c.p.d / 8, groups = WARPS * (32 / lanes);
  const size_t smem = (size_t)(groups + splits) * ROWS * (c.p.d + 2) * sizeof(float);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(items * splits));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)splits;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, packed_rows_kernel<T, ROWS>, c, row_blocks, splits);
}
template <typename T>
cudaError_t launch_rows(const PackedCall& c, cudaStream_t s) {
  const int rows = c.p.max_q * (c.p.heads / c.p.kv_heads);
  return rows == 1 ? launch_variant<T, 1>(c, s) : rows == 2 ? launch_variant<T, 2>(c, s) : launch_variant<T, 4>(c, s);
}

}  // namespace

// Four rows at most in bf16 (2 images of 1025 tokens, 16 heads of 64: 5.9, 7.1, 11 and 22 us for 1, 2, 4 and 8 rows,
// against 18 us of the kernel that works on tiles of 128 rows), eight in fp32, whose other kernel has no tensor core.
// Measured with few images, where latency counts; with many, where the crossing lies is not known.
bool attention_rows_supported(const vit_attention_problem& p, bool act_bf16) {
  return (int64_t)p.max_q * (p.heads / p.kv_heads) <= (act_bf16 ? 4 : 8);
}
cudaError_t launch_attention_rows(const PackedCall& c, bool act_bf16, cudaStream_t s) {
  return act_bf16 ? launch_rows<bf16>(c, s) : launch_rows<float>(c, s);
}

}  // namespace vit
