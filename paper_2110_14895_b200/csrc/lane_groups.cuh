// Sums over groups of neighbouring lanes of any size up to 16.
#pragma once
#include <cuda_runtime.h>

namespace vit {

// Sums over the lanes of a group (1 to 16, not always a power of two): those beyond the largest power of two are
// folded in first and fetch the result at the end.  from[k]: the lane whose sum joins in the step of 8 >> k.
struct HeadSum { int lanes, pow2, first, beyond, from[4]; };
__device__ __forceinline__ HeadSum head_sum_plan(int lanes, int at, int first) {
  HeadSum p;
  p.lanes = lanes;
  p.first = first;
  p.pow2 = lanes >= 16 ? 16 : lanes >= 8 ? 8 : lanes >= 4 ? 4 : lanes >= 2 ? 2 : 1;
  p.beyond = at + p.pow2 < lanes ? first + at + p.pow2 : -1;
#pragma unroll
  for (int k = 0; k < 4; ++k) p.from[k] = (first + (at ^ (8 >> k))) & 31;
  return p;
}
// N sums step by step together: every step waits for a shuffle
template <int N>
__device__ __forceinline__ void head_sums(float (&v)[N], const HeadSum& p) {
  const unsigned full = 0xffffffffu;
  if (p.pow2 < p.lanes) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float beyond = __shfl_sync(full, v[i], p.beyond & 31);
      if (p.beyond >= 0) v[i] += beyond;
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (p.pow2 > 8 >> k) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += __shfl_sync(full, v[i], p.from[k]);   // lanes beyond pow2 gather nothing of use
    }
  if (p.pow2 < p.lanes) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __shfl_sync(full, v[i], p.first);
  }
}
__device__ __forceinline__ float head_sum(float v, const HeadSum& p) {
  float one[1] = {v};
  head_sums(one, p);
  return one[0];
}

}  // namespace vit
