// Sums and maxima over a wave or a workgroup of whole waves.
#pragma once

#include <hip/hip_runtime.h>

namespace cleave {

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  return x;
}
// NaN wins.
__device__ __forceinline__ float nan_max(float a, float b) { return (a > b || a != a) ? a : b; }
__device__ __forceinline__ float wave_nan_max(float x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x = nan_max(x, __shfl_xor(x, d));
  return x;
}

// Over the NW waves that share `slots` (NW floats of LDS): every thread gets the result, joined in
// wave order.  One wave needs no LDS.  Two calls in a row take different slots.
template <int NW, typename Join>
__device__ __forceinline__ float join_waves(float x, float* slots, Join join) {
  if constexpr (NW > 1) {
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = x;
    __syncthreads();
    x = slots[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) x = join(x, slots[w]);
  }
  return x;
}
template <int NW>
__device__ __forceinline__ float group_sum(float x, float* slots) {
  return join_waves<NW>(wave_sum(x), slots, [](float a, float b) { return a + b; });
}
template <int NW>
__device__ __forceinline__ float group_nan_max(float x, float* slots) {
  return join_waves<NW>(wave_nan_max(x), slots, nan_max);
}

}  // namespace cleave
