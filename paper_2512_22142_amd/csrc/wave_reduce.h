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
// The same sums across lanes without LDS: rows of sixteen lanes by DPP, the four rows through scalar registers.  (In another order than
// wave_sum: kernels keep the one that they have.)
template <int CTRL>
__device__ __forceinline__ float dpp_of(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float lane_of(float x, int lane) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
}
template <int LANES, typename Join>   // eight or sixteen lanes for themselves
__device__ __forceinline__ float lanes_join(float x, Join join) {
  static_assert(LANES == 8 || LANES == 16, "halves of rows, or rows");
  x = join(x, dpp_of<0xb1>(x));    // quad_perm 1 0 3 2
  x = join(x, dpp_of<0x4e>(x));    // quad_perm 2 3 0 1
  x = join(x, dpp_of<0x141>(x));   // row_half_mirror
  if constexpr (LANES == 16) x = join(x, dpp_of<0x140>(x));   // row_mirror
  return x;
}
template <typename Join>
__device__ __forceinline__ float wave_join(float x, Join join) {
  x = lanes_join<16>(x, join);
  return join(join(lane_of(x, 0), lane_of(x, 16)), join(lane_of(x, 32), lane_of(x, 48)));
}
__device__ __forceinline__ float wave_total(float x) {
  return wave_join(x, [](float a, float b) { return a + b; });
}
// Over the NT threads of a row: eight or sixteen lanes, or whole waves (join_waves).
template <int NT>
__device__ __forceinline__ float lanes_total(float x) {
  if constexpr (NT < 64) return lanes_join<NT>(x, [](float a, float b) { return a + b; });
  else return wave_total(x);
}
template <int NT>
__device__ __forceinline__ float group_total(float x, float* slots) {
  return join_waves<NT / 64>(lanes_total<NT>(x), slots, [](float a, float b) { return a + b; });
}
// Two sums behind one barrier; twice the slots.
template <int NT>
__device__ __forceinline__ void group_totals(float& x, float& y, float* slots) {
  constexpr int NW = NT / 64;
  x = lanes_total<NT>(x);
  y = lanes_total<NT>(y);
  if constexpr (NW > 1) {
    if ((threadIdx.x & 63) == 0) {
      slots[threadIdx.x >> 6] = x;
      slots[NW + (threadIdx.x >> 6)] = y;
    }
    __syncthreads();
    x = slots[0];
    y = slots[NW];
#pragma unroll
    for (int w = 1; w < NW; ++w) {
      x += slots[w];
      y += slots[NW + w];
    }
  }
}
template <int NW>
__device__ __forceinline__ float group_nan_max(float x, float* slots) {
  return join_waves<NW>(wave_nan_max(x), slots, nan_max);
}
template <int NT>
__device__ __forceinline__ float row_nan_max(float x, float* slots) {
  if constexpr (NT < 64) return lanes_join<NT>(x, nan_max);
  else return group_nan_max<NT / 64>(x, slots);
}

}  // namespace cleave
