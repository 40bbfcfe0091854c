// fp32 <-> e4m3 (4 exponent bits, 3 of mantissa, no infinities) on the GPU.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace cleave {

constexpr float kE4M3Max = 448.0f;
constexpr float kE4M3Least = 0.001953125f;   // 2^-9, the smallest above zero
// A row or block whose largest magnitude is below is stored as zeros with a scale of zero:
// the reciprocal of its scale would leave fp32's range.
constexpr float kLeastScaled = 7.8886090522101181e-31f;   // 2^-100

// Two values rounded to nearest even, the first in the low byte.  |x| <= 448 (1 + 2^-20), or NaN.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b) {
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false)) & 0xffffu;
}
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}
template <int BYTE>
__device__ __forceinline__ float from_e4m3(uint32_t word) {
  return __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(word), BYTE);
}

// Eight e4m3 values of two words as bf16, which holds them exactly.
__device__ __forceinline__ auto bf16_of_e4m3(uint32_t lo, uint32_t hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The scale of values of which `most` is the largest magnitude, most * (1 / 448), and its reciprocal; both zero
// below kLeastScaled, both NaN where it is infinite or NaN.
struct BlockScale {
  float scale, inverse;
};
__device__ __forceinline__ BlockScale block_scale(float most) {
  if (most < kLeastScaled) return {0.0f, 0.0f};
  if (!(most < __builtin_inff())) return {__builtin_nanf(""), __builtin_nanf("")};
  const float scale = most * (1.0f / kE4M3Max);
  return {scale, 1.0f / scale};
}

}  // namespace cleave
