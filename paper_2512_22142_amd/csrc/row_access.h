// Elements of a row of fp32 or bf16 values, sixteen bytes or one element at a time.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "bf16_round.h"

namespace cleave {

struct Bf16 {
  uint16_t bits;
};

template <typename T>
struct Vec16;
template <>
struct Vec16<float> {
  static constexpr int N = 4;
};
template <>
struct Vec16<Bf16> {
  static constexpr int N = 8;
};

typedef float row_f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t row_u32x4 __attribute__((ext_vector_type(4)));

// VEC elements from p on: 1, or sixteen bytes' worth (p aligned to that).
template <int VEC>
__device__ __forceinline__ void load_elements(const float* p, float (&out)[VEC]) {
  if constexpr (VEC == 1) {
    out[0] = *p;
  } else {
    static_assert(VEC % 4 == 0, "whole 16 bytes");
#pragma unroll
    for (int q = 0; q < VEC / 4; ++q) {
      const row_f32x4 v = reinterpret_cast<const row_f32x4*>(p)[q];
#pragma unroll
      for (int e = 0; e < 4; ++e) out[4 * q + e] = v[e];
    }
  }
}
template <int VEC>
__device__ __forceinline__ void load_elements(const Bf16* p, float (&out)[VEC]) {
  if constexpr (VEC == 1) {
    out[0] = __builtin_bit_cast(float, static_cast<uint32_t>(p->bits) << 16);
  } else {
    static_assert(VEC == 8, "16 bytes");
    const row_u32x4 v = *reinterpret_cast<const row_u32x4*>(p);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      out[2 * q] = __builtin_bit_cast(float, v[q] << 16);
      out[2 * q + 1] = __builtin_bit_cast(float, v[q] & 0xffff0000u);
    }
  }
}
template <int VEC>
__device__ __forceinline__ void store_elements(float* p, const float (&in)[VEC]) {
  if constexpr (VEC == 1) {
    *p = in[0];
  } else {
#pragma unroll
    for (int q = 0; q < VEC / 4; ++q)
      reinterpret_cast<row_f32x4*>(p)[q] = row_f32x4{in[4 * q], in[4 * q + 1], in[4 * q + 2], in[4 * q + 3]};
  }
}
template <int VEC>
__device__ __forceinline__ void store_elements(Bf16* p, const float (&in)[VEC]) {
  if constexpr (VEC == 1) {
    p->bits = to_bf16_bits(in[0]);
  } else {
    *reinterpret_cast<row_u32x4*>(p) = row_u32x4{pack_bf16(in[0], in[1]), pack_bf16(in[2], in[3]),
                                                 pack_bf16(in[4], in[5]), pack_bf16(in[6], in[7])};
  }
}

}  // namespace cleave
