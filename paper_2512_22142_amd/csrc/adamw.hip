// AdamW over many tensors in one launch (paper Sec. 4.1 and Sec. 6: optimizer
// updates stay on the parameter server and stream over its weights):
//   g = c g;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2
//   w = w - lr ( (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps) + wd w )
// in fp32, every operation rounded by itself (no fused multiply-adds), so that a
// program of elementary operations gets the same bits.
//
// 8-bit states: m and r = sqrt(v) as e4m3 with one fp32 scale per 256 consecutive elements, the
// largest magnitude over 448.  e4m3 spans 2^-9 to 448, so r covers a range of 2^35 in v within
// a block to 6 % steps, where v itself would leave it; an r above zero is never rounded to
// zero, which would leave m over eps alone as the step.  A value that is not finite becomes
// NaN and leaves its block's scale to the others.  The update of w uses m and v before they are
// rounded.
//
// Bound by memory: 28 bytes per weight and step in 32 bits with a bf16 gradient and copy, 16 in 8 bits.  A wave has a block
// of 256 weights, four to a lane, so a block's largest magnitude is a reduction over the wave and every access is a run of the
// whole wave; a workgroup has 4096 weights, and the tensors' list travels in the kernel's arguments, so up to
// 56 of any sizes share a launch.  7.1 M weights in 32 bits 36-37 us (5.4 TB/s), 202 M in 8 bits 601-640 us (5.1 to 5.4).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "bf16_round.h"
#include "fp8_round.h"
#include "operators.h"

namespace cleave {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// A lane's four neighbouring elements of a block, at any alignment; `left`: how many there are.  What is not there reads as zero
// and is not written.
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32_any __attribute__((aligned(1)));

__device__ __forceinline__ f32x4 load_four(const float* p, int left) {
  if (left >= 4) return *reinterpret_cast<const f32x4_any*>(p);
  f32x4 x{};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < left) x[e] = p[e];
  return x;
}
__device__ __forceinline__ f32x4 load_four(const uint16_t* p, int left) {
  if (left >= 4) {
    const u32x2 b = *reinterpret_cast<const u32x2_any*>(p);
    return f32x4{__builtin_bit_cast(float, b[0] << 16), __builtin_bit_cast(float, b[0] & 0xffff0000u),
                 __builtin_bit_cast(float, b[1] << 16), __builtin_bit_cast(float, b[1] & 0xffff0000u)};
  }
  f32x4 x{};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < left) x[e] = __builtin_bit_cast(float, static_cast<uint32_t>(p[e]) << 16);
  return x;
}
__device__ __forceinline__ uint32_t load_four(const uint8_t* p, int left) {
  if (left >= 4) return *reinterpret_cast<const u32_any*>(p);
  uint32_t x = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < left) x |= static_cast<uint32_t>(p[e]) << (8 * e);
  return x;
}
__device__ __forceinline__ void store_four(float* p, f32x4 x, int left) {
  if (left >= 4) {
    *reinterpret_cast<f32x4_any*>(p) = x;
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < left) p[e] = x[e];
}
__device__ __forceinline__ void store_four(uint16_t* p, f32x4 x, int left) {
  if (left >= 4) {
    *reinterpret_cast<u32x2_any*>(p) = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < left) p[e] = to_bf16_bits(x[e]);
}
__device__ __forceinline__ void store_four(uint8_t* p, uint32_t x, int left) {
  if (left >= 4) {
    *reinterpret_cast<u32_any*>(p) = x;
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < left) p[e] = static_cast<uint8_t>(x >> (8 * e));
}

__device__ __forceinline__ f32x4 decode(uint32_t q, float scale) {
#pragma clang fp contract(off)
  return f32x4{from_e4m3<0>(q) * scale, from_e4m3<1>(q) * scale, from_e4m3<2>(q) * scale, from_e4m3<3>(q) * scale};
}

// The largest finite magnitude of a block.
__device__ __forceinline__ float largest(f32x4 x) {
  float most = 0.0f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float a = __builtin_fabsf(x[e]);
    most = a > most && a < __builtin_inff() ? a : most;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) most = __builtin_fmaxf(most, __shfl_xor(most, d));
  return most;
}

template <bool UP>
__device__ __forceinline__ uint32_t encode(f32x4 x, float inverse) {
#pragma clang fp contract(off)
  float q[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    q[e] = x[e] * inverse;
    if (UP && x[e] > 0.0f && inverse > 0.0f) q[e] = __builtin_fmaxf(q[e], kE4M3Least);
    // infinities and NaN: NaN, whatever the instruction makes of what lies beyond 448
    if (!(__builtin_fabsf(x[e]) < __builtin_inff())) q[e] = __builtin_nanf("");
  }
  return pack_e4m3(q[0], q[1], q[2], q[3]);
}

struct Block {
  f32x4 w, g, m, v;
};

template <bool GRAD_BF16, bool STATES_8>
struct Update {
  const AdamTensor& t;
  const AdamWArgs& args;
  float clip;

  // This lane's elements of the block that starts at element `first`: from `at` on, `left` of them there.
  __device__ __forceinline__ Block load(uint64_t first, uint64_t at, int left) const {
    Block b;
    b.w = load_four(t.w + at, left);
    if constexpr (GRAD_BF16) b.g = load_four(static_cast<const uint16_t*>(t.g) + at, left);
    else b.g = load_four(static_cast<const float*>(t.g) + at, left);
    if constexpr (STATES_8) {
      const uint32_t qm = load_four(static_cast<const uint8_t*>(t.m) + at, left);
      const uint32_t qv = load_four(static_cast<const uint8_t*>(t.v) + at, left);
      b.m = decode(qm, t.m_scale[first / kStateBlock]);
      b.v = decode(qv, t.v_scale[first / kStateBlock]);
    } else {
      b.m = load_four(static_cast<const float*>(t.m) + at, left);
      b.v = load_four(static_cast<const float*>(t.v) + at, left);
    }
    return b;
  }

  __device__ __forceinline__ void step(Block b, uint64_t first, uint64_t at, int left, int lane) const {
#pragma clang fp contract(off)
    f32x4 w1, m1, v1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float g = b.g[e] * clip;
      const float v0 = STATES_8 ? b.v[e] * b.v[e] : b.v[e];
      m1[e] = args.beta1 * b.m[e] + args.one_minus_beta1 * g;
      v1[e] = args.beta2 * v0 + args.one_minus_beta2 * (g * g);
      const float root = __builtin_sqrtf(v1[e] * args.inv_bias2) + args.eps;
      w1[e] = b.w[e] - args.lr * ((m1[e] * args.inv_bias1) / root + args.weight_decay * b.w[e]);
    }
    store_four(t.w + at, w1, left);
    if (t.copy) store_four(t.copy + at, w1, left);
    if constexpr (STATES_8) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v1[e] = __builtin_sqrtf(v1[e]);
        if (e >= left) m1[e] = v1[e] = 0.0f;   // (0 times a scale of the gradients that is not finite)
      }
      const BlockScale sm = block_scale(largest(m1)), sv = block_scale(largest(v1));
      store_four(static_cast<uint8_t*>(t.m) + at, encode<false>(m1, sm.inverse), left);
      store_four(static_cast<uint8_t*>(t.v) + at, encode<true>(v1, sv.inverse), left);
      if (lane == 0) {
        t.m_scale[first / kStateBlock] = sm.scale;
        t.v_scale[first / kStateBlock] = sv.scale;
      }
    } else {
      store_four(static_cast<float*>(t.m) + at, m1, left);
      store_four(static_cast<float*>(t.v) + at, v1, left);
    }
  }

  // Wave `wave` of the workgroup takes every kWaves-th block of 256 of the chunk.
  __device__ __forceinline__ void chunk(uint64_t start, int wave, int lane) const {
    const uint64_t end = start + kAdamChunk < t.n ? start + kAdamChunk : t.n;
    for (uint64_t first = start + wave * kStateBlock; first < end; first += kWaves * kStateBlock) {
      const uint64_t at = first + 4 * lane;
      const int left = at < end ? static_cast<int>(end - at < 4 ? end - at : 4) : 0;
      step(load(first, at, left), first, at, left, lane);
    }
  }
};

template <bool GRAD_BF16, bool STATES_8>
__global__ __launch_bounds__(kThreads) void adamw_kernel(AdamWArgs args) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // The tensor that chunk blockIdx.x belongs to: as many as end before it.  (A lane looks at one.)
  const bool before = lane < args.n_tensors && args.chunk_end[lane] <= blockIdx.x;
  const int k = __popcll(__ballot(before));
  const AdamTensor& t = args.tensors[k];
  const uint32_t chunk0 = k > 0 ? args.chunk_end[k - 1] : 0;
  const uint64_t first = static_cast<uint64_t>(blockIdx.x - chunk0) * kAdamChunk;
  const float clip = args.grad_scale ? *args.grad_scale : 1.0f;
  Update<GRAD_BF16, STATES_8>{t, args, clip}.chunk(first, wave, lane);
}

}  // namespace

hipError_t launch_adamw(const AdamWArgs& args, uint32_t chunks, int grad_dtype, bool states_8bit, hipStream_t stream) {
  const dim3 g(chunks), b(kThreads);
  const bool bf16 = grad_dtype == CLEAVE_BF16;
  if (bf16 && states_8bit) hipLaunchKernelGGL((adamw_kernel<true, true>), g, b, 0, stream, args);
  else if (bf16) hipLaunchKernelGGL((adamw_kernel<true, false>), g, b, 0, stream, args);
  else if (states_8bit) hipLaunchKernelGGL((adamw_kernel<false, true>), g, b, 0, stream, args);
  else hipLaunchKernelGGL((adamw_kernel<false, false>), g, b, 0, stream, args);
  return hipGetLastError();
}

}  // namespace cleave
