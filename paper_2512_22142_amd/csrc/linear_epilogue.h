// What a product's elements go through on their way out: bias, activation (or an
// activation's slope) and residual, and the stores of the two execute kernels with that.
//
//   z = sum sa sb + b;  y = act(z) + r          (z kept if asked for)
//   y = (sum sa sb) act'(z) + r                 (z given: the gradient of an activation's input)
//
// in fp32, rounded once to the output's type.  sa, sb: scales of A's rows and B's columns
// (8-bit operands).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "bf16_round.h"
#include "kernels.h"
#include "tile_store.h"

namespace cleave {

// ---- activations -------------------------------------------------------------

// 1 / (1 + e^-x).  The exponential and the reciprocal are the hardware's (an ulp or two);
// e^-x may overflow: the reciprocal of infinity is zero.
__device__ __forceinline__ float sigmoid(float x) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896f * x));
}
// gelu with tanh: z/2 (1 + tanh(u)) = z sigmoid(2 u), u = sqrt(2 / pi) (z + 0.044715 z^3).
constexpr float kGelu2 = 1.5957691216057308f;   // 2 sqrt(2 / pi)
constexpr float kGelu3 = 0.044715f;

__device__ __forceinline__ float act_value(float z, int act) {
  switch (act) {
    case CLEAVE_ACT_RELU: return z < 0.0f ? 0.0f : z;   // NaN stays
    case CLEAVE_ACT_GELU_TANH: return z * sigmoid(kGelu2 * (z + kGelu3 * z * z * z));
    case CLEAVE_ACT_SILU: return z * sigmoid(z);
    default: return z;
  }
}
__device__ __forceinline__ float act_slope(float z, int act) {
  switch (act) {
    case CLEAVE_ACT_RELU: return z > 0.0f ? 1.0f : 0.0f;
    case CLEAVE_ACT_GELU_TANH: {
      const float p = sigmoid(kGelu2 * (z + kGelu3 * z * z * z)), q = p * (1.0f - p);
      return q > 0.0f ? p + z * q * (kGelu2 * (1.0f + 3.0f * kGelu3 * z * z)) : p;   // (infinite z: p)
    }
    case CLEAVE_ACT_SILU: {
      const float p = sigmoid(z), q = p * (1.0f - p);
      return q > 0.0f ? p + z * q : p;
    }
    default: return 1.0f;
  }
}

// No epilogue: the kernels as cleave_execute and cleave_execute_assemble run them.
struct NoEpilogue {
  static constexpr bool kLinear = false;
};
struct LinearEpilogue : LinearArgs {
  static constexpr bool kLinear = true;
};

// The epilogue's arguments, read from the kernel's argument segment (`OFFSET` bytes in) where they are needed:
// held from the kernel's start on, they take scalar registers that the K loop then spills.
template <size_t OFFSET>
__device__ __forceinline__ LinearArgs late_linear_args() {
  static_assert(OFFSET % 8 == 0 && sizeof(LinearArgs) % 8 == 0, "whole words");
  typedef const __attribute__((address_space(4))) unsigned char* const_bytes;
  typedef const __attribute__((address_space(4))) uint64_t* const_words;
  const_bytes p = (const_bytes)__builtin_amdgcn_kernarg_segment_ptr() + OFFSET;
  asm volatile("" : "+s"(p));
  const_words src = (const_words)p;
  uint64_t words[sizeof(LinearArgs) / 8];
#pragma unroll
  for (size_t k = 0; k < sizeof(LinearArgs) / 8; ++k) words[k] = src[k];
  LinearArgs e;
  __builtin_memcpy(&e, words, sizeof(e));
  return e;
}

// ---- sixteen bytes of a row ------------------------------------------------------

// Elements of the output's type in sixteen bytes of a row, as floats.
template <bool BF16>
struct Piece {
  static constexpr int N = BF16 ? 8 : 4;
  typedef uint32_t Raw __attribute__((ext_vector_type(4)));
  typedef uint32_t RawAny __attribute__((ext_vector_type(4), aligned(2)));   // at any element
  float v[N];

  __device__ __forceinline__ static Raw read(const void* p) { return *static_cast<const RawAny*>(p); }
  // The first `n` elements, fewer than N.
  __device__ __forceinline__ static Raw read(const void* p, int n) {
    Raw w{};
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if (e >= n) continue;
      if constexpr (BF16) w[e / 2] |= static_cast<uint32_t>(static_cast<const uint16_t*>(p)[e]) << (16 * (e % 2));
      else w[e] = static_cast<const uint32_t*>(p)[e];
    }
    return w;
  }
  __device__ __forceinline__ void store(void* p, int n) const {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if (e >= n) continue;
      if constexpr (BF16) static_cast<uint16_t*>(p)[e] = to_bf16_bits(v[e]);
      else static_cast<float*>(p)[e] = v[e];
    }
  }
  __device__ __forceinline__ static Piece of(Raw w) {
    Piece x;
    // (the whole vector is cast: a bit_cast of one element of it is miscompiled into a read of element 0)
    typedef float Floats __attribute__((ext_vector_type(4)));
    [[maybe_unused]] const Floats f = __builtin_bit_cast(Floats, w);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (BF16) {
        x.v[2 * e] = __builtin_bit_cast(float, w[e] << 16);
        x.v[2 * e + 1] = __builtin_bit_cast(float, w[e] & 0xffff0000u);
      } else {
        x.v[e] = f[e];
      }
    }
    return x;
  }
  __device__ __forceinline__ void store(void* p) const {
    Raw w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (BF16) w[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
      else w[e] = __builtin_bit_cast(uint32_t, v[e]);
    }
    *static_cast<RawAny*>(p) = w;
  }
};

// The epilogue of N elements of a row.  t: the sums, then what is stored; z: the given z's, then (without
// `grad`) the new ones.
template <int N>
__device__ __forceinline__ void finish(const LinearArgs& e, float (&t)[N], float (&z)[N], const float (&bias)[N],
                                       const float (&scale_b)[N], float scale_a, const float (&residual)[N]) {
  if (e.scale_a) {
#pragma unroll
    for (int k = 0; k < N; ++k) t[k] = t[k] * scale_a * scale_b[k];
  }
  if (e.grad) {
#pragma unroll
    for (int k = 0; k < N; ++k) t[k] *= act_slope(z[k], e.act);
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      z[k] = t[k] + bias[k];
      t[k] = act_value(z[k], e.act);
    }
  }
#pragma unroll
  for (int k = 0; k < N; ++k) t[k] += residual[k];
}

// ---- stores of the direct kernel -------------------------------------------------

// store_rows (tile_store.h) with the epilogue: the sums go through the wave's image in fp32, and a
// lane takes sixteen output bytes' worth of a row from it.  m_base / n_base: the sub-tile's place in the
// output.  One turn per row of blocks, not unrolled: with all of them in line the code is beyond
// the instruction cache and its addresses spill.  What a turn reads is fetched during the one before.
template <bool BF16, bool INTERIOR, int MB, int NB>
__device__ __forceinline__ void store_linear_rows(const tile_f32x4 (&acc)[MB][NB], const LinearArgs& e, const TileTarget& t,
                                                  unsigned char* image, int wave_row0, int wave_col0, int lane, int m_valid,
                                                  int n_valid, int64_t m_base, int64_t n_base) {
  typedef Piece<BF16> P;
  constexpr int N = P::N;
  constexpr int EB = BF16 ? 2 : 4;
  constexpr int Q = NB * 4;                    // 16-byte pieces of an image row
  constexpr int R = 16 / Q;                    // image rows in a cycle of the banks
  constexpr int L = NB * 16 / N;               // lanes to a row
  constexpr int RR = 64 / L;                   // rows per read of the whole wave
  constexpr int K = 16 / RR;                   // reads of the whole wave per row of blocks
  static_assert(16 * Q * 16 <= kBlockImageBytes && Q * R == 16 && 16 % RR == 0, "image");
  const int wrow = lane & 15, wflip = (wrow / R) & (Q - 1);
  const int rrow = lane / L, rpiece = (lane % L) * (N / 4);
  int row = wave_row0 + rrow;
  const int col = wave_col0 + rpiece * 4;
  // columns of this lane's that there are: all N, where every row of the output is whole pieces
  const int cols = INTERIOR ? N : min(N, n_valid - col);
  const auto valid = [&](int r) { return INTERIOR || (r < m_valid && cols > 0); };
  const auto read = [&](const unsigned char* p) { return INTERIOR || cols == N ? P::read(p) : P::read(p, cols); };
  const auto store = [&](const P& x, unsigned char* p) {
    if (INTERIOR || cols == N) x.store(p);
    else x.store(p, cols);
  };

  float bias[N] = {}, scale_b[N] = {};
  const auto read_columns = [&](const float* from, float (&to)[N]) {
    typedef float quad __attribute__((ext_vector_type(4), aligned(4)));
    const float* p = from + n_base + col;
    if (INTERIOR || cols == N) {
#pragma unroll
      for (int q = 0; q < N / 4; ++q) {
        const quad b = reinterpret_cast<const quad*>(p)[q];
#pragma unroll
        for (int c = 0; c < 4; ++c) to[4 * q + c] = b[c];
      }
    } else {
#pragma unroll
      for (int c = 0; c < N; ++c)
        if (c < cols) to[c] = p[c];
    }
  };
  if (e.bias) read_columns(e.bias, bias);
  if (e.scale_b) read_columns(e.scale_b, scale_b);
  const int64_t grow = m_base + row, gcol = n_base + col;
  unsigned char* out = t.base + (row * t.ld + col) * EB;
  unsigned char* zp = static_cast<unsigned char*>(e.preact) + (grow * e.ldz + gcol) * EB;
  const unsigned char* rp = static_cast<const unsigned char*>(e.residual) + (grow * e.ldr + gcol) * EB;
  const float* sp = e.scale_a + grow;
  const int64_t out_pitch = t.ld * EB, z_pitch = e.ldz * EB, r_pitch = e.ldr * EB;
  const bool reads_z = e.grad && e.preact, writes_z = !e.grad && e.preact;

  typename P::Raw z_next[K], r_next[K];
  float s_next[K];
  const auto fetch = [&](int first) {   // rows first + RR k from the pointers as they stand
#pragma unroll
    for (int k = 0; k < K; ++k) {
      z_next[k] = r_next[k] = typename P::Raw{};
      s_next[k] = 0.0f;
      if (!valid(first + RR * k)) continue;
      if (reads_z) z_next[k] = read(zp + RR * k * z_pitch);
      if (e.residual) r_next[k] = read(rp + RR * k * r_pitch);
      if (e.scale_a) s_next[k] = sp[RR * k];
    }
  };
  fetch(row);
#pragma unroll 1
  for (int i = 0; i < MB; ++i) {
    asm volatile("" ::: "memory");
#pragma unroll
    for (int ii = 0; ii < MB; ++ii)
      if (ii == i) {
#pragma unroll
        for (int j = 0; j < NB; ++j)
          *reinterpret_cast<tile_f32x4*>(image + (wrow * Q + ((4 * j + (lane >> 4)) ^ wflip)) * 16) = acc[ii][j];
      }
    asm volatile("" ::: "memory");
    typename P::Raw z_raw[K], r_raw[K];
    float s_now[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      z_raw[k] = z_next[k];
      r_raw[k] = r_next[k];
      s_now[k] = s_next[k];
    }
    unsigned char* const z_out = zp;
    zp += 16 * z_pitch;
    rp += 16 * r_pitch;
    sp += 16;
    if (i + 1 < MB) fetch(row + 16);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int r = rrow + RR * k;
      float x[N];
#pragma unroll
      for (int q = 0; q < N / 4; ++q) {
        const tile_f32x4 part =
            *reinterpret_cast<const tile_f32x4*>(image + (r * Q + ((rpiece + q) ^ ((r / R) & (Q - 1)))) * 16);
#pragma unroll
        for (int c = 0; c < 4; ++c) x[4 * q + c] = part[c];
      }
      P z = P::of(z_raw[k]);
      const P residual = P::of(r_raw[k]);
      finish<N>(e, x, z.v, bias, scale_b, s_now[k], residual.v);
      if (valid(row + RR * k)) {
        if (writes_z) store(z, z_out + RR * k * z_pitch);
        P y;
#pragma unroll
        for (int c = 0; c < N; ++c) y.v[c] = x[c];
        store(y, out + RR * k * out_pitch);
      }
    }
    asm volatile("" ::: "memory");
    row += 16;
    out += 16 * out_pitch;
  }
}

// ---- single elements -------------------------------------------------------------

template <bool BF16>
__device__ __forceinline__ float load_element(const void* base, int64_t at) {
  if constexpr (BF16)
    return __builtin_bit_cast(float, static_cast<uint32_t>(static_cast<const uint16_t*>(base)[at]) << 16);
  else
    return static_cast<const float*>(base)[at];
}
template <bool BF16>
__device__ __forceinline__ void store_element(void* base, int64_t at, float x) {
  if constexpr (BF16) static_cast<uint16_t*>(base)[at] = to_bf16_bits(x);
  else static_cast<float*>(base)[at] = x;
}
// Element (row, col) of the output, from its sum: what is stored.
template <bool BF16>
__device__ __forceinline__ float finish_element(const LinearArgs& e, float sum, int64_t row, int64_t col) {
  float t[1] = {sum}, z[1] = {0.0f};
  if (e.grad && e.preact) z[0] = load_element<BF16>(e.preact, row * e.ldz + col);
  const float bias[1] = {e.bias ? e.bias[col] : 0.0f}, scale_b[1] = {e.scale_b ? e.scale_b[col] : 0.0f};
  const float residual[1] = {e.residual ? load_element<BF16>(e.residual, row * e.ldr + col) : 0.0f};
  finish<1>(e, t, z, bias, scale_b, e.scale_a ? e.scale_a[row] : 0.0f, residual);
  if (!e.grad && e.preact) store_element<BF16>(e.preact, row * e.ldz + col, z[0]);
  return t[0];
}

// ---- stores of the general kernel ------------------------------------------------

// store_tile with the epilogue, a block of 32 x 32 sums at a time.
template <bool BF16, int MB, int NB>
__device__ __forceinline__ void store_linear_tile_as(const tile_f32x16 (&acc)[MB][NB], const LinearArgs& e, const TileTarget& t,
                                                     int row0, int col0, int m_valid, int n_valid, int64_t m_base,
                                                     int64_t n_base) {
#pragma unroll 1
  for (int b = 0; b < MB * NB; ++b) {
    tile_f32x16 block{};
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
        if (b == i * NB + j) block = acc[i][j];
    const int col = col0 + b % NB * 32;
    if (col >= n_valid) continue;
#pragma unroll 1
    for (int q = 0; q < 4; ++q) {
      float four[4] = {};
#pragma unroll
      for (int p = 0; p < 4; ++p)
        if (p == q) {
#pragma unroll
          for (int r = 0; r < 4; ++r) four[r] = block[p * 4 + r];
        }
      const int row = row0 + b / NB * 32 + q * 8;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (row + r < m_valid)
          store_element<BF16>(t.base, (row + r) * t.ld + col, finish_element<BF16>(e, four[r], m_base + row + r, n_base + col));
    }
  }
}
template <int MB, int NB>
__device__ __forceinline__ void store_linear_tile(const tile_f32x16 (&acc)[MB][NB], const LinearArgs& e, const TileTarget& t,
                                                  bool bf16, int row0, int col0, int m_valid, int n_valid, int64_t m_base,
                                                  int64_t n_base) {
  if (bf16) store_linear_tile_as<true, MB, NB>(acc, e, t, row0, col0, m_valid, n_valid, m_base, n_base);
  else store_linear_tile_as<false, MB, NB>(acc, e, t, row0, col0, m_valid, n_valid, m_base, n_base);
}

}  // namespace cleave
