// Elements of a row of fp32 or bf16 values, sixteen bytes at a time, at any alignment of the elements.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "bf16_round.h"
#include "fp8_round.h"

namespace cleave {

struct Bf16 {
  uint16_t bits;
};

// N neighbouring elements in sixteen bytes.  `left`: how many there are from p on; what is not there reads as zero and is
// not written.  (A row's last group is the only one that is not whole.)  read() and unpack() are apart so that several reads are
// on their way before the first is waited for.
typedef uint32_t Raw16 __attribute__((ext_vector_type(4)));

template <typename T>
struct Group16;

template <>
struct Group16<float> {
  static constexpr int N = 4;
  typedef uint32_t Any __attribute__((ext_vector_type(4), aligned(4)));
  static __device__ __forceinline__ Raw16 read(const float* p, int left) {
    if (left >= N) return *reinterpret_cast<const Any*>(p);
    Raw16 w{};
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < left) w[e] = reinterpret_cast<const uint32_t*>(p)[e];
    return w;
  }
  static __device__ __forceinline__ void unpack(Raw16 w, float (&out)[N]) {
    typedef float Floats __attribute__((ext_vector_type(4)));
    const Floats v = __builtin_bit_cast(Floats, w);
#pragma unroll
    for (int e = 0; e < N; ++e) out[e] = v[e];
  }
  static __device__ __forceinline__ void store_streamed(float* p, int left, const float (&in)[N]) {
    typedef float FloatsAny __attribute__((ext_vector_type(4), aligned(4)));
    if (left >= N) __builtin_nontemporal_store(FloatsAny{in[0], in[1], in[2], in[3]}, reinterpret_cast<FloatsAny*>(p));
    else store(p, left, in);
  }
  static __device__ __forceinline__ void store(float* p, int left, const float (&in)[N]) {
    typedef float FloatsAny __attribute__((ext_vector_type(4), aligned(4)));
    if (left >= N) {
      *reinterpret_cast<FloatsAny*>(p) = FloatsAny{in[0], in[1], in[2], in[3]};
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e < left) p[e] = in[e];
    }
  }
};

template <>
struct Group16<Bf16> {
  static constexpr int N = 8;
  typedef uint32_t Any __attribute__((ext_vector_type(4), aligned(2)));
  static __device__ __forceinline__ Raw16 read(const Bf16* p, int left) {
    if (left >= N) return *reinterpret_cast<const Any*>(p);
    Raw16 w{};
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < left) w[e / 2] |= static_cast<uint32_t>(p[e].bits) << (16 * (e % 2));
    return w;
  }
  static __device__ __forceinline__ void unpack(Raw16 w, float (&out)[N]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      out[2 * q] = __builtin_bit_cast(float, w[q] << 16);
      out[2 * q + 1] = __builtin_bit_cast(float, w[q] & 0xffff0000u);
    }
  }
  // Non-temporal.
  static __device__ __forceinline__ void store_streamed(Bf16* p, int left, const float (&in)[N]) {
    if (left >= N)
      __builtin_nontemporal_store(
          Any{pack_bf16(in[0], in[1]), pack_bf16(in[2], in[3]), pack_bf16(in[4], in[5]), pack_bf16(in[6], in[7])},
          reinterpret_cast<Any*>(p));
    else
      store(p, left, in);
  }
  static __device__ __forceinline__ void store(Bf16* p, int left, const float (&in)[N]) {
    if (left >= N) {
      *reinterpret_cast<Any*>(p) =
          Any{pack_bf16(in[0], in[1]), pack_bf16(in[2], in[3]), pack_bf16(in[4], in[5]), pack_bf16(in[6], in[7])};
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e < left) p[e].bits = to_bf16_bits(in[e]);
    }
  }
};

// Groups of a row of eight bf16 and more, without a branch: a last group that is not whole is read so that it ends with the row, what lies
// behind the row as that one; settle() then moves what there is of it to the front, zeros behind.
__device__ __forceinline__ Raw16 read_ending(const Bf16* p, int left) {
  typedef Group16<Bf16> G;
  return G::read(p + min(left - G::N, 0), G::N);
}
__device__ __forceinline__ Raw16 settle(Raw16 w, int left) {
  constexpr int N = Group16<Bf16>::N;
  if (left >= N) return w;
  const int off = N - max(left, 0);
  if (off % 2 != 0) w = Raw16{w[0] >> 16 | w[1] << 16, w[1] >> 16 | w[2] << 16, w[2] >> 16 | w[3] << 16, w[3] >> 16};
  if (off / 2 & 1) w = Raw16{w[1], w[2], w[3], 0};
  if (off / 2 & 2) w = Raw16{w[2], w[3], 0, 0};
  if (off == N) w = Raw16{};
  return w;
}

// Single elements.
__device__ __forceinline__ float element(const float* p) { return *p; }
__device__ __forceinline__ float element(const Bf16* p) {
  return __builtin_bit_cast(float, static_cast<uint32_t>(p->bits) << 16);
}
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(Bf16* p, float x) { p->bits = to_bf16_bits(x); }

// A row per group of NT threads, which holds up to NT * V * N elements of it (N in sixteen bytes); a wave (NT = 64)
// has its row to itself, four rows to a workgroup, and eight or sixteen lanes a narrow one.
template <int NT>
struct RowGroup {
  static constexpr int kThreads = NT <= 64 ? 256 : NT;
  static constexpr int kRows = kThreads / NT;
  static constexpr int kWaves = NT < 64 ? 1 : NT / 64;
};

// N floats beside a group of either type.
template <int N>
struct Floats16 {
  Raw16 raw[N / 4];
  __device__ __forceinline__ void read(const float* p, int left) {
#pragma unroll
    for (int q = 0; q < N / 4; ++q) raw[q] = Group16<float>::read(p + 4 * q, left - 4 * q);
  }
  __device__ __forceinline__ void unpack(float (&out)[N]) const {
#pragma unroll
    for (int q = 0; q < N / 4; ++q) {
      float four[4];
      Group16<float>::unpack(raw[q], four);
#pragma unroll
      for (int e = 0; e < 4; ++e) out[4 * q + e] = four[e];
    }
  }
};
template <int N>
__device__ __forceinline__ void store_floats(float* p, int left, const float (&in)[N]) {
#pragma unroll
  for (int q = 0; q < N / 4; ++q) {
    const float four[4] = {in[4 * q], in[4 * q + 1], in[4 * q + 2], in[4 * q + 3]};
    Group16<float>::store(p + 4 * q, left - 4 * q, four);
  }
}
// N e4m3 values.
template <int N>
__device__ __forceinline__ void store_e4m3(uint8_t* p, int left, const float (&in)[N]) {
  typedef uint32_t Words __attribute__((ext_vector_type(N / 4)));
  typedef uint32_t WordsAny __attribute__((ext_vector_type(N / 4), aligned(1)));
  if (left >= N) {
    Words w;
#pragma unroll
    for (int q = 0; q < N / 4; ++q) w[q] = pack_e4m3(in[4 * q], in[4 * q + 1], in[4 * q + 2], in[4 * q + 3]);
    *reinterpret_cast<WordsAny*>(p) = w;
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < left) p[e] = static_cast<uint8_t>(pack_e4m3(in[e], in[e]));
  }
}

}  // namespace cleave
