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
#include <type_traits>

#include "bf16_round.h"
#include "kernels.h"
#include "tile_store.h"

namespace cleave {

// ---- activations -------------------------------------------------------------

// 1 / (1 + e^-x), to a few ulps of itself for every x: e^-x = 2^t e^(-x - t ln 2) with t = -x log2(e) rounded, whose second
// factor is 1 + rest (the rounding of t, up to 2^-18 at |x| = 87, would be an error of as much).  The exponential and the reciprocal are
// the hardware's (an ulp each); 2^t may overflow: the reciprocal of infinity is zero, and what is below 2^-126 may be.
__device__ __forceinline__ float sigmoid(float x) {
  constexpr float kLn2 = 0.693147180559945309f, kLn2Rest = -1.904654299957768e-9f;   // ln 2 - kLn2
  const float t = -1.44269504088896f * x;
  // (infinite x: no number, which the bounds take out)
  const float rest = __builtin_amdgcn_fmed3f(__builtin_fmaf(-t, kLn2Rest, __builtin_fmaf(-t, kLn2, -x)), -0.5f, 0.5f);
  return __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_amdgcn_exp2f(t), 1.0f + rest, 1.0f));
}
// gelu with tanh: z/2 (1 + tanh(u)) = z sigmoid(2 u), u = sqrt(2 / pi) (z + 0.044715 z^3).
// (2 u is an fp32 value: its rounding is 2^-23 |2 u| of a small sigmoid.)
constexpr float kGelu2 = 1.5957691216057308f;   // 2 sqrt(2 / pi)
constexpr float kGelu3 = 0.044715f;

__device__ __forceinline__ float relu(float z) { return z < 0.0f ? 0.0f : z; }   // NaN stays
__device__ __forceinline__ float gelu(float z) { return z * sigmoid(kGelu2 * z * (1.0f + kGelu3 * z * z)); }
__device__ __forceinline__ float silu(float z) { return z * sigmoid(z); }
__device__ __forceinline__ float relu_slope(float z) { return z > 0.0f ? 1.0f : 0.0f; }
// (where the sigmoid is 0 or 1 it is the slope, also for infinite z)
__device__ __forceinline__ float gelu_slope(float z) {
  const float p = sigmoid(kGelu2 * z * (1.0f + kGelu3 * z * z)), q = p * (1.0f - p);
  return q > 0.0f ? p + z * q * (kGelu2 * (1.0f + 3.0f * kGelu3 * z * z)) : p;
}
__device__ __forceinline__ float silu_slope(float z) {
  const float p = sigmoid(z), q = p * (1.0f - p);
  return q > 0.0f ? p + z * q : p;
}

// No epilogue: the kernels as cleave_execute and cleave_execute_assemble run them.
struct NoEpilogue {
  static constexpr bool kLinear = false, kGated = false;
};
struct LinearEpilogue : LinearArgs {
  static constexpr bool kLinear = true, kGated = false;
};

// The epilogue's arguments, read from the kernel's argument segment (`OFFSET` bytes in) where they are needed:
// held from the kernel's start on, they take scalar registers that the K loop then spills.
template <size_t OFFSET, typename Args = LinearArgs>
__device__ __forceinline__ Args late_linear_args() {
  static_assert(OFFSET % 8 == 0 && sizeof(Args) % 8 == 0, "whole words");
  typedef const __attribute__((address_space(4))) unsigned char* const_bytes;
  typedef const __attribute__((address_space(4))) uint64_t* const_words;
  const_bytes p = (const_bytes)__builtin_amdgcn_kernarg_segment_ptr() + OFFSET;
  asm volatile("" : "+s"(p));
  const_words src = (const_words)p;
  uint64_t words[sizeof(Args) / 8];
#pragma unroll
  for (size_t k = 0; k < sizeof(Args) / 8; ++k) words[k] = src[k];
  Args e;
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

// The epilogue of N elements of a row, but for the residual (SCALED: operands with scales).  t: the sums, then act(z) or the sums times the slope;
// z: the given z's, or (without `grad`) the new ones.  Branches are uniform and taken once for all N.
template <bool SCALED, int N>
__device__ __forceinline__ void finish(const LinearArgs& e, float (&t)[N], float (&z)[N], const float (&bias)[N],
                                       const float (&scale_b)[N], float scale_a) {
  if constexpr (SCALED) {
#pragma unroll
    for (int k = 0; k < N; ++k) t[k] = t[k] * scale_a * scale_b[k];
  }
  if (e.grad) {
    switch (e.act) {
      case CLEAVE_ACT_RELU:
#pragma unroll
        for (int k = 0; k < N; ++k) t[k] *= relu_slope(z[k]);
        break;
      case CLEAVE_ACT_GELU_TANH:
#pragma unroll
        for (int k = 0; k < N; ++k) t[k] *= gelu_slope(z[k]);
        break;
      case CLEAVE_ACT_SILU:
#pragma unroll
        for (int k = 0; k < N; ++k) t[k] *= silu_slope(z[k]);
        break;
      default: break;
    }
    return;
  }
  if (e.bias) {
#pragma unroll
    for (int k = 0; k < N; ++k) t[k] += bias[k];
  }
#pragma unroll
  for (int k = 0; k < N; ++k) z[k] = t[k];
  switch (e.act) {
    case CLEAVE_ACT_RELU:
#pragma unroll
      for (int k = 0; k < N; ++k) t[k] = relu(z[k]);
      break;
    case CLEAVE_ACT_GELU_TANH:
#pragma unroll
      for (int k = 0; k < N; ++k) t[k] = gelu(z[k]);
      break;
    case CLEAVE_ACT_SILU:
#pragma unroll
      for (int k = 0; k < N; ++k) t[k] = silu(z[k]);
      break;
    default: break;
  }
}

// Byte offset of the 16-byte piece `q` of row `row` in an image of Q pieces to a row: pieces are exchanged so that a
// write's rows and a read's pieces fall into different banks.
template <int Q>
__device__ __forceinline__ int image_piece(int row, int q) {
  constexpr int R = Q < 16 ? 16 / Q : 1;   // rows in a cycle of the banks
  return (row * Q + (q ^ ((row / R) & (Q < 16 ? Q - 1 : 15)))) * 16;
}
template <int ROWS, int COLS, int N>
__device__ __forceinline__ void read_image(const unsigned char* image, int row, int piece, float (&v)[N]) {
#pragma unroll
  for (int q = 0; q < N / 4; ++q) {
    const tile_f32x4 part = *reinterpret_cast<const tile_f32x4*>(image + image_piece<COLS / 4>(row, piece + q));
#pragma unroll
    for (int c = 0; c < 4; ++c) v[4 * q + c] = part[c];
  }
}

// ---- a wave's part of the output, image by image -----------------------------------

// At the end of a branch that picks accumulators by a number: different text in each keeps the compiler from merging them
// into one access through a computed address, for which the accumulators would live in memory.
#define CLEAVE_KEEP_APART(which) asm volatile("; part %0" ::"n"(which) : "memory")

// Walks `count` images, each ROWS x COLS sums that `write(i)` puts into the wave's piece of LDS: a lane takes sixteen output
// bytes' worth of a row at a time.  The images lie under each other (their columns are the same).
// LDS executes a wave's accesses in order and no other wave touches the image: no barrier.
// One turn per image, not unrolled: with all of them in line the code is beyond the instruction
// cache and its addresses spill.  The vector-memory counter retires loads and stores in order, so a load waits for
// the stores issued before it: what a turn reads is fetched AHEAD turns before, and nothing else is
// loaded between stores (the rows' scales come from registers, across lanes).  4096 x 11008 x 4096 bf16 with bias, gelu and the stored
// argument (180 MB out) takes 309-321 us (1.15 to 1.2 PFLOP/s), as long as with the bias alone.
//   row0, col0: the first image's place in the sub-tile, of which m_valid x n_valid elements exist.
//   out: element (0, 0) of the sub-tile, `ld` elements to a row; m_base, n_base: its place in the output.
template <bool BF16, bool INTERIOR, bool SCALED, int ROWS, int COLS, int AHEAD, typename Write>
__device__ __forceinline__ void emit_images(const LinearArgs& e, unsigned char* out_base, int64_t ld,
                                            const unsigned char* image, int count, int row0, int col0, int lane, int m_valid,
                                            int n_valid, int64_t m_base, int64_t n_base, Write write) {
  typedef Piece<BF16> P;
  constexpr int N = P::N;
  constexpr int EB = BF16 ? 2 : 4;
  constexpr int L = COLS / N;                  // lanes to a row
  constexpr int RR = 64 / L;                   // rows per read of the whole wave
  constexpr int K = ROWS / RR;                 // reads of the whole wave per image
  static_assert(ROWS % RR == 0 && AHEAD >= 1, "image");
  const int rrow = lane / L, rpiece = (lane % L) * (N / 4);
  int row = row0 + rrow;
  const int col = col0 + rpiece * 4;
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
  [[maybe_unused]] float scales = 0.0f;   // of row row0 + lane (SCALED: the images are 64 rows at most)
  if constexpr (SCALED) {
    read_columns(e.scale_b, scale_b);
    scales = e.scale_a[m_base + min(row0 + lane, m_valid - 1)];
  }
  const int64_t grow = m_base + row, gcol = n_base + col;
  unsigned char* out = out_base + (row * ld + col) * EB;
  unsigned char* zp = static_cast<unsigned char*>(e.preact) + (grow * e.ldz + gcol) * EB;   // this turn's
  const unsigned char* rp = static_cast<const unsigned char*>(e.residual) + (grow * e.ldr + gcol) * EB;
  const int64_t out_pitch = ld * EB, z_pitch = e.ldz * EB, r_pitch = e.ldr * EB;
  const bool reads_z = e.grad && e.preact, writes_z = !e.grad && e.preact;

  typename P::Raw z_raw[AHEAD + 1][K], r_raw[AHEAD + 1][K];
  const auto fetch = [&](int ahead, int d) {   // image i + ahead, into place d
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int r = ROWS * ahead + RR * k;
      if (!valid(row + r)) continue;
      if (reads_z) z_raw[d][k] = read(zp + r * z_pitch);
      if (e.residual) r_raw[d][k] = read(rp + r * r_pitch);
    }
  };
#pragma unroll
  for (int d = 0; d <= AHEAD; ++d)
#pragma unroll
    for (int k = 0; k < K; ++k) z_raw[d][k] = r_raw[d][k] = typename P::Raw{};
#pragma unroll
  for (int d = 0; d < AHEAD; ++d)
    if (d < count) fetch(d, d);
#pragma unroll 1
  for (int i = 0; i < count; ++i) {
    asm volatile("" ::: "memory");
    write(i);
    asm volatile("" ::: "memory");
    if (i + AHEAD < count) fetch(AHEAD, AHEAD);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int r = rrow + RR * k;
      P y, z;
      read_image<ROWS, COLS, N>(image, r, rpiece, y.v);
      float scale_a = 0.0f;
      if constexpr (SCALED) scale_a = __shfl(scales, ROWS * i + r);
      if (reads_z) z = P::of(z_raw[0][k]);
      finish<SCALED>(e, y.v, z.v, bias, scale_b, scale_a);
      if (e.residual) {
        const P residual = P::of(r_raw[0][k]);
#pragma unroll
        for (int c = 0; c < N; ++c) y.v[c] += residual.v[c];
      }
      if (valid(row + RR * k)) {
        if (writes_z) store(z, zp + RR * k * z_pitch);
        store(y, out + RR * k * out_pitch);
      }
    }
    asm volatile("" ::: "memory");
    row += ROWS;
    out += ROWS * out_pitch;
    zp += ROWS * z_pitch;
    rp += ROWS * r_pitch;
#pragma unroll
    for (int d = 0; d < AHEAD; ++d)
#pragma unroll
      for (int k = 0; k < K; ++k) {
        z_raw[d][k] = z_raw[d + 1][k];
        r_raw[d][k] = r_raw[d + 1][k];
      }
  }
}

// ---- stores of the direct kernel -------------------------------------------------

// store_rows (tile_store.h) with the epilogue: a row of 16 x 16 blocks is an image.
template <bool BF16, bool INTERIOR, bool SCALED, int AHEAD, int MB, int NB>
__device__ __forceinline__ void store_linear_rows(const tile_f32x4 (&acc)[MB][NB], const LinearArgs& e, const TileTarget& t,
                                                  unsigned char* image, int wave_row0, int wave_col0, int lane, int m_valid,
                                                  int n_valid, int64_t m_base, int64_t n_base) {
  static_assert(!SCALED || MB * 16 <= 64, "the rows' scales are held one to a lane");
  const int row = lane & 15, quad = lane >> 4;   // lane's row and which four columns of a block
  emit_images<BF16, INTERIOR, SCALED, 16, NB * 16, AHEAD>(
      e, t.base, t.ld, image, MB, wave_row0, wave_col0, lane, m_valid, n_valid, m_base, n_base, [&](int i) {
#pragma unroll
        for (int ii = 0; ii < MB; ++ii)
          if (ii == i) {
#pragma unroll
            for (int j = 0; j < NB; ++j)
              *reinterpret_cast<tile_f32x4*>(image + image_piece<NB * 4>(row, 4 * j + quad)) = acc[ii][j];
            CLEAVE_KEEP_APART(ii);
          }
      });
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
  if (e.scale_a) finish<true>(e, t, z, bias, scale_b, e.scale_a[row]);
  else finish<false>(e, t, z, bias, scale_b, 0.0f);
  if (e.residual) t[0] += load_element<BF16>(e.residual, row * e.ldr + col);
  if (!e.grad && e.preact) store_element<BF16>(e.preact, row * e.ldz + col, z[0]);
  return t[0];
}

// ---- stores of the general kernel ------------------------------------------------

// Bytes of a wave's image there: half a block of 32 x 32 sums (a whole one would spill at four waves to a SIMD).
constexpr int kTileImageBytes = 16 * 32 * 4;

// store_tile with the epilogue: half a block is an image; `image` is this wave's, no longer read as operands.
template <bool BF16, bool INTERIOR, int MB, int NB>
__device__ __forceinline__ void store_linear_tile_as(const tile_f32x16 (&acc)[MB][NB], const LinearArgs& e, const TileTarget& t,
                                                     unsigned char* image, int wave_row0, int wave_col0, int lane, int m_valid,
                                                     int n_valid, int64_t m_base, int64_t n_base) {
  const int l32 = lane & 31, lh = lane >> 5;   // lane has column l32 and rows 8 q + 4 lh + r
#pragma unroll 1
  for (int j = 0; j < NB; ++j) {
    emit_images<BF16, INTERIOR, false, 16, 32, 1>(
        e, t.base, t.ld, image, 2 * MB, wave_row0, wave_col0 + 32 * j, lane, m_valid, n_valid, m_base, n_base, [&](int i) {
#pragma unroll
          for (int ii = 0; ii < 2 * MB; ++ii)
#pragma unroll
            for (int jj = 0; jj < NB; ++jj)
              if (ii == i && jj == j) {
#pragma unroll
                for (int q = 0; q < 2; ++q)
#pragma unroll
                  for (int r = 0; r < 4; ++r)
                    *reinterpret_cast<float*>(image + image_piece<8>(8 * q + 4 * lh + r, l32 / 4) + 4 * (l32 % 4)) =
                        acc[ii / 2][jj][8 * (ii % 2) + 4 * q + r];
                CLEAVE_KEEP_APART(ii * NB + jj);
              }
        });
  }
}
template <int MB, int NB>
__device__ __forceinline__ void store_linear_tile(const tile_f32x16 (&acc)[MB][NB], const LinearArgs& e, const TileTarget& t,
                                                  bool bf16, unsigned char* image, int wave_row0, int wave_col0, int lane,
                                                  int m_valid, int n_valid, int64_t m_base, int64_t n_base, bool interior) {
  const auto as = [&](auto bf16_tag, auto interior_tag) {
    store_linear_tile_as<decltype(bf16_tag)::value, decltype(interior_tag)::value, MB, NB>(
        acc, e, t, image, wave_row0, wave_col0, lane, m_valid, n_valid, m_base, n_base);
  };
  constexpr std::true_type yes{};
  constexpr std::false_type no{};
  if (bf16) interior ? as(yes, yes) : as(yes, no);
  else interior ? as(no, yes) : as(no, no);
}

}  // namespace cleave
