// The gated product's way out, and its gradient's.
//
//   zg = sum_g sa sg + bg;  zu = sum_u sa su + bu;  y = act(zg) zu          (zg and zu kept if asked for)
//   p = sum;  dgate = p zu act'(zg);  dup = p act(zg)                        (zg and zu given)
//
// in fp32, each output rounded once.  sa, sg, su: scales of A's rows and of the weights' columns (8-bit operands).
//
// Bound by the products in front of them: neither sum is stored and read again, and A is read once.  4096 rows, both weights 4096 x 11008,
// bf16, us: K x N 591-606 (1.22 to 1.25 PFLOP/s; 8192^3 of the library: 1.22 to 1.24), e4m3 572-590; the gradient's product 4096 x 11008 x 4096
// K x N 337, N x K 368 (1.0 PFLOP/s, with 360 MB of zg, zu, dgate and dup on the way).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "linear_epilogue.h"

namespace cleave {

// Two operands B: of a tile's columns the first half of every wave's are gate's, the second half up's.
struct GatedEpilogue : GatedArgs {
  static constexpr bool kLinear = true, kGated = true;
};
// The gradient: one operand B, two outputs.
struct GatedGradEpilogue : GatedArgs {
  static constexpr bool kLinear = true, kGated = false;
};

// act(z) and act'(z); one sigmoid for both.
struct ActAndSlope {
  float value, slope;
};
__device__ __forceinline__ ActAndSlope gelu_both(float z) {
  const float p = sigmoid(kGelu2 * z * (1.0f + kGelu3 * z * z)), q = p * (1.0f - p);
  return {z * p, q > 0.0f ? p + z * q * (kGelu2 * (1.0f + 3.0f * kGelu3 * z * z)) : p};
}
__device__ __forceinline__ ActAndSlope silu_both(float z) {
  const float p = sigmoid(z), q = p * (1.0f - p);
  return {z * p, q > 0.0f ? p + z * q : p};
}

// N elements: g and u become the arguments zg and zu, the product is returned in y.  Branches are uniform and taken once for all N.
template <bool SCALED, int N>
__device__ __forceinline__ void finish_gated(int act, float (&g)[N], float (&u)[N], float (&y)[N], const float (&bias_g)[N],
                                             const float (&bias_u)[N], const float (&scale_g)[N], const float (&scale_u)[N],
                                             float scale_a) {
#pragma unroll
  for (int k = 0; k < N; ++k) {
    if constexpr (SCALED) {
      g[k] = g[k] * scale_a * scale_g[k];
      u[k] = u[k] * scale_a * scale_u[k];
    }
    g[k] += bias_g[k];
    u[k] += bias_u[k];
  }
  switch (act) {
    case CLEAVE_ACT_RELU:
#pragma unroll
      for (int k = 0; k < N; ++k) y[k] = relu(g[k]) * u[k];
      break;
    case CLEAVE_ACT_GELU_TANH:
#pragma unroll
      for (int k = 0; k < N; ++k) y[k] = gelu(g[k]) * u[k];
      break;
    case CLEAVE_ACT_SILU:
#pragma unroll
      for (int k = 0; k < N; ++k) y[k] = silu(g[k]) * u[k];
      break;
    default:
#pragma unroll
      for (int k = 0; k < N; ++k) y[k] = g[k] * u[k];
      break;
  }
}
// p becomes dgate, zu dup.
template <int N>
__device__ __forceinline__ void finish_gated_grad(int act, float (&p)[N], const float (&zg)[N], float (&zu)[N]) {
  const auto put = [&](int k, ActAndSlope a) {
    const float dgate = p[k] * zu[k] * a.slope;
    zu[k] = p[k] * a.value;
    p[k] = dgate;
  };
  switch (act) {
    case CLEAVE_ACT_RELU:
#pragma unroll
      for (int k = 0; k < N; ++k) put(k, {relu(zg[k]), relu_slope(zg[k])});
      break;
    case CLEAVE_ACT_GELU_TANH:
#pragma unroll
      for (int k = 0; k < N; ++k) put(k, gelu_both(zg[k]));
      break;
    case CLEAVE_ACT_SILU:
#pragma unroll
      for (int k = 0; k < N; ++k) put(k, silu_both(zg[k]));
      break;
    default:
#pragma unroll
      for (int k = 0; k < N; ++k) put(k, {zg[k], 1.0f});
      break;
  }
}

// N floats of a vector from column `at` on; the first `n` only.
template <int N>
__device__ __forceinline__ void read_columns(const float* from, int64_t at, int n, float (&to)[N]) {
  typedef float quad __attribute__((ext_vector_type(4), aligned(4)));
  if (n >= N) {
#pragma unroll
    for (int q = 0; q < N / 4; ++q) {
      const quad b = reinterpret_cast<const quad*>(from + at)[q];
#pragma unroll
      for (int c = 0; c < 4; ++c) to[4 * q + c] = b[c];
    }
  } else {
#pragma unroll
    for (int c = 0; c < N; ++c)
      if (c < n) to[c] = from[at + c];
  }
}

// ---- stores of the direct kernel -------------------------------------------------

// Stores one lane issues for a full tile of MB x NB blocks, at least: what the kernel's waits may count on.
template <bool BF16, int MB, int NB>
constexpr int gated_stores() {
  constexpr int lanes = NB * 8 / Piece<BF16>::N;   // to a row
  return MB * (lanes >= 4 ? lanes / 4 : 1);
}

// The product of a wave's accumulators: a row of 16 x 16 blocks is an image (store_linear_rows), whose first half of columns
// is gate's and second half up's, so that a lane has the same columns of both.
template <bool BF16, bool INTERIOR, bool SCALED, int MB, int NB>
__device__ __forceinline__ void store_gated_rows(const tile_f32x4 (&acc)[MB][NB], const GatedArgs& e, const TileTarget& t,
                                                 unsigned char* image, int wave_row0, int wave_col0, int lane, int m_valid,
                                                 int n_valid, int64_t m_base, int64_t n_base) {
  static_assert(!SCALED || MB * 16 <= 64, "the rows' scales are held one to a lane");
  typedef Piece<BF16> P;
  constexpr int N = P::N, EB = BF16 ? 2 : 4, COLS = NB * 8;
  constexpr int L = COLS / N;                  // lanes to a row
  constexpr int RR = 64 / L;                   // rows per read of the whole wave (more than there are: the rest is idle)
  constexpr int K = RR < 16 ? 16 / RR : 1;
  const int wrow = lane & 15, quad = lane >> 4;
  const int rrow = lane / L, rpiece = (lane % L) * (N / 4);
  const int col = wave_col0 + rpiece * 4;
  const int cols = INTERIOR ? N : min(N, n_valid - col);   // of this lane's that there are
  float bias_g[N] = {}, bias_u[N] = {}, scale_g[N] = {}, scale_u[N] = {};
  if (e.bias_gate) read_columns<N>(e.bias_gate, n_base + col, cols, bias_g);
  if (e.bias_up) read_columns<N>(e.bias_up, n_base + col, cols, bias_u);
  [[maybe_unused]] float scales = 0.0f;   // of row wave_row0 + lane
  if constexpr (SCALED) {
    read_columns<N>(e.scale_gate, n_base + col, cols, scale_g);
    read_columns<N>(e.scale_up, n_base + col, cols, scale_u);
    scales = e.scale_a[m_base + min(wave_row0 + lane, m_valid - 1)];
  }
  const auto store = [&](const P& x, unsigned char* p) {
    if (INTERIOR || cols == N) x.store(p);
    else x.store(p, cols);
  };
  const int64_t row0 = wave_row0 + rrow;
  unsigned char* out = t.base + (row0 * t.ld + col) * EB;
  unsigned char* gp = static_cast<unsigned char*>(e.gate) + ((m_base + row0) * e.ld_gate + n_base + col) * EB;
  unsigned char* up = static_cast<unsigned char*>(e.up) + ((m_base + row0) * e.ld_up + n_base + col) * EB;
  // one turn per row of blocks, not unrolled (emit_images)
#pragma unroll 1
  for (int i = 0; i < MB; ++i) {
    asm volatile("" ::: "memory");
#pragma unroll
    for (int ii = 0; ii < MB; ++ii)
      if (ii == i) {
#pragma unroll
        for (int j = 0; j < NB; ++j)
          *reinterpret_cast<tile_f32x4*>(image + image_piece<NB * 4>(wrow, 4 * j + quad)) = acc[ii][j];
        CLEAVE_KEEP_APART(ii);
      }
    asm volatile("" ::: "memory");
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int r = rrow + RR * k;
      if (RR > 16 && r >= 16) continue;
      P g, u, y;
      read_image<16, NB * 16, N>(image, r, rpiece, g.v);
      read_image<16, NB * 16, N>(image, r, rpiece + COLS / 4, u.v);
      float scale_a = 0.0f;
      if constexpr (SCALED) scale_a = __shfl(scales, 16 * i + r);
      finish_gated<SCALED>(static_cast<int>(e.act), g.v, u.v, y.v, bias_g, bias_u, scale_g, scale_u, scale_a);
      if (INTERIOR || (wave_row0 + 16 * i + r < m_valid && cols > 0)) {
        if (e.gate) store(g, gp + RR * k * e.ld_gate * EB);
        if (e.up) store(u, up + RR * k * e.ld_up * EB);
        store(y, out + RR * k * t.ld * EB);
      }
    }
    asm volatile("" ::: "memory");
    out += 16 * t.ld * EB;
    gp += 16 * e.ld_gate * EB;
    up += 16 * e.ld_up * EB;
  }
}

// The gradient.  A turn takes the rows that the wave reads at a time (half an image of bf16), its arguments are fetched
// AHEAD turns before (emit_images).
constexpr int kGradAhead = 1;
template <bool BF16, bool INTERIOR, int AHEAD, int MB, int NB>
__device__ __forceinline__ void store_gated_grad_rows(const tile_f32x4 (&acc)[MB][NB], const GatedArgs& e, const TileTarget& t,
                                                      unsigned char* image, int wave_row0, int wave_col0, int lane, int m_valid,
                                                      int n_valid, int64_t m_base, int64_t n_base) {
  typedef Piece<BF16> P;
  constexpr int N = P::N, EB = BF16 ? 2 : 4, COLS = NB * 16;
  constexpr int L = COLS / N, RR = 64 / L, K = 16 / RR;   // lanes to a row, rows of a turn, turns of an image
  static_assert(RR <= 16, "image");
  const int wrow = lane & 15, quad = lane >> 4;
  const int rrow = lane / L, rpiece = (lane % L) * (N / 4);
  int row = wave_row0 + rrow;
  const int col = wave_col0 + rpiece * 4;
  const int cols = INTERIOR ? N : min(N, n_valid - col);
  const auto valid = [&](int r) { return INTERIOR || (r < m_valid && cols > 0); };
  const auto read = [&](const unsigned char* p) { return INTERIOR || cols == N ? P::read(p) : P::read(p, cols); };
  const auto store = [&](const P& x, unsigned char* p) {
    if (INTERIOR || cols == N) x.store(p);
    else x.store(p, cols);
  };
  const int64_t grow = m_base + row, gcol = n_base + col;
  unsigned char* out = t.base + (row * t.ld + col) * EB;
  unsigned char* second = static_cast<unsigned char*>(e.second) + (grow * e.ld_second + gcol) * EB;
  const unsigned char* gp = static_cast<const unsigned char*>(e.gate) + (grow * e.ld_gate + gcol) * EB;
  const unsigned char* up = static_cast<const unsigned char*>(e.up) + (grow * e.ld_up + gcol) * EB;
  const int64_t out_pitch = t.ld * EB, second_pitch = e.ld_second * EB, g_pitch = e.ld_gate * EB, u_pitch = e.ld_up * EB;
  typename P::Raw g_raw[AHEAD + 1], u_raw[AHEAD + 1];
  const auto fetch = [&](int ahead, int d) {   // of the turn that far on, into place d
    g_raw[d] = u_raw[d] = typename P::Raw{};
    if (!valid(row + RR * ahead)) return;
    g_raw[d] = read(gp + RR * ahead * g_pitch);
    u_raw[d] = read(up + RR * ahead * u_pitch);
  };
#pragma unroll
  for (int d = 0; d < AHEAD; ++d)
    if (d < MB * K) fetch(d, d);
#pragma unroll 1
  for (int i = 0; i < MB * K; ++i) {
    asm volatile("" ::: "memory");
#pragma unroll
    for (int ii = 0; ii < MB; ++ii)
      if (K * ii == i) {
#pragma unroll
        for (int j = 0; j < NB; ++j)
          *reinterpret_cast<tile_f32x4*>(image + image_piece<NB * 4>(wrow, 4 * j + quad)) = acc[ii][j];
        CLEAVE_KEEP_APART(ii);
      }
    asm volatile("" ::: "memory");
    if (i + AHEAD < MB * K) fetch(AHEAD, AHEAD);
    P p;
    read_image<16, COLS, N>(image, rrow + RR * (i % K), rpiece, p.v);
    const P zg = P::of(g_raw[0]);
    P zu = P::of(u_raw[0]);
    finish_gated_grad(static_cast<int>(e.act), p.v, zg.v, zu.v);
    if (valid(row)) {
      store(zu, second);
      store(p, out);
    }
    asm volatile("" ::: "memory");
    row += RR;
    out += RR * out_pitch;
    second += RR * second_pitch;
    gp += RR * g_pitch;
    up += RR * u_pitch;
#pragma unroll
    for (int d = 0; d < AHEAD; ++d) {
      g_raw[d] = g_raw[d + 1];
      u_raw[d] = u_raw[d + 1];
    }
  }
}

// ---- single elements -------------------------------------------------------------

// Element (row, col) of the gated product, from its sums: what is stored.
template <bool BF16>
__device__ __forceinline__ float finish_gated_element(const GatedArgs& e, float gate, float up, int64_t row, int64_t col) {
  float g[1] = {gate}, u[1] = {up}, y[1];
  const float bg[1] = {e.bias_gate ? e.bias_gate[col] : 0.0f}, bu[1] = {e.bias_up ? e.bias_up[col] : 0.0f};
  const float sg[1] = {e.scale_gate ? e.scale_gate[col] : 0.0f}, su[1] = {e.scale_up ? e.scale_up[col] : 0.0f};
  if (e.scale_a) finish_gated<true>(static_cast<int>(e.act), g, u, y, bg, bu, sg, su, e.scale_a[row]);
  else finish_gated<false>(static_cast<int>(e.act), g, u, y, bg, bu, sg, su, 0.0f);
  if (e.gate) store_element<BF16>(e.gate, row * e.ld_gate + col, g[0]);
  if (e.up) store_element<BF16>(e.up, row * e.ld_up + col, u[0]);
  return y[0];
}

}  // namespace cleave
