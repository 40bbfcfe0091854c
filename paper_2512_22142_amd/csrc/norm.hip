// Root-mean-square norm of a residual stream, its gradient, and sums of columns
// (the non-GEMM operators that the paper keeps on the parameter server, Sec. 4.1).
//
//   h = x + r;  i = 1 / sqrt(mean(h^2) + eps);  y = h i w
// over the columns of each row, in fp32 from the unrounded h; y in x's type or, for a product
// with 8-bit operands, as e4m3 with the row's scale s = max|y| / 448.
//
// Gradient, with the stored h and i, g = dy w and xhat = h i:
//   dx = i (g - xhat mean(g xhat)) + dsum;   dw = sum over rows of dy xhat
//
// Bound by memory: every row is read once and kept in registers between its statistics, the
// scaling and the rounding.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "fp8_round.h"
#include "operators.h"
#include "row_access.h"
#include "wave_reduce.h"

namespace cleave {

namespace {

// e4m3 values of VEC elements, one scale.
template <int VEC>
__device__ __forceinline__ void store_e4m3(uint8_t* p, const float (&y)[VEC]) {
  if constexpr (VEC == 1) {
    *p = static_cast<uint8_t>(pack_e4m3(y[0], y[0]));
  } else {
#pragma unroll
    for (int q = 0; q < VEC / 4; ++q)
      reinterpret_cast<uint32_t*>(p)[q] = pack_e4m3(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
  }
}

// A row per group of NT threads, which holds up to NT * V * VEC elements of it; a wave (NT = 64)
// has its row to itself, four rows to a workgroup.
template <int NT>
struct RowGroup {
  static constexpr int kThreads = NT == 64 ? 256 : NT;
  static constexpr int kRows = kThreads / NT;
  static constexpr int kWaves = NT / 64;
};

template <typename T, int VEC, int NT, int V, bool E4M3>
__global__ __launch_bounds__(RowGroup<NT>::kThreads) void rms_norm_kernel(NormArgs args) {
  constexpr int NW = RowGroup<NT>::kWaves;
  __shared__ float slots[2][NW];
  const int t = threadIdx.x % NT;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * RowGroup<NT>::kRows + threadIdx.x / NT;
  if (row >= args.rows) return;   // whole waves, and with several waves to a row whole workgroups
  const T* x = static_cast<const T*>(args.x) + row * args.ldx;
  const T* r = static_cast<const T*>(args.residual) + (args.residual ? row * args.ldr : 0);
  T* sum_out = static_cast<T*>(args.sum_out) + (args.sum_out ? row * args.lds : 0);
  const int cols = static_cast<int>(args.cols);

  float h[V][VEC], w[V][VEC];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int c = (j * NT + t) * VEC;
    if (c < cols) load_elements<VEC>(x + c, h[j]);
    else
#pragma unroll
      for (int e = 0; e < VEC; ++e) h[j][e] = 0.0f;
  }
  if (args.residual) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = (j * NT + t) * VEC;
      float add[VEC] = {};
      if (c < cols) load_elements<VEC>(r + c, add);
#pragma unroll
      for (int e = 0; e < VEC; ++e) h[j][e] += add[e];
    }
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int c = (j * NT + t) * VEC;
#pragma unroll
    for (int e = 0; e < VEC; ++e) w[j][e] = 0.0f;
    if (c < cols) load_elements<VEC>(args.weight + c, w[j]);
  }
  float squares = 0.0f;
#pragma unroll
  for (int j = 0; j < V; ++j)
#pragma unroll
    for (int e = 0; e < VEC; ++e) squares += h[j][e] * h[j][e];
  if (args.sum_out) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = (j * NT + t) * VEC;
      if (c < cols) store_elements<VEC>(sum_out + c, h[j]);
    }
  }
  squares = group_sum<NW>(squares, slots[0]);
  const float inv = 1.0f / __builtin_sqrtf(squares / static_cast<float>(cols) + args.eps);
  if (args.inv_rms && t == 0) args.inv_rms[row] = inv;
#pragma unroll
  for (int j = 0; j < V; ++j)
#pragma unroll
    for (int e = 0; e < VEC; ++e) h[j][e] = h[j][e] * inv * w[j][e];
  if constexpr (E4M3) {
    float most = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int e = 0; e < VEC; ++e) most = nan_max(most, __builtin_fabsf(h[j][e]));
    const BlockScale s = block_scale(group_nan_max<NW>(most, slots[1]));
    if (t == 0) args.scales[row] = s.scale;
    uint8_t* y = static_cast<uint8_t*>(args.y) + row * args.ldy;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = (j * NT + t) * VEC;
#pragma unroll
      for (int e = 0; e < VEC; ++e) h[j][e] *= s.inverse;
      if (c < cols) store_e4m3<VEC>(y + c, h[j]);
    }
  } else {
    T* y = static_cast<T*>(args.y) + row * args.ldy;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = (j * NT + t) * VEC;
      if (c < cols) store_elements<VEC>(y + c, h[j]);
    }
  }
}

// Rows that no group's registers hold: read again for each use (from the caches).
constexpr int kLongThreads = 1024;
template <typename T, bool E4M3>
__global__ __launch_bounds__(kLongThreads) void rms_norm_long_kernel(NormArgs args) {
  constexpr int NW = kLongThreads / 64;
  __shared__ float slots[2][NW];
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(args.x) + row * args.ldx;
  const T* r = static_cast<const T*>(args.residual) + (args.residual ? row * args.ldr : 0);
  const auto at = [&](int64_t c) {
    float h[1];
    load_elements<1>(x + c, h);
    if (args.residual) {
      float add[1];
      load_elements<1>(r + c, add);
      h[0] += add[0];
    }
    return h[0];
  };
  float squares = 0.0f;
  for (int64_t c = threadIdx.x; c < args.cols; c += kLongThreads) {
    const float h = at(c);
    squares += h * h;
  }
  squares = group_sum<NW>(squares, slots[0]);
  const float inv = 1.0f / __builtin_sqrtf(squares / static_cast<float>(args.cols) + args.eps);
  if (args.inv_rms && threadIdx.x == 0) args.inv_rms[row] = inv;
  BlockScale s{1.0f, 1.0f};
  if constexpr (E4M3) {
    float most = 0.0f;
    for (int64_t c = threadIdx.x; c < args.cols; c += kLongThreads)
      most = nan_max(most, __builtin_fabsf(at(c) * inv * args.weight[c]));
    s = block_scale(group_nan_max<NW>(most, slots[1]));
    if (threadIdx.x == 0) args.scales[row] = s.scale;
  }
  // (an element is read, then written, by one thread: y or the sum may take x's or r's place)
  for (int64_t c = threadIdx.x; c < args.cols; c += kLongThreads) {
    const float h[1] = {at(c)};
    float y[1] = {h[0] * inv * args.weight[c]};
    if (args.sum_out) store_elements<1>(static_cast<T*>(args.sum_out) + row * args.lds + c, h);
    if constexpr (E4M3) {
      y[0] *= s.inverse;
      store_e4m3<1>(static_cast<uint8_t*>(args.y) + row * args.ldy + c, y);
    } else {
      store_elements<1>(static_cast<T*>(args.y) + row * args.ldy + c, y);
    }
  }
}

template <typename T, int VEC, int NT, int V>
hipError_t launch_norm(const NormArgs& args, hipStream_t stream) {
  constexpr int kRows = RowGroup<NT>::kRows;
  const dim3 g(static_cast<uint32_t>((args.rows + kRows - 1) / kRows)), b(RowGroup<NT>::kThreads);
  if (args.scales) hipLaunchKernelGGL((rms_norm_kernel<T, VEC, NT, V, true>), g, b, 0, stream, args);
  else hipLaunchKernelGGL((rms_norm_kernel<T, VEC, NT, V, false>), g, b, 0, stream, args);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_norm_of(const NormArgs& args, bool vec, hipStream_t stream) {
  constexpr int E = Vec16<T>::N;
  const int64_t n = args.cols;
  if (vec) {
    if (n <= 64 * E) return launch_norm<T, E, 64, 1>(args, stream);
    if (n <= 256 * E) return launch_norm<T, E, 256, 1>(args, stream);
    if (n <= 512 * E) return launch_norm<T, E, 256, 2>(args, stream);
    if (n <= 1024 * E) return launch_norm<T, E, 512, 2>(args, stream);
    if (n <= 2048 * E) return launch_norm<T, E, 1024, 2>(args, stream);
    if (n <= 4096 * E) return launch_norm<T, E, 1024, 4>(args, stream);
  } else {
    if (n <= 512) return launch_norm<T, 1, 64, 8>(args, stream);
    if (n <= 2048) return launch_norm<T, 1, 256, 8>(args, stream);
    if (n <= 8192) return launch_norm<T, 1, 1024, 8>(args, stream);
    if (n <= 16384) return launch_norm<T, 1, 1024, 16>(args, stream);
  }
  const dim3 g(static_cast<uint32_t>(args.rows)), b(kLongThreads);
  if (args.scales) hipLaunchKernelGGL((rms_norm_long_kernel<T, true>), g, b, 0, stream, args);
  else hipLaunchKernelGGL((rms_norm_long_kernel<T, false>), g, b, 0, stream, args);
  return hipGetLastError();
}

// ---- gradient ------------------------------------------------------------------

// Group `first` of the launch takes rows first, first + step, ... and holds its part of the weight's
// gradient in registers until the last of them: one row of partial sums for each group.
template <typename T, int VEC, int NT, int V>
__global__ __launch_bounds__(RowGroup<NT>::kThreads) void rms_norm_backward_kernel(NormBackwardArgs args, int groups) {
  constexpr int NW = RowGroup<NT>::kWaves;
  __shared__ float slots[2][NW];
  const int t = threadIdx.x % NT;
  const int group = blockIdx.x * RowGroup<NT>::kRows + threadIdx.x / NT;
  if (group >= groups) return;
  const int cols = static_cast<int>(args.cols);
  float dw[V][VEC] = {}, w[V][VEC] = {};
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int c = (j * NT + t) * VEC;
    if (c < cols) load_elements<VEC>(args.weight + c, w[j]);
  }
  int turn = 0;
  for (int64_t row = group; row < args.rows; row += groups, turn ^= 1) {
    const T* dy = static_cast<const T*>(args.dy) + row * args.lddy;
    const T* h = static_cast<const T*>(args.h) + row * args.ldh;
    const float inv = args.inv_rms[row];
    float g[V][VEC] = {}, xhat[V][VEC] = {}, add[V][VEC] = {};
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = (j * NT + t) * VEC;
      if (c < cols) {
        load_elements<VEC>(dy + c, g[j]);
        load_elements<VEC>(h + c, xhat[j]);
      }
    }
    if (args.dsum) {
      const T* dsum = static_cast<const T*>(args.dsum) + row * args.ldds;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int c = (j * NT + t) * VEC;
        if (c < cols) load_elements<VEC>(dsum + c, add[j]);
      }
    }
    float dot = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        xhat[j][e] *= inv;
        dw[j][e] += g[j][e] * xhat[j][e];
        g[j][e] *= w[j][e];
        dot += g[j][e] * xhat[j][e];
      }
    // (the slots of the row before last are free: every wave has passed the barrier of the last one)
    const float mean = group_sum<NW>(dot, slots[turn]) / static_cast<float>(cols);
    T* dx = static_cast<T*>(args.dx) + row * args.lddx;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = (j * NT + t) * VEC;
#pragma unroll
      for (int e = 0; e < VEC; ++e) g[j][e] = (g[j][e] - xhat[j][e] * mean) * inv + add[j][e];
      if (c < cols) store_elements<VEC>(dx + c, g[j]);
    }
  }
  float* out = args.partials + static_cast<int64_t>(group) * args.cols;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int c = (j * NT + t) * VEC;
    if (c < cols) {
      if constexpr (VEC == 1) out[c] = dw[j][0];
      else store_elements<VEC>(out + c, dw[j]);
    }
  }
}

// Rows that no group's registers hold: the partial sums are kept in the group's row of them.
template <typename T>
__global__ __launch_bounds__(kLongThreads) void rms_norm_backward_long_kernel(NormBackwardArgs args, int groups) {
  constexpr int NW = kLongThreads / 64;
  __shared__ float slots[2][NW];
  float* out = args.partials + static_cast<int64_t>(blockIdx.x) * args.cols;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < args.rows; row += groups, turn ^= 1) {
    const T* dy = static_cast<const T*>(args.dy) + row * args.lddy;
    const T* h = static_cast<const T*>(args.h) + row * args.ldh;
    const float inv = args.inv_rms[row];
    const bool fresh = row == blockIdx.x;
    float dot = 0.0f;
    for (int64_t c = threadIdx.x; c < args.cols; c += kLongThreads) {
      float g[1], x[1];
      load_elements<1>(dy + c, g);
      load_elements<1>(h + c, x);
      x[0] *= inv;
      out[c] = (fresh ? 0.0f : out[c]) + g[0] * x[0];
      dot += g[0] * args.weight[c] * x[0];
    }
    const float mean = group_sum<NW>(dot, slots[turn]) / static_cast<float>(args.cols);
    for (int64_t c = threadIdx.x; c < args.cols; c += kLongThreads) {
      float g[1], x[1], add[1] = {0.0f};
      load_elements<1>(dy + c, g);
      load_elements<1>(h + c, x);
      if (args.dsum) load_elements<1>(static_cast<const T*>(args.dsum) + row * args.ldds + c, add);
      g[0] = (g[0] * args.weight[c] - x[0] * inv * mean) * inv + add[0];
      store_elements<1>(static_cast<T*>(args.dx) + row * args.lddx + c, g);
    }
  }
}

template <typename T, int VEC, int NT, int V>
hipError_t launch_backward(const NormBackwardArgs& args, int groups, hipStream_t stream) {
  constexpr int kRows = RowGroup<NT>::kRows;
  hipLaunchKernelGGL((rms_norm_backward_kernel<T, VEC, NT, V>), dim3((groups + kRows - 1) / kRows),
                     dim3(RowGroup<NT>::kThreads), 0, stream, args, groups);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_backward_of(const NormBackwardArgs& args, bool vec, int groups, hipStream_t stream) {
  constexpr int E = Vec16<T>::N;
  const int64_t n = args.cols;
  if (vec) {
    if (n <= 64 * E) return launch_backward<T, E, 64, 1>(args, groups, stream);
    if (n <= 256 * E) return launch_backward<T, E, 256, 1>(args, groups, stream);
    if (n <= 512 * E) return launch_backward<T, E, 512, 1>(args, groups, stream);
    if (n <= 1024 * E) return launch_backward<T, E, 1024, 1>(args, groups, stream);
    if (n <= 2048 * E) return launch_backward<T, E, 1024, 2>(args, groups, stream);
  } else {
    if (n <= 512) return launch_backward<T, 1, 64, 8>(args, groups, stream);
    if (n <= 2048) return launch_backward<T, 1, 256, 8>(args, groups, stream);
    if (n <= 8192) return launch_backward<T, 1, 1024, 8>(args, groups, stream);
  }
  hipLaunchKernelGGL((rms_norm_backward_long_kernel<T>), dim3(groups), dim3(kLongThreads), 0, stream, args, groups);
  return hipGetLastError();
}

// ---- sums of columns -------------------------------------------------------------

// A workgroup sums one chunk of rows for 64 VEC columns: each of its NW waves every NW-th row, joined
// in wave order.
template <typename T, int VEC, int NW>
__global__ __launch_bounds__(64 * NW) void column_sum_kernel(ColumnSumArgs args) {
  __shared__ float part[NW - 1][64 * VEC];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = (static_cast<int64_t>(blockIdx.x) * 64 + lane) * VEC;
  const int64_t per = (args.rows + args.chunks - 1) / args.chunks;
  const int64_t first = blockIdx.y * per, end = std::min<int64_t>(first + per, args.rows);
  float sum[VEC] = {};
  if (c < args.cols) {
    const T* p = static_cast<const T*>(args.in) + c;
#pragma unroll 4
    for (int64_t row = first + wave; row < end; row += NW) {
      float x[VEC];
      load_elements<VEC>(p + row * args.ld, x);
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum[e] += x[e];
    }
  }
  if (wave > 0) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) part[wave - 1][e * 64 + lane] = sum[e];
  }
  __syncthreads();
  if (wave > 0 || c >= args.cols) return;
#pragma unroll
  for (int w = 0; w < NW - 1; ++w)
#pragma unroll
    for (int e = 0; e < VEC; ++e) sum[e] += part[w][e * 64 + lane];
  float* out = args.chunks > 1 ? args.partials + blockIdx.y * args.cols : args.out;
#pragma unroll
  for (int e = 0; e < VEC; ++e)
    if (c + e < args.cols) out[c + e] = sum[e];
}

template <typename T, int VEC, int NW>
hipError_t launch_sum(const ColumnSumArgs& args, hipStream_t stream) {
  const dim3 g(static_cast<uint32_t>((args.cols + 64 * VEC - 1) / (64 * VEC)), args.chunks);
  hipLaunchKernelGGL((column_sum_kernel<T, VEC, NW>), g, dim3(64 * NW), 0, stream, args);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rms_norm(const NormArgs& args, int dtype, bool vec, hipStream_t stream) {
  return dtype == CLEAVE_BF16 ? launch_norm_of<Bf16>(args, vec, stream) : launch_norm_of<float>(args, vec, stream);
}

int rms_norm_partial_rows(int64_t rows, int64_t cols) {
  (void)cols;
  return static_cast<int>(std::min<int64_t>(rows, 512));
}

hipError_t launch_rms_norm_backward(const NormBackwardArgs& args, int dtype, bool vec, int partial_rows,
                                    hipStream_t stream) {
  return dtype == CLEAVE_BF16 ? launch_backward_of<Bf16>(args, vec, partial_rows, stream)
                              : launch_backward_of<float>(args, vec, partial_rows, stream);
}

int column_sum_chunks(int64_t rows, int64_t cols) {
  const int64_t groups = (cols + 255) / 256;
  const int64_t want = (1024 + groups - 1) / groups;
  return static_cast<int>(std::max<int64_t>(1, std::min({want, (rows + 31) / 32, int64_t{256}})));
}

hipError_t launch_join_rows(const float* rows, int n, int64_t cols, float* out, hipStream_t stream) {
  ColumnSumArgs join{};
  join.in = rows;
  join.ld = cols;
  join.rows = n;
  join.cols = cols;
  join.out = out;
  join.chunks = 1;
  // one column per lane and sixteen waves: as many loads in flight as there can be
  return launch_sum<float, 1, 16>(join, stream);
}

hipError_t launch_column_sum(const ColumnSumArgs& args, int dtype, bool vec, hipStream_t stream) {
  hipError_t e;
  if (dtype == CLEAVE_BF16) e = vec ? launch_sum<Bf16, 8, 4>(args, stream) : launch_sum<Bf16, 1, 4>(args, stream);
  else e = vec ? launch_sum<float, 4, 4>(args, stream) : launch_sum<float, 1, 4>(args, stream);
  if (e != hipSuccess || args.chunks == 1) return e;
  return launch_join_rows(args.partials, args.chunks, args.cols, args.out, stream);
}

}  // namespace cleave
