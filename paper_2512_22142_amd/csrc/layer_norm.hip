// Layer norm of a residual stream and its gradient (the paper keeps such operators on the parameter server, Sec. 4.1).
//
//   h = x + r;  m = mean(h);  i = 1 / sqrt(mean((h - m)^2) + eps);  y = (h - m) i w + b
// over the columns of each row, in fp32 from the unrounded h; y in x's type or, for a product with 8-bit
// operands, as e4m3 with the row's scale s = max|y| / 448.
// The mean is taken twice: m0 from the sum of h, then, with d = h - m0, m = m0 + mean(d) and the variance
// mean(d^2) - mean(d)^2, in which nothing cancels.  A mean that is large beside the deviations is then as good as fp32
// holds it (m0 alone is off by a few roundings of the mean, all of which would reach y).
//
// Gradient, with the stored h, m and i, g = dy w and xhat = (h - m) i:
//   dx = i (g - mean(g) - xhat mean(g xhat)) + dsum;   dw = sum over rows of dy xhat;   db = sum over rows of dy
//
// Bound by memory: every row is read once and kept in registers between its statistics, the scaling and the rounding.  A copy of
// 512 MB runs at 5.4 TB/s here.  us:
//   bf16 with a residual, the sum stored  8192 x 768 11.0 (4.6 TB/s); 4096 x 4096 22.0 (from the caches); 16384 x 5120 129 (5.2), into
//                                         e4m3 118 (5.0); 1 x 4096 into e4m3 3.9, a launch
//   gradient, both launches               16384 x 5120 bf16 with dsum 135-137 (4.9-5.0 TB/s); 2999 x 1111 fp32 14.5 (2.8)
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "fp8_round.h"
#include "operators.h"
#include "row_access.h"
#include "wave_reduce.h"

namespace cleave {

namespace {

// A row's group from column `at` on.  ENDING: rows of bf16 that are not in whole groups, few of them to a thread.  The branches of a last
// group's elements wait one after the other there, so wide loads that end with the row are put in place instead (fp32's do not wait, and
// threads with many groups have no registers for it).  us, branches / wide loads:
//   forward    8313 x 789 16.8 / 14.5, 1689 x 2596 12.2 / 9.8, whole groups 8192 x 768 11.0 / 11.7
//   gradient   8313 x 789 28.7 / 19.4, 1689 x 2596 22.0 / 16.7, 7353 x 9235 (512 x 3) 192 / 169
//   not taken  gradient of 512 x 4, 4566 x 13859 168 / 227; fp32 2999 x 1111 14.5 / 19
template <bool ENDING, typename T>
__device__ __forceinline__ Raw16 read_group(const T* row, int at, int cols) {
  if constexpr (ENDING) return read_ending(row + at, cols - at);
  else return Group16<T>::read(row + at, cols - at);
}
template <bool ENDING>
__device__ __forceinline__ Raw16 settle_group(Raw16 w, int at, int cols) {
  return ENDING ? settle(w, cols - at) : w;
}
bool takes_ending(int64_t cols) { return cols % 8 != 0 && cols > 8; }

template <typename T, int NT, int V, bool E4M3, bool ENDING>
__global__ __launch_bounds__(RowGroup<NT>::kThreads) void layer_norm_kernel(LayerNormArgs args) {
  typedef Group16<T> G;
  constexpr int NW = RowGroup<NT>::kWaves, N = G::N;
  __shared__ float slots[4][NW];
  const int t = threadIdx.x % NT;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * RowGroup<NT>::kRows + threadIdx.x / NT;
  if (row >= args.rows) return;   // whole sixteens of lanes, waves, or with several waves to a row workgroups
  const T* x = static_cast<const T*>(args.x) + row * args.ldx;
  const T* r = static_cast<const T*>(args.residual) + (args.residual ? row * args.ldr : 0);
  T* sum_out = static_cast<T*>(args.sum_out) + (args.sum_out ? row * args.lds : 0);
  const int cols = static_cast<int>(args.cols);
  const float part = 1.0f / static_cast<float>(cols);
  const auto at = [&](int j) { return (j * NT + t) * N; };

  // The weight and the bias of a thread's columns are on their way with the row where there are registers for them.
  constexpr bool EARLY = V * N <= 16;
  Raw16 x_raw[V], r_raw[V];
  [[maybe_unused]] Floats16<N> w_raw[V], b_raw[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    x_raw[j] = read_group<ENDING>(x, at(j), cols);
    if (args.residual) r_raw[j] = read_group<ENDING>(r, at(j), cols);
  }
  const auto read_weights = [&](int j) {
    w_raw[j].read(args.weight + at(j), cols - at(j));
    if (args.bias) b_raw[j].read(args.bias + at(j), cols - at(j));
  };
  if constexpr (EARLY) {
#pragma unroll
    for (int j = 0; j < V; ++j) read_weights(j);
  }
  float h[V][N];
#pragma unroll
  for (int j = 0; j < V; ++j) G::unpack(settle_group<ENDING>(x_raw[j], at(j), cols), h[j]);
  if (args.residual) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float add[N];
      G::unpack(settle_group<ENDING>(r_raw[j], at(j), cols), add);
#pragma unroll
      for (int e = 0; e < N; ++e) h[j][e] += add[e];
    }
  }
  float sum = 0.0f;
#pragma unroll
  for (int j = 0; j < V; ++j)
#pragma unroll
    for (int e = 0; e < N; ++e) sum += h[j][e];
  if (args.sum_out) {
#pragma unroll
    for (int j = 0; j < V; ++j) G::store(sum_out + at(j), cols - at(j), h[j]);
  }
  const float first = group_total<NT>(sum, slots[0]) * part;
  float rest = 0.0f, squares = 0.0f;
#pragma unroll
  for (int j = 0; j < V; ++j)
#pragma unroll
    for (int e = 0; e < N; ++e) {
      h[j][e] = at(j) + e < cols ? h[j][e] - first : 0.0f;
      rest += h[j][e];
      squares += h[j][e] * h[j][e];
    }
  group_totals<NT>(rest, squares, slots[1]);
  rest *= part;
  const float var = squares * part - rest * rest;
  const float inv = 1.0f / __builtin_sqrtf((var < 0.0f ? 0.0f : var) + args.eps);   // (NaN stays)
  if (t == 0) {
    if (args.mean) args.mean[row] = first + rest;
    if (args.inv_std) args.inv_std[row] = inv;
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    float w[N], b[N] = {};
    if constexpr (!EARLY) read_weights(j);
    w_raw[j].unpack(w);
    if (args.bias) b_raw[j].unpack(b);
#pragma unroll
    for (int e = 0; e < N; ++e) h[j][e] = (h[j][e] - rest) * inv * w[e] + b[e];
  }
  if constexpr (E4M3) {
    float most = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (at(j) + e < cols) most = nan_max(most, __builtin_fabsf(h[j][e]));
    const BlockScale s = block_scale(row_nan_max<NT>(most, slots[3]));
    if (t == 0) args.scales[row] = s.scale;
    uint8_t* y = static_cast<uint8_t*>(args.y) + row * args.ldy;
#pragma unroll
    for (int j = 0; j < V; ++j) {
#pragma unroll
      for (int e = 0; e < N; ++e) h[j][e] *= s.inverse;
      store_e4m3<N>(y + at(j), cols - at(j), h[j]);
    }
  } else {
    T* y = static_cast<T*>(args.y) + row * args.ldy;
#pragma unroll
    for (int j = 0; j < V; ++j) G::store(y + at(j), cols - at(j), h[j]);
  }
}

// Rows that no group's registers hold: read again for each use (from the caches).
constexpr int kLongThreads = 1024;

template <typename T, bool E4M3>
__global__ __launch_bounds__(kLongThreads) void layer_norm_long_kernel(LayerNormArgs args) {
  constexpr int NW = kLongThreads / 64;
  __shared__ float slots[4][NW];
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(args.x) + row * args.ldx;
  const T* r = static_cast<const T*>(args.residual) + (args.residual ? row * args.ldr : 0);
  const float count = static_cast<float>(args.cols);
  const auto at = [&](int64_t c) { return args.residual ? element(x + c) + element(r + c) : element(x + c); };
  float sum = 0.0f;
  for (int64_t c = threadIdx.x; c < args.cols; c += kLongThreads) sum += at(c);
  const float first = group_total<kLongThreads>(sum, slots[0]) / count;
  float rest = 0.0f, squares = 0.0f;
  for (int64_t c = threadIdx.x; c < args.cols; c += kLongThreads) {
    const float d = at(c) - first;
    rest += d;
    squares += d * d;
  }
  group_totals<kLongThreads>(rest, squares, slots[1]);
  rest /= count;
  const float var = squares / count - rest * rest;
  const float inv = 1.0f / __builtin_sqrtf((var < 0.0f ? 0.0f : var) + args.eps);
  if (threadIdx.x == 0) {
    if (args.mean) args.mean[row] = first + rest;
    if (args.inv_std) args.inv_std[row] = inv;
  }
  const auto norm = [&](float h, int64_t c) {
    return ((h - first) - rest) * inv * args.weight[c] + (args.bias ? args.bias[c] : 0.0f);
  };
  BlockScale s{1.0f, 1.0f};
  if constexpr (E4M3) {
    float most = 0.0f;
    for (int64_t c = threadIdx.x; c < args.cols; c += kLongThreads) most = nan_max(most, __builtin_fabsf(norm(at(c), c)));
    s = block_scale(group_nan_max<NW>(most, slots[3]));
    if (threadIdx.x == 0) args.scales[row] = s.scale;
  }
  // (an element is read, then written, by one thread: y or the sum may take x's or r's place)
  for (int64_t c = threadIdx.x; c < args.cols; c += kLongThreads) {
    const float h = at(c), y = norm(h, c);
    if (args.sum_out) put(static_cast<T*>(args.sum_out) + row * args.lds + c, h);
    if constexpr (E4M3)
      static_cast<uint8_t*>(args.y)[row * args.ldy + c] = static_cast<uint8_t>(pack_e4m3(y * s.inverse, 0.0f));
    else
      put(static_cast<T*>(args.y) + row * args.ldy + c, y);
  }
}

template <typename T, int NT, int V>
hipError_t launch_norm(const LayerNormArgs& args, hipStream_t stream) {
  constexpr int kRows = RowGroup<NT>::kRows;
  const dim3 g(static_cast<uint32_t>((args.rows + kRows - 1) / kRows)), b(RowGroup<NT>::kThreads);
  if constexpr (Group16<T>::N == 8 && V <= 3) {
    if (takes_ending(args.cols)) {
      if (args.scales) hipLaunchKernelGGL((layer_norm_kernel<T, NT, V, true, true>), g, b, 0, stream, args);
      else hipLaunchKernelGGL((layer_norm_kernel<T, NT, V, false, true>), g, b, 0, stream, args);
      return hipGetLastError();
    }
  }
  if (args.scales) hipLaunchKernelGGL((layer_norm_kernel<T, NT, V, true, false>), g, b, 0, stream, args);
  else hipLaunchKernelGGL((layer_norm_kernel<T, NT, V, false, false>), g, b, 0, stream, args);
  return hipGetLastError();
}

// `v` groups to a thread, up to MOST: the least that holds a row.
template <typename T, int NT, int MOST, int V = 1>
hipError_t launch_norm_fit(const LayerNormArgs& args, int64_t v, hipStream_t stream) {
  if constexpr (V < MOST) {
    if (v > V) return launch_norm_fit<T, NT, MOST, V + 1>(args, v, stream);
  }
  return launch_norm<T, NT, V>(args, stream);
}

// Which threads share a row: as few lanes or waves as hold it in one or a few groups each; for few rows, whose latency counts, in one
// group each up to 512 threads (more waves wait longer for each other at each sum).  us, threads x groups of each, bf16 with a residual where
// nothing else is said:
//   a head's width, no residual   262144 x 64: 64 x 1 86, 16 x 1 22.2, 8 x 1 14.0 (4.8 TB/s); 16 x 64: 3.0, 2.8, 2.4
//                                 131072 x 128: 64 x 1 43, 16 x 1 13.6, 8 x 2 13.4; 300 x 128: 3.1, 2.6, 3.0
//                                 131072 x 128 fp32: 64 x 1 33.8, 16 x 2 21.2
//                                 65536 x 256: 64 x 1 24.4, 16 x 2 13.6, 8 x 4 14.6
//   many rows, up to 192 groups   8192 x 768: 64 x 2 11.9, 128 x 1 12.1, 256 x 1 17.2
//   many rows, up to 2048         4096 x 4096: 128 x 4 23.0, 256 x 2 21.9, 1024 x 1 33
//                                 16384 x 5120: 64 x 10 154, 128 x 5 134, 256 x 3 129, 512 x 2 125, 1024 x 1 149
//                                 the same into 8 bits: 192, 125, 118, 137, 185
//                                 20000 x 1000 fp32: 64 x 4 65, 256 x 1 58
//   one row                       1024 columns: 128 x 1 2.8, 256 x 1 3.3, 512 x 1 3.4, 1024 x 1 4.3; into 8 bits 3.3, 3.9, 4.2, 5.4
//                                 4096: 256 x 2 3.3, 512 x 1 3.1, 1024 x 1 4.1; into 8 bits 4.0, 3.9, 5.4
//                                 8192: 512 x 2 3.7, 1024 x 1 4.0 (250 rows 5.1, 5.5)
//                                 16384: 512 x 4 5.3, 1024 x 2 5.2; into 8 bits 6.4, 6.7
template <typename T>
hipError_t launch_norm_of(const LayerNormArgs& args, hipStream_t stream) {
  const int64_t groups = (args.cols + Group16<T>::N - 1) / Group16<T>::N;
  if (groups <= 8) return launch_norm<T, 8, 1>(args, stream);
  if (groups <= 16) return launch_norm<T, 16, 1>(args, stream);
  if (groups <= 32) return launch_norm<T, 16, 2>(args, stream);
  if (groups <= 64) return launch_norm<T, 64, 1>(args, stream);
  if (groups <= 3 * 64 && args.rows > 1024) return launch_norm_fit<T, 64, 3>(args, (groups + 63) / 64, stream);
  if (groups <= 128 && args.rows <= 1024) return launch_norm<T, 128, 1>(args, stream);
  if (groups <= 8 * 256 && args.rows > 256) return launch_norm_fit<T, 256, 8>(args, (groups + 255) / 256, stream);
  if (groups <= 256) return launch_norm<T, 256, 1>(args, stream);
  if (groups <= 4 * 512) return launch_norm_fit<T, 512, 4>(args, (groups + 511) / 512, stream);
  if (groups <= 3 * 1024) return launch_norm<T, 1024, 3>(args, stream);
  if (groups <= 4 * 1024) return launch_norm<T, 1024, 4>(args, stream);
  const dim3 g(static_cast<uint32_t>(args.rows)), b(kLongThreads);
  if (args.scales) hipLaunchKernelGGL((layer_norm_long_kernel<T, true>), g, b, 0, stream, args);
  else hipLaunchKernelGGL((layer_norm_long_kernel<T, false>), g, b, 0, stream, args);
  return hipGetLastError();
}

// ---- gradient ------------------------------------------------------------------

// Floats of the weight's sums in a row of partial sums, the bias's behind them: whole quads.
__host__ __device__ __forceinline__ int64_t padded(int64_t cols) { return (cols + 3) / 4 * 4; }

// One pass over dy and h for dx and for the sums over rows: every group of the launch takes every groups-th row and holds its
// part of dw and db in registers until the last of them, one row of partial sums for each workgroup, whose groups (a
// wave each, where there are several) are joined in order.  The next row's loads are on their way while a row's sums are joined.
// (Groups of fewer than 64 threads add theirs by columns.)
template <typename T, int V>
struct BackwardRow {
  Raw16 dy[V], h[V], add[V];
  float mean, inv;
};
template <typename T, int NT, int V, bool ENDING>
__global__ __launch_bounds__(RowGroup<NT>::kThreads) void layer_norm_backward_kernel(LayerNormBackwardArgs args) {
  typedef Group16<T> G;
  constexpr int NW = RowGroup<NT>::kWaves, N = G::N, GROUPS = RowGroup<NT>::kRows;
  __shared__ float slots[2][2 * NW];
  const int t = threadIdx.x % NT;
  const int64_t group = static_cast<int64_t>(blockIdx.x) * GROUPS + threadIdx.x / NT, groups = static_cast<int64_t>(gridDim.x) * GROUPS;
  const int cols = static_cast<int>(args.cols);
  const float count = static_cast<float>(cols);
  const auto at = [&](int j) { return (j * NT + t) * N; };
  float dw[V][N] = {}, db[V][N] = {}, w[V][N];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    Floats16<N> raw;
    raw.read(args.weight + at(j), cols - at(j));
    raw.unpack(w[j]);
  }
  const auto fetch = [&](int64_t row, BackwardRow<T, V>& to) {
    const T* dy = static_cast<const T*>(args.dy) + row * args.lddy;
    const T* h = static_cast<const T*>(args.h) + row * args.ldh;
    to.mean = args.mean[row];
    to.inv = args.inv_std[row];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      to.dy[j] = read_group<ENDING>(dy, at(j), cols);
      to.h[j] = read_group<ENDING>(h, at(j), cols);
    }
    if (args.dsum) {
      const T* dsum = static_cast<const T*>(args.dsum) + row * args.ldds;
#pragma unroll
      for (int j = 0; j < V; ++j) to.add[j] = read_group<ENDING>(dsum, at(j), cols);
    }
  };
  // (where there are registers for two rows)
  constexpr bool AHEAD = NT < 1024 && V * N <= 24;
  BackwardRow<T, V> cur, next;
  if (AHEAD && group < args.rows) fetch(group, cur);
  int turn = 0;
  for (int64_t row = group; row < args.rows; row += groups, turn ^= 1) {
    if (!AHEAD) fetch(row, cur);
    else if (row + groups < args.rows) fetch(row + groups, next);
    float g[V][N], xhat[V][N];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      G::unpack(settle_group<ENDING>(cur.dy[j], at(j), cols), g[j]);
      G::unpack(settle_group<ENDING>(cur.h[j], at(j), cols), xhat[j]);
    }
    float sum = 0.0f, dot = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        xhat[j][e] = at(j) + e < cols ? (xhat[j][e] - cur.mean) * cur.inv : 0.0f;
        dw[j][e] += g[j][e] * xhat[j][e];
        db[j][e] += g[j][e];
        g[j][e] *= w[j][e];
        sum += g[j][e];
        dot += g[j][e] * xhat[j][e];
      }
    // (the slots of the row before last are free: every wave has passed the barrier of the last one)
    group_totals<NT>(sum, dot, slots[turn]);
    sum /= count;
    dot /= count;
    T* dx = static_cast<T*>(args.dx) + row * args.lddx;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float add[N] = {};
      if (args.dsum) G::unpack(settle_group<ENDING>(cur.add[j], at(j), cols), add);
#pragma unroll
      for (int e = 0; e < N; ++e) g[j][e] = (g[j][e] - sum - xhat[j][e] * dot) * cur.inv + add[e];
      G::store(dx + at(j), cols - at(j), g[j]);
    }
    if (AHEAD) cur = next;
  }
  const int64_t half = padded(args.cols);
  float* out = args.partials + static_cast<int64_t>(blockIdx.x) * 2 * half;
  if constexpr (NT < 64) {   // a column to a thread
    constexpr int kWide = NT * V * N;
    __shared__ float joined[GROUPS][2][kWide];
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        joined[threadIdx.x / NT][0][at(j) + e] = dw[j][e];
        joined[threadIdx.x / NT][1][at(j) + e] = db[j][e];
      }
    __syncthreads();
    for (int c = threadIdx.x; c < cols; c += RowGroup<NT>::kThreads) {
      float sums[2] = {};
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        sums[0] += joined[g][0][c];
        sums[1] += joined[g][1][c];
      }
      out[c] = sums[0];
      out[half + c] = sums[1];
    }
    return;
  }
  if constexpr (NT == 64) {
    __shared__ float joined[GROUPS - 1][2 * V * N][NT];
    if (threadIdx.x >= NT) {
#pragma unroll
      for (int j = 0; j < V; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) {
          joined[threadIdx.x / NT - 1][j * N + e][t] = dw[j][e];
          joined[threadIdx.x / NT - 1][(V + j) * N + e][t] = db[j][e];
        }
    }
    __syncthreads();
    if (threadIdx.x >= NT) return;
#pragma unroll
    for (int g = 0; g < GROUPS - 1; ++g)
#pragma unroll
      for (int j = 0; j < V; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) {
          dw[j][e] += joined[g][j * N + e][t];
          db[j][e] += joined[g][(V + j) * N + e][t];
        }
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    store_floats<N>(out + at(j), cols - at(j), dw[j]);
    store_floats<N>(out + half + at(j), cols - at(j), db[j]);
  }
}

// Rows that no group's registers hold: the partial sums are kept in the group's row of them.
template <typename T>
__global__ __launch_bounds__(kLongThreads) void layer_norm_backward_long_kernel(LayerNormBackwardArgs args) {
  constexpr int NW = kLongThreads / 64;
  __shared__ float slots[2][2 * NW];
  const int64_t half = padded(args.cols);
  float* out = args.partials + static_cast<int64_t>(blockIdx.x) * 2 * half;
  const float count = static_cast<float>(args.cols);
  int turn = 0;
  for (int64_t row = blockIdx.x; row < args.rows; row += gridDim.x, turn ^= 1) {
    const T* dy = static_cast<const T*>(args.dy) + row * args.lddy;
    const T* h = static_cast<const T*>(args.h) + row * args.ldh;
    const float inv = args.inv_std[row], mean = args.mean[row];
    const bool fresh = row == blockIdx.x;
    float sum = 0.0f, dot = 0.0f;
    for (int64_t c = threadIdx.x; c < args.cols; c += kLongThreads) {
      const float d = element(dy + c), x = (element(h + c) - mean) * inv, g = d * args.weight[c];
      out[c] = (fresh ? 0.0f : out[c]) + d * x;
      out[half + c] = (fresh ? 0.0f : out[half + c]) + d;
      sum += g;
      dot += g * x;
    }
    group_totals<kLongThreads>(sum, dot, slots[turn]);
    sum /= count;
    dot /= count;
    for (int64_t c = threadIdx.x; c < args.cols; c += kLongThreads) {
      const float add = args.dsum ? element(static_cast<const T*>(args.dsum) + row * args.ldds + c) : 0.0f;
      put(static_cast<T*>(args.dx) + row * args.lddx + c,
          (element(dy + c) * args.weight[c] - sum - (element(h + c) - mean) * inv * dot) * inv + add);
    }
  }
}

// The rows of partial sums, in a fixed order: 64 columns to a workgroup, sixteen bytes to a thread, 64 rows at a time.  (What lies between
// a half's end and the next quad is read and not used.)
constexpr int kJoinThreads = 1024, kJoinCols = 64;
__global__ __launch_bounds__(kJoinThreads) void layer_norm_join_kernel(const float* in, int rows, int64_t first, int64_t cols,
                                                                       float* dweight, float* dbias) {
  typedef Group16<float> G;
  constexpr int kRows = kJoinThreads / 16;
  __shared__ float part[kJoinThreads / 64][kJoinCols];
  const int quad = threadIdx.x % 16;
  const int64_t half = padded(cols), all = 2 * half, c0 = first + static_cast<int64_t>(blockIdx.x) * kJoinCols;
  const float* p = in + min(c0 + 4 * quad, all - 4);
  float sum[4] = {};
#pragma unroll 8
  for (int row = threadIdx.x / 16; row < rows; row += kRows) {
    float x[4];
    G::unpack(G::read(p + row * all, 4), x);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] += x[e];
  }
  // a wave's four rows, then the waves
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    sum[e] += __shfl_xor(sum[e], 16);
    sum[e] += __shfl_xor(sum[e], 32);
    if ((threadIdx.x & 63) < 16) part[threadIdx.x / 64][4 * quad + e] = sum[e];
  }
  __syncthreads();
  const int64_t c = c0 + threadIdx.x;
  if (threadIdx.x >= kJoinCols) return;
  float total = part[0][threadIdx.x];
#pragma unroll
  for (int w = 1; w < kJoinThreads / 64; ++w) total += part[w][threadIdx.x];
  if (c < cols) dweight[c] = total;
  else if (dbias && c >= half && c < half + cols) dbias[c - half] = total;
}

// Threads of a row, groups of sixteen bytes of each, and workgroups: what the CUs hold at a time, so that a workgroup's rows share
// one row of partial sums.  Narrow rows are a wave's, four to a workgroup, without a barrier, or eight or sixteen lanes'.  us, the first launch
// alone, threads x groups of each (in so many workgroups), groups of a row in brackets, bf16 where nothing else is said:
//   a head's width, no dsum  262144 x 64 [8]: 64 x 1 (1024) 100, 16 x 1 (512, 1024) 36.2, 26.8, 8 x 1 (512, 1024) 19.4 (5.2 TB/s), 18.1
//                            32768 x 64 [8]: the same 16.4, 7.0, 6.3, 5.0, 5.3
//                            65536 x 100 [13]: 64 x 1 47, 16 x 1 20.9, 15.1, 8 x 2 14.5, 17.1
//                            65536 x 256 [32]: 64 x 1 30.3, 16 x 2 (512, 1024) 19.2, 21.1; 30000 x 256: 128 x 1 28, 64 x 1 17.4
//   a wave                   8192 x 768 [96]: 256 x 1 17.2, 128 x 1 (2048) 13.1, 64 x 2 (512) 13.7
//                            2999 x 1111 fp32 [278]: 512 x 1 12.2, 256 x 2 10.8, 64 x 5 11.0 with half the rows of partial sums
//   one workgroup            8192 x 1536 [192]: 64 x 3 20.4, 256 x 1 (512, 768, 1024) 23.5, 20.1, 19.8
//                            8192 x 4096 [512]: 1024 x 1 71, 256 x 2 50.5, 512 x 1 49.9
//                            16384 x 5120 with dsum [640]: 1024 x 1 155, 512 x 2 158, 128 x 5 145, 256 x 3 (256, 512, 768, 1024) 160, 133, 154, 140
//                            1000 x 8192 [1024]: 512 x 2 (256, 512) 16.8, 21.4
//   with the next row on its way 1024 threads have too few registers for two groups of bf16
//                            2048 x 12288 [1536]: 1024 x 2 98, 512 x 3 44
//                            2048 x 16384 [2048], without the next row: 1024 x 2 114, 512 x 4 67 (with it 132)
//   wider, fp32 only         1024 x 8832 [2208]: read twice (the long kernel) 63, 512 x 5 27.4, 1024 x 3 32.3
//                            1024 x 12288: read twice 85, 512 x 6 65, 1024 x 3 46
//                            1024 x 16384 [4096]: read twice 108, 512 x 8 78, 1024 x 4 89
struct BackwardShape {
  int threads, groups, workgroups;
};
BackwardShape backward_shape(int64_t rows, int64_t cols, int n) {
  const int64_t g = (cols + n - 1) / n;
  const auto at_most = [&](int most, int of_workgroup) {
    return static_cast<int>(std::min<int64_t>(most, (rows + of_workgroup - 1) / of_workgroup));
  };
  if (g <= 8) return {8, 1, at_most(512, 32)};
  if (g <= 16) return {16, 1, at_most(1024, 16)};
  if (g <= 32) return {16, 2, at_most(512, 16)};
  if (g <= (n == 8 ? 192 : 320)) return {64, static_cast<int>((g + 63) / 64), at_most(g <= 64 ? 1024 : 512, 4)};
  if (g <= 256) return {256, 1, at_most(768, 1)};
  if (g <= 512) return {512, 1, at_most(512, 1)};
  if (g <= 768) return {256, 3, at_most(512, 1)};
  if (g <= 1024) return {512, 2, at_most(256, 1)};
  if (g <= 1536) return {512, 3, at_most(256, 1)};
  if (g <= 2048) return {512, 4, at_most(256, 1)};
  if (n == 4 && g <= 2560) return {512, 5, at_most(256, 1)};
  if (n == 4 && g <= 3 * 1024) return {1024, 3, at_most(256, 1)};
  if (n == 4 && g <= 4096) return {512, 8, at_most(256, 1)};
  return {kLongThreads, 0, at_most(512, 1)};
}

template <typename T, int NT, int V>
hipError_t launch_backward(const LayerNormBackwardArgs& args, int workgroups, hipStream_t stream) {
  const dim3 g(workgroups), b(RowGroup<NT>::kThreads);
  if constexpr (Group16<T>::N == 8 && V <= 3) {
    if (takes_ending(args.cols)) {
      hipLaunchKernelGGL((layer_norm_backward_kernel<T, NT, V, true>), g, b, 0, stream, args);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((layer_norm_backward_kernel<T, NT, V, false>), g, b, 0, stream, args);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_backward_of(const LayerNormBackwardArgs& args, const BackwardShape& s, hipStream_t stream) {
  switch (s.threads) {
    case 8: return launch_backward<T, 8, 1>(args, s.workgroups, stream);
    case 16:
      return s.groups == 1 ? launch_backward<T, 16, 1>(args, s.workgroups, stream) : launch_backward<T, 16, 2>(args, s.workgroups, stream);
    case 64:
      switch (s.groups) {
        case 1: return launch_backward<T, 64, 1>(args, s.workgroups, stream);
        case 2: return launch_backward<T, 64, 2>(args, s.workgroups, stream);
        case 3: return launch_backward<T, 64, 3>(args, s.workgroups, stream);
        default: break;
      }
      if constexpr (Group16<T>::N == 4)
        return s.groups == 4 ? launch_backward<T, 64, 4>(args, s.workgroups, stream) : launch_backward<T, 64, 5>(args, s.workgroups, stream);
      else
        return hipErrorInvalidValue;   // (backward_shape gives a wave three of bf16 at most)
    case 256:
      return s.groups == 1 ? launch_backward<T, 256, 1>(args, s.workgroups, stream) : launch_backward<T, 256, 3>(args, s.workgroups, stream);
    case 512:
      switch (s.groups) {
        case 1: return launch_backward<T, 512, 1>(args, s.workgroups, stream);
        case 2: return launch_backward<T, 512, 2>(args, s.workgroups, stream);
        case 3: return launch_backward<T, 512, 3>(args, s.workgroups, stream);
        case 4: return launch_backward<T, 512, 4>(args, s.workgroups, stream);
        default: break;
      }
      break;
    default: break;
  }
  if constexpr (Group16<T>::N == 4) {   // (rows of bf16 are read twice from 2049 groups on)
    if (s.groups == 5) return launch_backward<T, 512, 5>(args, s.workgroups, stream);
    if (s.groups == 8) return launch_backward<T, 512, 8>(args, s.workgroups, stream);
    if (s.groups == 3) return launch_backward<T, 1024, 3>(args, s.workgroups, stream);
  }
  hipLaunchKernelGGL((layer_norm_backward_long_kernel<T>), dim3(s.workgroups), dim3(kLongThreads), 0, stream, args);
  return hipGetLastError();
}

}  // namespace

// A launch has fewer than 2^32 threads: more rows than these take several.
constexpr int64_t kLaunchRows = int64_t{1} << 21;

hipError_t launch_layer_norm(const LayerNormArgs& args, int dtype, hipStream_t stream) {
  const int64_t eb = dtype == CLEAVE_BF16 ? 2 : 4, yb = args.scales ? 1 : eb;
  for (int64_t row = 0; row < args.rows; row += kLaunchRows) {
    const auto down = [&](auto* p, int64_t bytes) {
      return p ? reinterpret_cast<decltype(p)>(reinterpret_cast<uintptr_t>(p) + row * bytes) : p;
    };
    LayerNormArgs some = args;
    some.rows = std::min(args.rows - row, kLaunchRows);
    some.x = down(args.x, args.ldx * eb);
    some.residual = down(args.residual, args.ldr * eb);
    some.sum_out = down(args.sum_out, args.lds * eb);
    some.y = down(args.y, args.ldy * yb);
    some.scales = down(args.scales, 4);
    some.mean = down(args.mean, 4);
    some.inv_std = down(args.inv_std, 4);
    const hipError_t e = dtype == CLEAVE_BF16 ? launch_norm_of<Bf16>(some, stream) : launch_norm_of<float>(some, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

int layer_norm_partial_rows(int64_t rows, int64_t cols) {
  return std::max(backward_shape(rows, cols, 4).workgroups, backward_shape(rows, cols, 8).workgroups);
}

hipError_t launch_layer_norm_backward(const LayerNormBackwardArgs& args, int dtype, hipStream_t stream) {
  const bool bf16 = dtype == CLEAVE_BF16;
  const BackwardShape s = backward_shape(args.rows, args.cols, bf16 ? 8 : 4);
  if (args.rows > 0) {
    const hipError_t e = bf16 ? launch_backward_of<Bf16>(args, s, stream) : launch_backward_of<float>(args, s, stream);
    if (e != hipSuccess) return e;
  }
  // (no rows: zeros; a launch has fewer than 2^32 threads)
  constexpr int64_t kLaunchCols = int64_t{1} << 27;
  const int64_t all = args.dbias ? 2 * padded(args.cols) : args.cols;
  for (int64_t c = 0; c < all; c += kLaunchCols) {
    const dim3 g(static_cast<uint32_t>((std::min(all - c, kLaunchCols) + kJoinCols - 1) / kJoinCols));
    hipLaunchKernelGGL(layer_norm_join_kernel, g, dim3(kJoinThreads), 0, stream, args.partials, s.workgroups, c, args.cols, args.dweight,
                       args.dbias);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace cleave
