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
// scaling and the rounding.  A copy of 512 MB runs at 5.4 TB/s here.  bf16 with a residual, the sum stored:
//   norm            4096 x 4096 27 us (5.0 TB/s); 16384 x 5120 into e4m3 103-106 (5.6); 1 x 4096 into e4m3 5.0, a launch
//   gradient        8192 x 4096 with dsum 53-55 us, both launches (5.0 TB/s); fp32 3001 x 1001 13.1 (2.8)
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "fp8_round.h"
#include "operators.h"
#include "row_access.h"
#include "wave_reduce.h"

namespace cleave {

namespace {

// A row per group of NT threads, which holds up to NT * V * N elements of it (N in sixteen bytes); a wave (NT = 64)
// has its row to itself, four rows to a workgroup.
template <int NT>
struct RowGroup {
  static constexpr int kThreads = NT == 64 ? 256 : NT;
  static constexpr int kRows = kThreads / NT;
  static constexpr int kWaves = NT / 64;
};

template <typename T, int NT, int V, bool E4M3>
__global__ __launch_bounds__(RowGroup<NT>::kThreads) void rms_norm_kernel(NormArgs args) {
  typedef Group16<T> G;
  constexpr int NW = RowGroup<NT>::kWaves, N = G::N;
  __shared__ float slots[2][NW];
  const int t = threadIdx.x % NT;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * RowGroup<NT>::kRows + threadIdx.x / NT;
  if (row >= args.rows) return;   // whole waves, and with several waves to a row whole workgroups
  const T* x = static_cast<const T*>(args.x) + row * args.ldx;
  const T* r = static_cast<const T*>(args.residual) + (args.residual ? row * args.ldr : 0);
  T* sum_out = static_cast<T*>(args.sum_out) + (args.sum_out ? row * args.lds : 0);
  const int cols = static_cast<int>(args.cols);
  const auto at = [&](int j) { return (j * NT + t) * N; };

  Raw16 x_raw[V], r_raw[V];
  Floats16<N> w_raw[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    x_raw[j] = G::read(x + at(j), cols - at(j));
    if (args.residual) r_raw[j] = G::read(r + at(j), cols - at(j));
  }
#pragma unroll
  for (int j = 0; j < V; ++j) w_raw[j].read(args.weight + at(j), cols - at(j));
  float h[V][N], w[V][N];
#pragma unroll
  for (int j = 0; j < V; ++j) G::unpack(x_raw[j], h[j]);
  if (args.residual) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float add[N];
      G::unpack(r_raw[j], add);
#pragma unroll
      for (int e = 0; e < N; ++e) h[j][e] += add[e];
    }
  }
  float squares = 0.0f;
#pragma unroll
  for (int j = 0; j < V; ++j)
#pragma unroll
    for (int e = 0; e < N; ++e) squares += h[j][e] * h[j][e];
  if (args.sum_out) {
#pragma unroll
    for (int j = 0; j < V; ++j) G::store(sum_out + at(j), cols - at(j), h[j]);
  }
  squares = group_sum<NW>(squares, slots[0]);
  const float inv = 1.0f / __builtin_sqrtf(squares / static_cast<float>(cols) + args.eps);
  if (args.inv_rms && t == 0) args.inv_rms[row] = inv;
#pragma unroll
  for (int j = 0; j < V; ++j) w_raw[j].unpack(w[j]);
#pragma unroll
  for (int j = 0; j < V; ++j)
#pragma unroll
    for (int e = 0; e < N; ++e) h[j][e] = h[j][e] * inv * w[j][e];
  if constexpr (E4M3) {
    float most = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (at(j) + e < cols) most = nan_max(most, __builtin_fabsf(h[j][e]));   // (inv may be infinite)
    const BlockScale s = block_scale(group_nan_max<NW>(most, slots[1]));
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
__device__ __forceinline__ float element(const float* p) { return *p; }
__device__ __forceinline__ float element(const Bf16* p) {
  return __builtin_bit_cast(float, static_cast<uint32_t>(p->bits) << 16);
}
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(Bf16* p, float x) { p->bits = to_bf16_bits(x); }

template <typename T, bool E4M3>
__global__ __launch_bounds__(kLongThreads) void rms_norm_long_kernel(NormArgs args) {
  constexpr int NW = kLongThreads / 64;
  __shared__ float slots[2][NW];
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(args.x) + row * args.ldx;
  const T* r = static_cast<const T*>(args.residual) + (args.residual ? row * args.ldr : 0);
  const auto at = [&](int64_t c) { return args.residual ? element(x + c) + element(r + c) : element(x + c); };
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
    const float h = at(c), y = h * inv * args.weight[c];
    if (args.sum_out) put(static_cast<T*>(args.sum_out) + row * args.lds + c, h);
    if constexpr (E4M3)
      static_cast<uint8_t*>(args.y)[row * args.ldy + c] = static_cast<uint8_t>(pack_e4m3(y * s.inverse, 0.0f));
    else
      put(static_cast<T*>(args.y) + row * args.ldy + c, y);
  }
}

template <typename T, int NT, int V>
hipError_t launch_norm(const NormArgs& args, hipStream_t stream) {
  constexpr int kRows = RowGroup<NT>::kRows;
  const dim3 g(static_cast<uint32_t>((args.rows + kRows - 1) / kRows)), b(RowGroup<NT>::kThreads);
  if (args.scales) hipLaunchKernelGGL((rms_norm_kernel<T, NT, V, true>), g, b, 0, stream, args);
  else hipLaunchKernelGGL((rms_norm_kernel<T, NT, V, false>), g, b, 0, stream, args);
  return hipGetLastError();
}

// `v` groups to a thread, up to MOST: the least that holds a row.
template <typename T, int NT, int MOST, int V = 1>
hipError_t launch_norm_fit(const NormArgs& args, int64_t v, hipStream_t stream) {
  if constexpr (V < MOST) {
    if (v > V) return launch_norm_fit<T, NT, MOST, V + 1>(args, v, stream);
  }
  return launch_norm<T, NT, V>(args, stream);
}

// Which threads share a row.  Groups of sixteen bytes beyond the row's end leave lanes idle, so a thread holds as
// many as fit the row; wide groups of threads serve few rows, whose latency counts, narrow ones many.  us, 256 and 512
// threads with one or two groups each / these: 16384 x 5120 bf16 into 8 bits 111 / 106, 7247 x 9984 119 / 96, 7232 x 8960
// 97 / 87; 20000 x 768 bf16 with a residual, 256 threads / a wave to a row, 32.4 / 24.5, into 8 bits 39 / 23.
template <typename T>
hipError_t launch_norm_of(const NormArgs& args, hipStream_t stream) {
  const int64_t groups = (args.cols + Group16<T>::N - 1) / Group16<T>::N;
  if (groups <= 64) return launch_norm<T, 64, 1>(args, stream);
  if (groups <= 4 * 64 && args.rows > 1024) return launch_norm_fit<T, 64, 4>(args, (groups + 63) / 64, stream);
  if (groups <= 8 * 256 && args.rows > 256) return launch_norm_fit<T, 256, 8>(args, (groups + 255) / 256, stream);
  if (groups <= 4 * 1024) return launch_norm_fit<T, 1024, 4>(args, (groups + 1023) / 1024, stream);
  const dim3 g(static_cast<uint32_t>(args.rows)), b(kLongThreads);
  if (args.scales) hipLaunchKernelGGL((rms_norm_long_kernel<T, true>), g, b, 0, stream, args);
  else hipLaunchKernelGGL((rms_norm_long_kernel<T, false>), g, b, 0, stream, args);
  return hipGetLastError();
}

// ---- gradient ------------------------------------------------------------------

// dx needs a row's whole sum, dw a sum over the rows: both leave one pass over dy and h.  Every group of the launch takes
// every groups-th row and holds its part of the weight's gradient in registers until the last of them: one row of partial sums
// for each workgroup (8192 x 4096: 512 rows of 16 KB, 8 MB beside the 268 MB of the pass; 5 us to join), whose groups (a wave
// each, where there are several) are joined in order.
template <typename T, int NT, int V>
__global__ __launch_bounds__(RowGroup<NT>::kThreads) void rms_norm_backward_kernel(NormBackwardArgs args) {
  typedef Group16<T> G;
  constexpr int NW = RowGroup<NT>::kWaves, N = G::N, GROUPS = RowGroup<NT>::kRows;
  __shared__ float slots[2][NW];
  const int t = threadIdx.x % NT;
  const int group = blockIdx.x * GROUPS + threadIdx.x / NT, groups = gridDim.x * GROUPS;
  const int cols = static_cast<int>(args.cols);
  const auto at = [&](int j) { return (j * NT + t) * N; };
  float dw[V][N] = {}, w[V][N];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    Floats16<N> raw;
    raw.read(args.weight + at(j), cols - at(j));
    raw.unpack(w[j]);
  }
  int turn = 0;
  for (int64_t row = group; row < args.rows; row += groups, turn ^= 1) {
    const T* dy = static_cast<const T*>(args.dy) + row * args.lddy;
    const T* h = static_cast<const T*>(args.h) + row * args.ldh;
    const float inv = args.inv_rms[row];
    Raw16 g_raw[V], h_raw[V], add_raw[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      g_raw[j] = G::read(dy + at(j), cols - at(j));
      h_raw[j] = G::read(h + at(j), cols - at(j));
    }
    if (args.dsum) {
      const T* dsum = static_cast<const T*>(args.dsum) + row * args.ldds;
#pragma unroll
      for (int j = 0; j < V; ++j) add_raw[j] = G::read(dsum + at(j), cols - at(j));
    }
    float g[V][N], xhat[V][N];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      G::unpack(g_raw[j], g[j]);
      G::unpack(h_raw[j], xhat[j]);
    }
    float dot = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        if (at(j) + e >= cols) xhat[j][e] = 0.0f;   // (inv may be infinite)
        else xhat[j][e] *= inv;
        dw[j][e] += g[j][e] * xhat[j][e];
        g[j][e] *= w[j][e];
        dot += g[j][e] * xhat[j][e];
      }
    // (the slots of the row before last are free: every wave has passed the barrier of the last one)
    const float mean = group_sum<NW>(dot, slots[turn]) / static_cast<float>(cols);
    T* dx = static_cast<T*>(args.dx) + row * args.lddx;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float add[N] = {};
      if (args.dsum) G::unpack(add_raw[j], add);
#pragma unroll
      for (int e = 0; e < N; ++e) g[j][e] = (g[j][e] - xhat[j][e] * mean) * inv + add[e];
      G::store(dx + at(j), cols - at(j), g[j]);
    }
  }
  if constexpr (GROUPS > 1) {
    __shared__ float joined[GROUPS - 1][V * N][NT];
    if (threadIdx.x >= NT) {
#pragma unroll
      for (int j = 0; j < V; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) joined[threadIdx.x / NT - 1][j * N + e][t] = dw[j][e];
    }
    __syncthreads();
    if (threadIdx.x >= NT) return;
#pragma unroll
    for (int g = 0; g < GROUPS - 1; ++g)
#pragma unroll
      for (int j = 0; j < V; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) dw[j][e] += joined[g][j * N + e][t];
  }
  float* out = args.partials + static_cast<int64_t>(blockIdx.x) * args.cols;
#pragma unroll
  for (int j = 0; j < V; ++j) store_floats<N>(out + at(j), cols - at(j), dw[j]);
}

// Rows that no group's registers hold: the partial sums are kept in the group's row of them.
template <typename T>
__global__ __launch_bounds__(kLongThreads) void rms_norm_backward_long_kernel(NormBackwardArgs args) {
  constexpr int NW = kLongThreads / 64;
  __shared__ float slots[2][NW];
  float* out = args.partials + static_cast<int64_t>(blockIdx.x) * args.cols;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < args.rows; row += gridDim.x, turn ^= 1) {
    const T* dy = static_cast<const T*>(args.dy) + row * args.lddy;
    const T* h = static_cast<const T*>(args.h) + row * args.ldh;
    const float inv = args.inv_rms[row];
    const bool fresh = row == blockIdx.x;
    float dot = 0.0f;
    for (int64_t c = threadIdx.x; c < args.cols; c += kLongThreads) {
      const float g = element(dy + c), x = element(h + c) * inv;
      out[c] = (fresh ? 0.0f : out[c]) + g * x;
      dot += g * args.weight[c] * x;
    }
    const float mean = group_sum<NW>(dot, slots[turn]) / static_cast<float>(args.cols);
    for (int64_t c = threadIdx.x; c < args.cols; c += kLongThreads) {
      const float add = args.dsum ? element(static_cast<const T*>(args.dsum) + row * args.ldds + c) : 0.0f;
      put(static_cast<T*>(args.dx) + row * args.lddx + c,
          (element(dy + c) * args.weight[c] - element(h + c) * inv * mean) * inv + add);
    }
  }
}

template <typename T, int NT, int V>
hipError_t launch_backward(const NormBackwardArgs& args, int workgroups, hipStream_t stream) {
  hipLaunchKernelGGL((rms_norm_backward_kernel<T, NT, V>), dim3(workgroups), dim3(RowGroup<NT>::kThreads), 0, stream, args);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_backward_of(const NormBackwardArgs& args, int groups, hipStream_t stream) {
  constexpr int N = Group16<T>::N;
  const int64_t n = args.cols;
  if (n <= 64 * N) return launch_backward<T, 64, 1>(args, groups, stream);
  if (n <= 128 * N && args.rows > 2048) return launch_backward<T, 64, 2>(args, groups, stream);
  if (n <= 256 * N) return launch_backward<T, 256, 1>(args, groups, stream);
  if (n <= 512 * N) return launch_backward<T, 512, 1>(args, groups, stream);
  if (n <= 1024 * N) return launch_backward<T, 1024, 1>(args, groups, stream);
  if (n <= 2048 * N) return launch_backward<T, 1024, 2>(args, groups, stream);
  if constexpr (N == 4) {   // (fp32 up to 16384 columns in registers, as bf16 above; us, read again / so, 887 x 8960 53.6 / 33.6)
    if (n <= 3072 * N) return launch_backward<T, 1024, 3>(args, groups, stream);
    if (n <= 4096 * N) return launch_backward<T, 1024, 4>(args, groups, stream);
  }
  hipLaunchKernelGGL((rms_norm_backward_long_kernel<T>), dim3(groups), dim3(kLongThreads), 0, stream, args);
  return hipGetLastError();
}

// ---- sums of columns -------------------------------------------------------------

// A workgroup sums one chunk of rows for 64 groups of columns: each of its NW waves every NW-th row, joined
// in wave order; the chunks by the kernel below.  Bound by memory: 4096 x 11008 bf16, not in any cache, 19 us and 4 for the join.
template <typename T, int NW>
__global__ __launch_bounds__(64 * NW) void column_sum_kernel(ColumnSumArgs args) {
  typedef Group16<T> G;
  constexpr int N = G::N;
  __shared__ float part[NW - 1][64 * N];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = (static_cast<int64_t>(blockIdx.x) * 64 + lane) * N;
  const int64_t per = (args.rows + args.chunks - 1) / args.chunks;
  const int64_t first = blockIdx.y * per, end = std::min<int64_t>(first + per, args.rows);
  const int left = static_cast<int>(std::min<int64_t>(args.cols - c, N));
  float sum[N] = {};
  if (left > 0) {
    const T* p = static_cast<const T*>(args.in) + c;
#pragma unroll 4
    for (int64_t row = first + wave; row < end; row += NW) {
      float x[N];
      G::unpack(G::read(p + row * args.ld, left), x);
#pragma unroll
      for (int e = 0; e < N; ++e) sum[e] += x[e];
    }
  }
  if (wave > 0) {
#pragma unroll
    for (int e = 0; e < N; ++e) part[wave - 1][e * 64 + lane] = sum[e];
  }
  __syncthreads();
  if (wave > 0 || left <= 0) return;
#pragma unroll
  for (int w = 0; w < NW - 1; ++w)
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] += part[w][e * 64 + lane];
  store_floats<N>((args.chunks > 1 ? args.partials + blockIdx.y * args.cols : args.out) + c, left, sum);
}

template <typename T, int NW>
hipError_t launch_sum(const ColumnSumArgs& args, hipStream_t stream) {
  constexpr int kCols = 64 * Group16<T>::N;
  const dim3 g(static_cast<uint32_t>((args.cols + kCols - 1) / kCols), args.chunks);
  hipLaunchKernelGGL((column_sum_kernel<T, NW>), g, dim3(64 * NW), 0, stream, args);
  return hipGetLastError();
}

// The rows of partial sums: sixteen columns to a workgroup and 64 rows at a time, so that a few hundred rows are a few loads
// of each thread.
constexpr int kJoinThreads = 1024, kJoinCols = 16;
__global__ __launch_bounds__(kJoinThreads) void join_rows_kernel(const float* in, int rows, int64_t ld, int64_t cols, float* out) {
  constexpr int kRows = kJoinThreads / kJoinCols;
  __shared__ float part[kJoinThreads / 64][kJoinCols];
  const int at = threadIdx.x % kJoinCols, first = threadIdx.x / kJoinCols;
  const int64_t c = static_cast<int64_t>(blockIdx.x) * kJoinCols + at;
  float sum = 0.0f;
  if (c < cols) {
#pragma unroll 8
    for (int row = first; row < rows; row += kRows) sum += in[row * ld + c];
  }
  // a wave's four rows, then the waves
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  if ((threadIdx.x & 63) < kJoinCols) part[threadIdx.x / 64][at] = sum;
  __syncthreads();
  if (threadIdx.x >= kJoinCols || c >= cols) return;
  sum = part[0][at];
#pragma unroll
  for (int w = 1; w < kJoinThreads / 64; ++w) sum += part[w][at];
  out[c] = sum;
}

}  // namespace

// A launch has fewer than 2^32 threads: more rows (columns, of a join) than these take several.
constexpr int64_t kLaunchRows = int64_t{1} << 21, kLaunchCols = int64_t{1} << 25;

hipError_t launch_rms_norm(const NormArgs& args, int dtype, hipStream_t stream) {
  const int64_t eb = dtype == CLEAVE_BF16 ? 2 : 4, yb = args.scales ? 1 : eb;
  for (int64_t row = 0; row < args.rows; row += kLaunchRows) {
    const auto down = [&](auto* p, int64_t bytes) {
      return p ? reinterpret_cast<decltype(p)>(reinterpret_cast<uintptr_t>(p) + row * bytes) : p;
    };
    NormArgs some = args;
    some.rows = std::min(args.rows - row, kLaunchRows);
    some.x = down(args.x, args.ldx * eb);
    some.residual = down(args.residual, args.ldr * eb);
    some.sum_out = down(args.sum_out, args.lds * eb);
    some.y = down(args.y, args.ldy * yb);
    some.scales = down(args.scales, 4);
    some.inv_rms = down(args.inv_rms, 4);
    const hipError_t e = dtype == CLEAVE_BF16 ? launch_norm_of<Bf16>(some, stream) : launch_norm_of<float>(some, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Workgroups of the gradient: what the CUs hold at a time, where every group of threads gets a few rows.  (Narrow rows have four
// groups to a workgroup.)
int rms_norm_partial_rows(int64_t rows, int64_t cols) {
  const int64_t groups = cols <= 1024 ? 8192 : cols <= 2048 ? 1024 : 512;
  const int64_t some = std::min(groups, rows <= 2048 ? rows : std::max<int64_t>((rows + 3) / 4, 2048));
  return static_cast<int>(cols <= 1024 ? (some + 3) / 4 : std::min<int64_t>(some, groups));
}

hipError_t launch_rms_norm_backward(const NormBackwardArgs& args, int dtype, int partial_rows, hipStream_t stream) {
  return dtype == CLEAVE_BF16 ? launch_backward_of<Bf16>(args, partial_rows, stream)
                              : launch_backward_of<float>(args, partial_rows, stream);
}

int column_sum_chunks(int64_t rows, int64_t cols) {
  const int64_t groups = (cols + 255) / 256;
  const int64_t want = (1024 + groups - 1) / groups;
  return static_cast<int>(std::max<int64_t>(1, std::min({want, (rows + 31) / 32, int64_t{256}})));
}

hipError_t launch_join_rows(const float* rows, int n, int64_t cols, float* out, hipStream_t stream) {
  for (int64_t c = 0; c < cols; c += kLaunchCols) {
    const int64_t some = std::min(cols - c, kLaunchCols);
    hipLaunchKernelGGL(join_rows_kernel, dim3(static_cast<uint32_t>((some + kJoinCols - 1) / kJoinCols)), dim3(kJoinThreads), 0,
                       stream, rows + c, n, cols, some, out + c);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_column_sum(const ColumnSumArgs& args, int dtype, hipStream_t stream) {
  const hipError_t e = dtype == CLEAVE_BF16 ? launch_sum<Bf16, 4>(args, stream) : launch_sum<float, 4>(args, stream);
  if (e != hipSuccess || args.chunks == 1) return e;
  return launch_join_rows(args.partials, args.chunks, args.cols, args.out, stream);
}

}  // namespace cleave
