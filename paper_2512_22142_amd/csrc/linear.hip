// Linear products of few rows -- tokens being served -- and the join of a split
// inner dimension with the epilogue.
//
// Few rows: y = x . W with at most 16 rows of x reads W once and does nothing else that counts, so it is
// bound by memory.  A workgroup has 64 columns, its waves take groups of k in turn; no LDS stands between the loads and the
// matrix instructions (E: elements in 16 bytes; a group: 4 E k's):
//   N x K: lane (n, q) loads the E k's from E q on of column n, and x's rows likewise: fragments as they are.
//   K x N: lane (n, q) loads the columns 4 n .. 4 n + 3 of the rows k = E q .. E q + E - 1, sixteen lanes the 64
//     columns of a row in one run.  It holds, for each of its four columns, the E k's of a fragment; bf16 are put
//     together by v_perm, 4 per fragment, and fragment c belongs to the columns 4 n + c.
// The waves are joined through LDS in wave order.  Sixteen of them leave the output itself, in one launch; where N's columns
// go round the CUs unevenly, four, whose workgroups split K and leave partial sums for a second kernel.
//   One row, bf16, K x N = 4096 x 11008 (90 MB): 17.3-17.6 us with the weights in the Infinity Cache (5.2 TB/s), 20.8-22.8 from memory (4.0-4.3; a
// pass that only sums the columns takes 19 and a second launch); 8192 x 28672 97 us (4.8 TB/s).  16 rows: 18.6 and 24.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "fp8_round.h"
#include "gated_epilogue.h"
#include "kernels.h"
#include "linear_epilogue.h"
#include "row_access.h"

namespace cleave {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kColumns = 64;   // of a workgroup

template <int DTYPE>
struct Type;
template <>
struct Type<CLEAVE_F32> {
  static constexpr int E = 4;
};
template <>
struct Type<CLEAVE_BF16> {
  static constexpr int E = 8;
};
template <>
struct Type<CLEAVE_E4M3> {
  static constexpr int E = 16;
};

// One group of 4 E k's: sixteen bytes of k's in each lane of both operands.
template <int DTYPE>
__device__ __forceinline__ f32x4 multiply(u32x4 x, u32x4 w, f32x4 acc) {
  if constexpr (DTYPE == CLEAVE_BF16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, w), acc, 0, 0, 0);
  } else if constexpr (DTYPE == CLEAVE_E4M3) {
    // (as bf16, exactly: the 8-bit instructions drop bits of the sum)
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_of_e4m3(x[0], x[1]), bf16_of_e4m3(w[0], w[1]), acc, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_of_e4m3(x[2], x[3]), bf16_of_e4m3(w[2], w[3]), acc, 0, 0, 0);
  } else {
    const f32x4 a = __builtin_bit_cast(f32x4, x), b = __builtin_bit_cast(f32x4, w);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], acc, 0, 0, 0);
    return acc;
  }
}

// Reads at any alignment.
template <typename V>
__device__ __forceinline__ V read_any(const unsigned char* p) {
  typedef uint32_t U4 __attribute__((ext_vector_type(4), aligned(1)));
  typedef uint32_t U2 __attribute__((ext_vector_type(2), aligned(1)));
  if constexpr (sizeof(V) == 16) return *reinterpret_cast<const U4*>(p);
  else return *reinterpret_cast<const U2*>(p);
}
// The first `n` elements of EB bytes; zeros behind them.
template <typename V, int EB>
__device__ __forceinline__ V read_some(const unsigned char* p, int n) {
  if (n >= static_cast<int>(sizeof(V)) / EB) return read_any<V>(p);
  V w{};
  if (n <= 0) return w;
#pragma unroll
  for (int e = 0; e < static_cast<int>(sizeof(V)) / EB; ++e) {
    if (e >= n) continue;
    if constexpr (EB == 4) w[e] = reinterpret_cast<const uint32_t*>(p)[e];
    else if constexpr (EB == 2) w[e / 2] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(p)[e]) << (16 * (e % 2));
    else w[e / 4] |= static_cast<uint32_t>(p[e]) << (8 * (e % 4));
  }
  return w;
}

// Sixteen bytes of a K x N operand's row, or the eight that hold four bf16.
template <int DTYPE>
using Columns4 = typename std::conditional<DTYPE == CLEAVE_BF16, u32x2, u32x4>::type;

template <int DTYPE, bool B_K>
struct Group {   // what a lane holds of a group of k's
  static constexpr int E = Type<DTYPE>::E;
  u32x4 x;
  std::conditional_t<B_K, u32x4, Columns4<DTYPE>> w[B_K ? 4 : E];
};

// Epi: LinearArgs, or GatedArgs: half of a workgroup's waves then read gate's columns and half the same columns of up, so that what a wave
// holds, and what it reads at a time, is as for one operand.
template <int DTYPE, bool B_K, int WAVES, typename Epi>
__global__ __launch_bounds__(64 * WAVES) void few_rows_kernel(ExecuteArgs args, Epi epi, int splits, int64_t chunk) {
  constexpr int E = Type<DTYPE>::E, KG = 4 * E, EB = 16 / E;
  constexpr bool GATED = std::is_same<Epi, GatedArgs>::value;
  constexpr int TURNS = GATED ? WAVES / 2 : WAVES;   // waves that share an operand
  __shared__ float sums[WAVES][kFewRows][kColumns];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, lq = lane >> 4;
  const int64_t M = args.M, N = args.N, K = args.K;
  const int64_t n0 = static_cast<int64_t>(blockIdx.x) * kColumns;
  // this workgroup's chunk of k, of which its waves take every WAVES-th group: what they read at a time lies together.  (A run of
  // groups each, with the weights from memory, us: 8192 x 28672 stored N x K 110 / 96, 4096 x 11008 27.1 / 23.6, K x N 21.2 / 20.8;
  // 8192 x 8192 N x K in two chunks 33 / 36.5, K x N 31.6 / 30.0.)
  const int64_t k0 = blockIdx.y * chunk, k1 = std::min(k0 + chunk, K);
  const int64_t g1 = (k1 - k0 + KG - 1) / KG;

  // rows and columns that are not there repeat the last ones: their sums are not stored, or are the same twice
  const unsigned char* B = static_cast<const unsigned char*>(args.B);
  if constexpr (GATED) {
    if (wave >= TURNS) B = static_cast<const unsigned char*>(epi.b_up);
  }
  const unsigned char* const xp =
      static_cast<const unsigned char*>(args.A) + (std::min<int64_t>(l16, M - 1) * args.lda + E * lq) * EB;
  const int first = static_cast<int>(std::min<int64_t>(4 * l16, std::max<int64_t>(N - 4, 0) - n0));   // of a K x N row's four
  const unsigned char* wp[B_K ? 4 : 1];
  if constexpr (B_K) {
#pragma unroll
    for (int c = 0; c < 4; ++c) wp[c] = B + (std::min<int64_t>(n0 + 16 * c + l16, N - 1) * args.ldb + E * lq) * EB;
  } else {
    wp[0] = B + (n0 + first) * EB;
  }
  typedef Group<DTYPE, B_K> G;
  const auto load = [&](int64_t g, G& to) {
    const int64_t k = k0 + g * KG;          // wave-uniform
    typedef Columns4<DTYPE> C;
    if (k + KG <= k1 && (B_K || N >= 4)) {
      to.x = read_any<u32x4>(xp + k * EB);
      if constexpr (B_K) {
#pragma unroll
        for (int c = 0; c < 4; ++c) to.w[c] = read_any<u32x4>(wp[c] + k * EB);
      } else {
#pragma unroll
        for (int i = 0; i < E; ++i) to.w[i] = read_any<C>(wp[0] + (k + E * lq + i) * args.ldb * EB);
      }
      return;
    }
    // the chunk's last group, or rows of fewer than four: only what is there
    const int left = static_cast<int>(std::min<int64_t>(std::max<int64_t>(k1 - k - E * lq, 0), E));
    to.x = read_some<u32x4, EB>(xp + k * EB, left);
    if constexpr (B_K) {
#pragma unroll
      for (int c = 0; c < 4; ++c) to.w[c] = read_some<u32x4, EB>(wp[c] + k * EB, left);
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i)
        to.w[i] = i < left ? read_some<C, EB>(wp[0] + (k + E * lq + i) * args.ldb * EB, static_cast<int>(std::min<int64_t>(N, 4)))
                           : C{};
    }
  };
  f32x4 acc[4] = {};
  const auto compute = [&](const G& g) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      u32x4 w;
      if constexpr (B_K) {
        w = g.w[c];
      } else if constexpr (DTYPE == CLEAVE_BF16) {
        // column c: the low or high half of word c / 2 of the rows 2p and 2p + 1
#pragma unroll
        for (int p = 0; p < 4; ++p)
          w[p] = __builtin_amdgcn_perm(g.w[2 * p + 1][c / 2], g.w[2 * p][c / 2], c % 2 ? 0x07060302u : 0x05040100u);
      } else {
#pragma unroll
        for (int p = 0; p < 4; ++p) w[p] = g.w[p][c];
      }
      acc[c] = multiply<DTYPE>(g.x, w, acc[c]);
    }
  };
  // the next groups are on their way while one is multiplied
  G set[3];
  int64_t g = GATED ? wave % TURNS : wave;
  if (g < g1) load(g, set[0]);
  if (g + TURNS < g1) load(g + TURNS, set[1]);
  while (g < g1) {
#pragma unroll
    for (int s = 0; s < 3; ++s) {
      if (g >= g1) break;
      if (g + 2 * TURNS < g1) load(g + 2 * TURNS, set[(s + 2) % 3]);
      compute(set[s]);
      g += TURNS;
    }
  }

  // Lane (l16, lq) has rows 4 lq + j of columns first + c (K x N; some may be the workgroup's before) or 16 c + l16 (N x K).
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int col = B_K ? 16 * c + l16 : first + c;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (4 * lq + j < M && col >= 0) sums[wave][4 * lq + j][col] = acc[c][j];
  }
  __syncthreads();
  for (int at = threadIdx.x; at < static_cast<int>(M) * kColumns; at += 64 * WAVES) {
    const int row = at / kColumns, col = at % kColumns;
    const int64_t n = n0 + col;
    if (n >= N) continue;
    float sum = sums[0][row][col];
#pragma unroll
    for (int w = 1; w < TURNS; ++w) sum += sums[w][row][col];
    if constexpr (GATED) {
      float up = sums[TURNS][row][col];
#pragma unroll
      for (int w = TURNS + 1; w < WAVES; ++w) up += sums[w][row][col];
      if (splits > 1) {
        float* p = args.partials + (blockIdx.y * M + row) * 2 * N + n;
        p[0] = sum;
        p[N] = up;
      } else if (args.c_bf16) {
        store_element<true>(args.C, row * args.ldc + n, finish_gated_element<true>(epi, sum, up, row, n));
      } else {
        store_element<false>(args.C, row * args.ldc + n, finish_gated_element<false>(epi, sum, up, row, n));
      }
    } else if (splits > 1) args.partials[(blockIdx.y * M + row) * N + n] = sum;
    else if (args.c_bf16) store_element<true>(args.C, row * args.ldc + n, finish_element<true>(epi, sum, row, n));
    else store_element<false>(args.C, row * args.ldc + n, finish_element<false>(epi, sum, row, n));
  }
}

template <int DTYPE, bool B_K, typename Epi>
hipError_t launch_layout(const ExecuteArgs& args, const Epi& epi, int splits, int64_t chunk, hipStream_t stream) {
  const dim3 g(static_cast<uint32_t>((args.N + kColumns - 1) / kColumns), splits);
  if constexpr (std::is_same<Epi, GatedArgs>::value) {
    // One row, bf16, weights from memory, us, 4, 8, 16 waves: stored K x N, unsplit, 4096 x 11008 39, 36.1, 37.4, 5120 x 13824 60, 54.4, 55.8,
    // 2048 x 16384 33, 25.3, 26.2 (N x K 33, 30.5, 28.6; 1024 x 12000 14.5, 13.3, 13.2); in 4 splits 4096 x 4096 23, 18.7, 19.3,
    // 11008 x 4096 46, 38.3, 38.7, in 2 8192 x 8192 64, 51.6, 52.9.
    constexpr int kWhole = B_K ? 16 : 8;
    if (splits > 1) hipLaunchKernelGGL((few_rows_kernel<DTYPE, B_K, 8, Epi>), g, dim3(512), 0, stream, args, epi, splits, chunk);
    else hipLaunchKernelGGL((few_rows_kernel<DTYPE, B_K, kWhole, Epi>), g, dim3(64 * kWhole), 0, stream, args, epi, splits, chunk);
    return hipGetLastError();
  }
  if (splits > 1) hipLaunchKernelGGL((few_rows_kernel<DTYPE, B_K, 4, Epi>), g, dim3(256), 0, stream, args, epi, splits, chunk);
  else hipLaunchKernelGGL((few_rows_kernel<DTYPE, B_K, 16, Epi>), g, dim3(1024), 0, stream, args, epi, splits, chunk);
  return hipGetLastError();
}
template <typename Epi>
hipError_t launch_few_rows(const ExecuteArgs& args, const Epi& epi, int dtype, int splits, int64_t chunk, hipStream_t stream) {
  if (dtype == CLEAVE_E4M3) return launch_layout<CLEAVE_E4M3, true>(args, epi, splits, chunk, stream);
  if (dtype == CLEAVE_BF16)
    return args.transB ? launch_layout<CLEAVE_BF16, true>(args, epi, splits, chunk, stream)
                       : launch_layout<CLEAVE_BF16, false>(args, epi, splits, chunk, stream);
  return args.transB ? launch_layout<CLEAVE_F32, true>(args, epi, splits, chunk, stream)
                     : launch_layout<CLEAVE_F32, false>(args, epi, splits, chunk, stream);
}

// ---- join ------------------------------------------------------------------------

constexpr int kJoinThreads = 256;
constexpr int kJoinRun = 1024;   // elements of a workgroup where there is no table of runs

// Four neighbouring elements of a row.
template <bool BF16>
struct Quad {
  typedef uint32_t Words2 __attribute__((ext_vector_type(2), aligned(2)));
  typedef float Floats __attribute__((ext_vector_type(4), aligned(4)));
  static __device__ __forceinline__ void load(const void* base, int64_t at, float (&v)[4]) {
    if constexpr (BF16) {
      const Words2 w = *reinterpret_cast<const Words2*>(static_cast<const uint16_t*>(base) + at);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        v[2 * e] = __builtin_bit_cast(float, w[e] << 16);
        v[2 * e + 1] = __builtin_bit_cast(float, w[e] & 0xffff0000u);
      }
    } else {
      const Floats w = *reinterpret_cast<const Floats*>(static_cast<const float*>(base) + at);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = w[e];
    }
  }
  static __device__ __forceinline__ void store(void* base, int64_t at, const float (&v)[4]) {
    if constexpr (BF16) {
      Words2 w;
      w[0] = pack_bf16(v[0], v[1]);
      w[1] = pack_bf16(v[2], v[3]);
      *reinterpret_cast<Words2*>(static_cast<uint16_t*>(base) + at) = w;
    } else {
      *reinterpret_cast<Floats*>(static_cast<float*>(base) + at) = Floats{v[0], v[1], v[2], v[3]};
    }
  }
};

template <bool BF16, bool VEC>
__global__ __launch_bounds__(kJoinThreads) void linear_join_kernel(ReduceArgs args, LinearArgs epi, int64_t M, int64_t N,
                                                                   int splits) {
  for (int64_t it = blockIdx.x; it < args.n_items; it += gridDim.x) {
    uint64_t partial_off, block;
    int64_t m0, n0;
    uint32_t col0, n_len, count;
    int S;
    if (args.items) {
      const ReduceItem item = load_record(args.items, it);
      partial_off = item.partial_off;
      block = item.block;
      m0 = item.m0;
      n0 = item.n0;
      col0 = item.col0;
      n_len = item.n_len;
      count = item.count;
      S = item.ksplit_cnt;
    } else {
      const int64_t first = it * kJoinRun;
      partial_off = first;
      block = M * N;
      m0 = first / N;
      n0 = 0;
      col0 = static_cast<uint32_t>(first % N);
      n_len = static_cast<uint32_t>(N);
      count = static_cast<uint32_t>(std::min<int64_t>(kJoinRun, M * N - first));
      S = splits;
    }
    const float* p = args.partials + partial_off;
    constexpr int W = VEC ? 4 : 1;
    for (uint32_t e = threadIdx.x * W; e < count; e += kJoinThreads * W) {
      const uint32_t r = (col0 + e) / n_len;
      const int64_t row = m0 + r, col = n0 + (col0 + e - r * n_len);
      if constexpr (VEC) {
        f32x4 sum = *reinterpret_cast<const f32x4*>(p + e);
#pragma unroll 8
        for (int s = 1; s < S; ++s) sum = sum + *reinterpret_cast<const f32x4*>(p + s * block + e);
        float t[4] = {sum[0], sum[1], sum[2], sum[3]}, z[4] = {}, bias[4] = {}, scale_b[4] = {};
        if (epi.bias) Quad<false>::load(epi.bias, col, bias);
        if (epi.scale_b) Quad<false>::load(epi.scale_b, col, scale_b);
        if (epi.grad && epi.preact) Quad<BF16>::load(epi.preact, row * epi.ldz + col, z);
        if (epi.scale_a) finish<true>(epi, t, z, bias, scale_b, epi.scale_a[row]);
        else finish<false>(epi, t, z, bias, scale_b, 0.0f);
        if (epi.residual) {
          float residual[4];
          Quad<BF16>::load(epi.residual, row * epi.ldr + col, residual);
#pragma unroll
          for (int k = 0; k < 4; ++k) t[k] += residual[k];
        }
        if (!epi.grad && epi.preact) Quad<BF16>::store(epi.preact, row * epi.ldz + col, z);
        Quad<BF16>::store(args.C, row * args.ldc + col, t);
      } else {
        float sum = p[e];
#pragma unroll 8
        for (int s = 1; s < S; ++s) sum += p[s * block + e];
        store_element<BF16>(args.C, row * args.ldc + col, finish_element<BF16>(epi, sum, row, col));
      }
    }
  }
}

// The same for a gated product (two sums to an element) or its gradient (two outputs).  Without a table an element's sums lie at
// row * pitch + col of each of `splits` blocks.
template <bool BF16, bool GRAD, bool VEC>
__global__ __launch_bounds__(kJoinThreads) void gated_join_kernel(ReduceArgs args, GatedArgs epi, int64_t up_at, int64_t M, int64_t N,
                                                                  int64_t pitch, int splits) {
  constexpr int W = VEC ? 4 : 1, kRun = kJoinThreads * W;   // (one turn of every thread: few rows have few elements)
  for (int64_t it = blockIdx.x; it < args.n_items; it += gridDim.x) {
    ReduceItem item{};
    int64_t first = 0;
    if (args.items) {
      item = load_record(args.items, it);
    } else {
      first = it * kRun;
      item.block = static_cast<uint64_t>(M * pitch);
      item.n_len = static_cast<uint32_t>(N);
      item.m0 = static_cast<uint32_t>(first / N);
      item.col0 = static_cast<uint32_t>(first % N);
      item.count = static_cast<uint32_t>(std::min<int64_t>(kRun, M * N - first));
      item.ksplit_cnt = static_cast<uint32_t>(splits);
    }
    for (uint32_t e = threadIdx.x * W; e < item.count; e += kJoinThreads * W) {
      const uint32_t r = (item.col0 + e) / item.n_len;
      const int64_t row = int64_t{item.m0} + r, col = int64_t{item.n0} + (item.col0 + e - r * item.n_len);
      const float* p = args.partials + (args.items ? static_cast<int64_t>(item.partial_off) + e : row * pitch + col);
      if constexpr (VEC) {
        f32x4 sum = *reinterpret_cast<const f32x4*>(p), other{};
        if constexpr (!GRAD) other = *reinterpret_cast<const f32x4*>(p + up_at);
#pragma unroll 8
        for (uint32_t s = 1; s < item.ksplit_cnt; ++s) {
          sum = sum + *reinterpret_cast<const f32x4*>(p + s * item.block);
          if constexpr (!GRAD) other = other + *reinterpret_cast<const f32x4*>(p + up_at + s * item.block);
        }
        float a[4] = {sum[0], sum[1], sum[2], sum[3]}, b[4] = {other[0], other[1], other[2], other[3]};
        if constexpr (GRAD) {
          float zg[4];
          Quad<BF16>::load(epi.gate, row * epi.ld_gate + col, zg);
          Quad<BF16>::load(epi.up, row * epi.ld_up + col, b);
          finish_gated_grad(static_cast<int>(epi.act), a, zg, b);
          Quad<BF16>::store(epi.second, row * epi.ld_second + col, b);
          Quad<BF16>::store(args.C, row * args.ldc + col, a);
        } else {
          float bg[4] = {}, bu[4] = {}, sg[4] = {}, su[4] = {}, y[4];
          if (epi.bias_gate) Quad<false>::load(epi.bias_gate, col, bg);
          if (epi.bias_up) Quad<false>::load(epi.bias_up, col, bu);
          if (epi.scale_a) {
            Quad<false>::load(epi.scale_gate, col, sg);
            Quad<false>::load(epi.scale_up, col, su);
            finish_gated<true>(static_cast<int>(epi.act), a, b, y, bg, bu, sg, su, epi.scale_a[row]);
          } else {
            finish_gated<false>(static_cast<int>(epi.act), a, b, y, bg, bu, sg, su, 0.0f);
          }
          if (epi.gate) Quad<BF16>::store(epi.gate, row * epi.ld_gate + col, a);
          if (epi.up) Quad<BF16>::store(epi.up, row * epi.ld_up + col, b);
          Quad<BF16>::store(args.C, row * args.ldc + col, y);
        }
      } else {
        float sum = p[0], other = 0.0f;
        if constexpr (!GRAD) other = p[up_at];
#pragma unroll 8
        for (uint32_t s = 1; s < item.ksplit_cnt; ++s) {
          sum += p[s * item.block];
          if constexpr (!GRAD) other += p[up_at + s * item.block];
        }
        if constexpr (GRAD) {
          float a[1] = {sum}, zg[1] = {load_element<BF16>(epi.gate, row * epi.ld_gate + col)},
                b[1] = {load_element<BF16>(epi.up, row * epi.ld_up + col)};
          finish_gated_grad(static_cast<int>(epi.act), a, zg, b);
          store_element<BF16>(epi.second, row * epi.ld_second + col, b[0]);
          store_element<BF16>(args.C, row * args.ldc + col, a[0]);
        } else {
          store_element<BF16>(args.C, row * args.ldc + col, finish_gated_element<BF16>(epi, sum, other, row, col));
        }
      }
    }
  }
}

template <bool GRAD>
hipError_t launch_gated_joined(const ReduceArgs& args, const GatedArgs& epi, int64_t up_at, int64_t M, int64_t N, int splits,
                               int out_dtype, bool vec, hipStream_t stream) {
  ReduceArgs a = args;
  const int run = kJoinThreads * (vec ? 4 : 1);
  if (!a.items) a.n_items = (M * N + run - 1) / run;
  const int64_t pitch = GRAD ? N : 2 * N;
  const dim3 g(static_cast<uint32_t>(std::min<int64_t>(a.n_items, int64_t{1} << 20))), b(kJoinThreads);
  const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, g, b, 0, stream, a, epi, up_at, M, N, pitch, splits); };
  if (out_dtype == CLEAVE_BF16) vec ? launch(gated_join_kernel<true, GRAD, true>) : launch(gated_join_kernel<true, GRAD, false>);
  else vec ? launch(gated_join_kernel<false, GRAD, true>) : launch(gated_join_kernel<false, GRAD, false>);
  return hipGetLastError();
}

// ---- rows in whole sixteen bytes ---------------------------------------------------

// A wave takes 64 kPackGroups groups of a row.
constexpr int kPackGroups = 4;
__global__ __launch_bounds__(256) void pack_kernel(PackArgs args) {
  int64_t row = args.first + static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  int which = 0;
  while (which < args.count && row >= args.matrices[which].rows) row -= args.matrices[which++].rows;
  if (which == args.count) return;
  const PackMatrix m = args.matrices[which];
  const int64_t groups = (m.cols + 7) / 8;
  const Bf16* from = static_cast<const Bf16*>(m.from) + row * m.ld;
  u32x4* to = static_cast<u32x4*>(m.to) + row * groups;
  const int64_t first = static_cast<int64_t>(blockIdx.y) * 64 * kPackGroups + (threadIdx.x & 63);
  Raw16 raw[kPackGroups];
#pragma unroll
  for (int j = 0; j < kPackGroups; ++j) {
    const int64_t g = first + 64 * j;
    raw[j] = Group16<Bf16>::read(from + g * 8, static_cast<int>(max(min(m.cols - g * 8, int64_t{8}), int64_t{0})));
  }
#pragma unroll
  for (int j = 0; j < kPackGroups; ++j)
    if (first + 64 * j < groups) to[first + 64 * j] = raw[j];
}

}  // namespace

hipError_t launch_pack(const PackArgs& args, hipStream_t stream) {
  int64_t rows = 0, groups = 0;
  for (int k = 0; k < args.count; ++k) {
    rows += args.matrices[k].rows;
    groups = std::max(groups, (args.matrices[k].cols + 7) / 8);
  }
  // (a launch has fewer than 2^32 threads)
  const int64_t parts = (groups + 64 * kPackGroups - 1) / (64 * kPackGroups), most = std::max<int64_t>((int64_t{1} << 25) / parts / 4 * 4, 4);
  PackArgs some = args;
  for (some.first = 0; some.first < rows; some.first += most) {
    const dim3 g(static_cast<uint32_t>((std::min(rows - some.first, most) + 3) / 4), static_cast<uint32_t>(parts));
    hipLaunchKernelGGL(pack_kernel, g, dim3(256), 0, stream, some);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_gated_join(const ReduceArgs& args, const GatedArgs& epi, int64_t up_at, int64_t M, int64_t N, int splits,
                             int out_dtype, bool vec, hipStream_t stream) {
  return launch_gated_joined<false>(args, epi, up_at, M, N, splits, out_dtype, vec, stream);
}
hipError_t launch_gated_grad_join(const ReduceArgs& args, const GatedArgs& epi, int64_t M, int64_t N, int splits, int out_dtype,
                                  bool vec, hipStream_t stream) {
  return launch_gated_joined<true>(args, epi, 0, M, N, splits, out_dtype, vec, stream);
}

hipError_t launch_linear_few_rows(const ExecuteArgs& args, const LinearArgs& epi, int dtype, int splits, int64_t chunk,
                                  hipStream_t stream) {
  return launch_few_rows(args, epi, dtype, splits, chunk, stream);
}
hipError_t launch_gated_few_rows(const ExecuteArgs& args, const GatedArgs& epi, int dtype, int splits, int64_t chunk,
                                 hipStream_t stream) {
  return launch_few_rows(args, epi, dtype, splits, chunk, stream);
}

hipError_t launch_linear_join(const ReduceArgs& args, const LinearArgs& epi, int64_t M, int64_t N, int splits, int out_dtype,
                              bool vec, hipStream_t stream) {
  ReduceArgs a = args;
  if (!a.items) a.n_items = (M * N + kJoinRun - 1) / kJoinRun;
  const dim3 g(static_cast<uint32_t>(std::min<int64_t>(a.n_items, int64_t{1} << 20))), b(kJoinThreads);
  const bool bf16 = out_dtype == CLEAVE_BF16;
  if (bf16 && vec) hipLaunchKernelGGL((linear_join_kernel<true, true>), g, b, 0, stream, a, epi, M, N, splits);
  else if (bf16) hipLaunchKernelGGL((linear_join_kernel<true, false>), g, b, 0, stream, a, epi, M, N, splits);
  else if (vec) hipLaunchKernelGGL((linear_join_kernel<false, true>), g, b, 0, stream, a, epi, M, N, splits);
  else hipLaunchKernelGGL((linear_join_kernel<false, false>), g, b, 0, stream, a, epi, M, N, splits);
  return hipGetLastError();
}

}  // namespace cleave
