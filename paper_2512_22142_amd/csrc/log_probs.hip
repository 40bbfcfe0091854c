// Log probabilities of given tokens, with the distribution's entropy and its most likely tokens, and the gradient of the logits
// (what a step does behind its last product; the paper keeps such operators on the parameter server, Sec. 4.1).
//
//   l = a x;  lse = log sum e^l;  logp = l[id] - lse;  H = -sum p log p,  p = e^(l - lse)
// over the columns of each row, a being the scale.  One pass: a thread keeps the largest x so far, m, and, with d = a (x - m),
//   s = sum e^d,  w = sum e^d d     (m -> m': with f = e^(a (m - m')), s' = f s, w' = f (w + a (m - m') s))
// so lse = a m + log s and H = log s - w / s.  An x of minus infinity counts nothing (0 times minus infinity is 0 here).
//
// Gradient:  dx_j = a (dlogp (1[j = id] - p_j) - dH p_j (log p_j + H)).
//
// The most likely tokens: every thread also keeps its strip's first largest value.  Value and column make a 64-bit key, larger for a larger
// value or a lower column, so no two are equal.  The k-th largest of the threads' keys is a bound that at least k elements
// reach, and only the strips of the k threads that reach it hold such: those are read again, and their elements ranked.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "operators.h"
#include "row_access.h"
#include "wave_reduce.h"

namespace cleave {

namespace {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
constexpr float kInf = __builtin_inff();

// Minus infinity becomes a number, so that zero times it is zero.  (NaN becomes one too: beside it the exponential is NaN.)
__device__ __forceinline__ float floored(float x) { return __builtin_fmaxf(x, -1e30f); }

// A part of a row: its largest x, and the sums relative to it, w in units of log 2.
struct Stats {
  float m, s, w;
};
// Moves the sums to another, larger m.  (Without any value yet they are zero.)
__device__ __forceinline__ void move_to(Stats& a, float m, float c) {
  if (a.m > -kInf) {
    const float by = c * (a.m - m), f = __builtin_amdgcn_exp2f(by);
    a.w = f * (a.w + a.s * floored(by));
    a.s *= f;
  }
  a.m = m;
}
__device__ __forceinline__ Stats join(Stats a, Stats b, float c) {
  const float m = __builtin_fmaxf(a.m, b.m);
  if (m > -kInf) {
    // (equal ones stay: infinite ones would make NaN of what is left, which is what their sums are already)
    if (a.m != m) move_to(a, m, c);
    if (b.m != m) move_to(b, m, c);
  }
  return {m, a.s + b.s, a.w + b.w};
}

// ---- keys of the order -----------------------------------------------------------

typedef uint64_t Key;   // 0: none
__device__ __forceinline__ Key key_of(float x, uint32_t col) {
  x = x == x ? x + 0.0f : -kInf;   // (-0 is 0; NaN counts as minus infinity)
  const uint32_t b = __builtin_bit_cast(uint32_t, x);
  return static_cast<Key>(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | static_cast<uint32_t>(~col);
}
__device__ __forceinline__ uint32_t column_of(Key k) { return ~static_cast<uint32_t>(k); }
__device__ __forceinline__ float value_of(Key k) {
  const uint32_t b = static_cast<uint32_t>(k >> 32);
  return __builtin_bit_cast(float, b & 0x80000000u ? b & 0x7fffffffu : ~b);
}
// A wave's keys in descending order of lanes (bitonic).
__device__ __forceinline__ Key sort_wave(Key k) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int size = 2; size <= 64; size <<= 1)
#pragma unroll
    for (int d = size / 2; d > 0; d >>= 1) {
      const Key other = static_cast<Key>(__shfl_xor(static_cast<uint32_t>(k >> 32), d)) << 32 | __shfl_xor(static_cast<uint32_t>(k), d);
      const bool larger = ((lane & d) == 0) == ((lane & size) == 0);
      k = larger == (k > other) ? k : other;
    }
  return k;
}

constexpr int kCandidates = 2048;   // held in LDS at a time

template <int NW>
struct TopSpace {
  Key lists[NW][kMostTop];   // the waves' largest keys
  Key found[kCandidates];
  Key best[kMostTop];
  Key bound;
  int count;
};

// The `n` keys of `found` that are largest go to `best`, in order.
__device__ __forceinline__ void rank_keys(const Key* found, int count, Key* best, int n, int threads) {
  for (int i = threadIdx.x; i < count; i += threads) {
    const Key mine = found[i];
    int rank = 0;
    for (int j = 0; j < count; ++j) rank += found[j] > mine;
    if (rank < n) best[rank] = mine;
  }
}

// space.best: the largest `n` keys of the workgroup's elements; zeros where there are fewer.  `mine`: this thread's largest, `push`:
// (first, groups, take) calls take(key) for the elements of that many of this thread's groups, of `strip` at most.
template <int NT, int N, typename Push>
__device__ __forceinline__ void find_top(TopSpace<NT / 64>& space, Key mine, int n, int strip, Push push) {
  constexpr int NW = NT / 64;
  const int t = threadIdx.x, lane = t & 63;
  const Key sorted = sort_wave(mine);
  if (lane < n) space.lists[t >> 6][lane] = sorted;
  if (t == 0) {
    space.bound = 0;
    space.count = 0;
  }
  if (t < n) space.best[t] = 0;
  __syncthreads();
  for (int i = t; i < NW * n; i += NT) {
    const Key k = space.lists[i / n][i % n];
    int rank = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      // larger ones in a descending list
      int lo = 0;
#pragma unroll
      for (int d = kMostTop; d > 0; d >>= 1)
        if (lo + d <= n && space.lists[w][lo + d - 1] > k) lo += d;
      rank += lo;
    }
    if (rank == n - 1 && k) space.bound = k;
  }
  __syncthreads();
  const Key bound = space.bound;
  const bool reaches = mine && mine >= bound;
  // at most n threads reach it: as many groups at a time as fit beside the best so far
  const int some = max(1, (kCandidates / n - 1) / N);
  for (int first = 0; first < strip; first += some) {
    if (reaches)
      push(first, min(some, strip - first), [&](Key k) {
        if (k >= bound) space.found[atomicAdd(&space.count, 1)] = k;
      });
    __syncthreads();
    const int count = space.count;
    rank_keys(space.found, count, space.best, n, NT);
    __syncthreads();
    if (first + some < strip) {
      const int have = min(count, n);
      if (t < have) space.found[t] = space.best[t];
      if (t == 0) space.count = have;
      __syncthreads();
    }
  }
}

// ---- one pass over a row, or a part of it --------------------------------------------

// What is known of a whole row goes out.
__device__ __forceinline__ float log_prob(const LogProbArgs& args, float x, const Stats& all, float log_s) {
  return all.s == 0.0f ? -kInf : args.scale * (x - all.m) - log_s;   // (nothing left: every logit is minus infinity)
}
template <typename T>
__device__ __forceinline__ void put_row(const LogProbArgs& args, int64_t row, const Stats& all, float log_s) {
  const bool none = all.s == 0.0f;
  if (args.lse) args.lse[row] = none ? -kInf : args.scale * all.m + log_s;
  if (args.entropy) {
    const float h = log_s - kLn2 * all.w / all.s;
    args.entropy[row] = none || h < 0.0f ? 0.0f : h;
  }
  if (args.logp) {
    const int64_t id = args.ids[row];
    float p = 0.0f;   // no token
    if (id >= args.cols) p = __builtin_nanf("");
    else if (id >= 0) p = log_prob(args, element(static_cast<const T*>(args.logits) + row * args.ld + id), all, log_s);
    args.logp[row] = p;
  }
}
__device__ __forceinline__ void put_top(const LogProbArgs& args, int64_t row, int k, Key key, const Stats& all, float log_s) {
  args.top_ids[row * args.n_top + k] = column_of(key);
  // (a row with a NaN or an infinity: s is NaN)
  args.top_logp[row * args.n_top + k] = log_prob(args, value_of(key), all, log_s);
}

// Floats of a part's record: m, s, w, then n_top keys.
__host__ __device__ inline int record_floats(int n_top) { return 4 + 2 * n_top; }

// Groups of sixteen bytes that a thread has on their way at a time.
constexpr int kAhead = 4;

template <typename T, int NT, bool TOP, bool ENTROPY>
__global__ __launch_bounds__(NT) void log_probs_kernel(LogProbArgs args) {
  typedef Group16<T> G;
  constexpr int N = G::N, NW = NT / 64, U = kAhead;
  __shared__ Stats slots[NW];
  const int t = threadIdx.x;
  const int64_t row = blockIdx.x / static_cast<uint32_t>(args.parts);
  const int part = static_cast<int>(blockIdx.x % static_cast<uint32_t>(args.parts));
  const int first = part * args.chunk;   // below cols
  const int len = static_cast<int>(min(static_cast<int64_t>(args.chunk), args.cols - first));
  const T* x = static_cast<const T*>(args.logits) + row * args.ld + first;
  const float c = args.scale * kLog2e;
  const int groups = (len + N - 1) / N;

  Stats own{-kInf, 0.0f, 0.0f};
  float best = -kInf;
  int best_at = t * N;
  for (int g = t; g < groups; g += U * NT) {
    Raw16 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = G::read(x + static_cast<int64_t>(g + u * NT) * N, len - (g + u * NT) * N);
    float v[U][N];
    float most = -kInf;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      G::unpack(raw[u], v[u]);
      const int at = (g + u * NT) * N;
      if (at + N > len) {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (at + e >= len) v[u][e] = -kInf;
      }
      float here = v[u][0];
#pragma unroll
      for (int e = 1; e < N; ++e) here = __builtin_fmaxf(here, v[u][e]);
      if constexpr (TOP) {
        if (here > best) {
          best = here;
          int e0 = N - 1;
#pragma unroll
          for (int e = N - 2; e >= 0; --e)
            if (v[u][e] == here) e0 = e;
          best_at = at + e0;
        }
      }
      most = __builtin_fmaxf(most, here);
    }
    if (most > own.m) move_to(own, most, c);
    const float m = own.m > -kInf ? own.m : 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float d = c * (v[u][e] - m), p = __builtin_amdgcn_exp2f(d);
        own.s += p;
        if constexpr (ENTROPY) own.w += p * floored(d);
      }
  }
  Stats all = own;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) all = join(all, {__shfl_xor(all.m, d), __shfl_xor(all.s, d), __shfl_xor(all.w, d)}, c);
  if ((t & 63) == 0) slots[t >> 6] = all;
  __syncthreads();
  all = slots[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) all = join(all, slots[w], c);
  const float log_s = __builtin_logf(all.s);
  float* record = args.workspace + static_cast<int64_t>(blockIdx.x) * record_floats(args.n_top);
  if (t == 0) {
    if (args.parts == 1) {
      put_row<T>(args, row, all, log_s);
    } else {
      record[0] = all.m;
      record[1] = all.s;
      record[2] = all.w;
    }
  }
  if constexpr (TOP) {
    __shared__ TopSpace<NW> space;
    const Key mine = t < groups ? key_of(best, first + best_at) : 0;
    find_top<NT, N>(space, mine, args.n_top, (groups + NT - 1) / NT, [&](int j0, int count, auto take) {
      for (int j = j0; j < j0 + count; ++j) {
        const int at = (t + j * NT) * N;
        if (at >= len) break;
        float v[N];
        G::unpack(G::read(x + at, len - at), v);
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (at + e < len) take(key_of(v[e], first + at + e));
      }
    });
    if (t < args.n_top) {
      const Key k = space.best[t];
      if (args.parts == 1) {
        put_top(args, row, t, k, all, log_s);
      } else {
        uint32_t* words = reinterpret_cast<uint32_t*>(record) + 4 + 2 * t;
        words[0] = static_cast<uint32_t>(k);
        words[1] = static_cast<uint32_t>(k >> 32);
      }
    }
  }
}

// The parts of a row.
constexpr int kJoinThreads = 256;
template <typename T>
__global__ __launch_bounds__(kJoinThreads) void log_probs_join_kernel(LogProbArgs args) {
  __shared__ Key found[kMostParts * kMostTop], best[kMostTop];
  const int64_t row = blockIdx.x;
  const int stride = record_floats(args.n_top);
  const float* records = args.workspace + row * args.parts * stride;
  const float c = args.scale * kLog2e;
  Stats all{records[0], records[1], records[2]};
  for (int p = 1; p < args.parts; ++p) all = join(all, {records[p * stride], records[p * stride + 1], records[p * stride + 2]}, c);
  const float log_s = __builtin_logf(all.s);
  if (threadIdx.x == 0) put_row<T>(args, row, all, log_s);
  if (args.n_top == 0) return;
  const int count = args.parts * args.n_top;
  for (int i = threadIdx.x; i < count; i += kJoinThreads) {
    const uint32_t* words = reinterpret_cast<const uint32_t*>(records + (i / args.n_top) * stride) + 4 + 2 * (i % args.n_top);
    found[i] = static_cast<Key>(words[1]) << 32 | words[0];
  }
  __syncthreads();
  rank_keys(found, count, best, args.n_top, kJoinThreads);
  __syncthreads();
  if (static_cast<int>(threadIdx.x) < args.n_top) put_top(args, row, threadIdx.x, best[threadIdx.x], all, log_s);
}

template <typename T, int NT>
hipError_t launch_rows(const LogProbArgs& args, hipStream_t stream) {
  const dim3 g(static_cast<uint32_t>(args.rows * args.parts)), b(NT);
  if (args.n_top > 0) {
    if (args.entropy) hipLaunchKernelGGL((log_probs_kernel<T, NT, true, true>), g, b, 0, stream, args);
    else hipLaunchKernelGGL((log_probs_kernel<T, NT, true, false>), g, b, 0, stream, args);
  } else {
    if (args.entropy) hipLaunchKernelGGL((log_probs_kernel<T, NT, false, true>), g, b, 0, stream, args);
    else hipLaunchKernelGGL((log_probs_kernel<T, NT, false, false>), g, b, 0, stream, args);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || args.parts == 1) return e;
  hipLaunchKernelGGL((log_probs_join_kernel<T>), dim3(static_cast<uint32_t>(args.rows)), dim3(kJoinThreads), 0, stream, args);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_of(const LogProbArgs& args, hipStream_t stream) {
  if (args.rows * args.parts > 1024) return launch_rows<T, 256>(args, stream);
  return launch_rows<T, 1024>(args, stream);
}

// ---- gradient ------------------------------------------------------------------

constexpr int kGradThreads = 256;
constexpr int kGradGroups = 4;   // of sixteen bytes, of a thread

template <typename T>
__global__ __launch_bounds__(kGradThreads) void log_probs_backward_kernel(LogProbBackwardArgs args) {
  typedef Group16<T> G;
  constexpr int N = G::N;
  const int64_t row = blockIdx.x / static_cast<uint32_t>(args.parts);
  const int part = static_cast<int>(blockIdx.x % static_cast<uint32_t>(args.parts));
  const int cols = static_cast<int>(args.cols);
  const T* x = static_cast<const T*>(args.logits) + row * args.ld;
  T* dx = static_cast<T*>(args.dlogits) + row * args.ldd;
  const int64_t first = int64_t{part} * kGradThreads * kGradGroups * N;
  Raw16 raw[kGradGroups];
#pragma unroll
  for (int u = 0; u < kGradGroups; ++u) {
    const int64_t at = first + (u * kGradThreads + threadIdx.x) * N;
    raw[u] = G::read(x + at, static_cast<int>(max(int64_t{cols} - at, int64_t{0})));
  }
  const float lse = args.lse[row];
  float d = 0.0f, dh = 0.0f, h = 0.0f;
  int64_t id = -1;
  if (args.ids) {
    id = args.ids[row];
    if (id >= 0) d = id < args.cols ? args.dlogp[row] : __builtin_nanf("");
  }
  if (args.entropy) {
    h = args.entropy[row];
    dh = args.dentropy[row];
  }
  const bool none = lse == -kInf;   // nothing left
#pragma unroll
  for (int u = 0; u < kGradGroups; ++u) {
    const int64_t at = first + (u * kGradThreads + threadIdx.x) * N;
    if (at >= cols) break;
    float v[N];
    G::unpack(raw[u], v);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float logp = __builtin_fmaf(args.scale, v[e], -lse), p = __builtin_amdgcn_exp2f(kLog2e * logp);
      float g = -p * (d + dh * (floored(logp) + h));
      if (none) g = 0.0f * d;
      if (at + e == id) g = none ? g : g + d;
      v[e] = args.scale * g;
    }
    G::store(dx + at, static_cast<int>(cols - at), v);
  }
}

}  // namespace

// A launch has fewer than 2^32 threads.
constexpr int64_t kLaunchWorkgroups = int64_t{1} << 21;

// Parts of a row: one, but where few rows leave most CUs idle and a row is long.
int log_probs_parts(int64_t rows, int64_t cols) {
  if (rows > 64) return 1;
  const int64_t parts = std::min<int64_t>({cols / 16384, 256 / std::max<int64_t>(rows, 1), kMostParts});
  return static_cast<int>(cols >= 131072 && parts > 1 ? parts : 1);
}

hipError_t launch_log_probs(const LogProbArgs& args, int dtype, hipStream_t stream) {
  const int64_t eb = dtype == CLEAVE_BF16 ? 2 : 4;
  const int64_t most = kLaunchWorkgroups / args.parts;
  for (int64_t row = 0; row < args.rows; row += most) {
    LogProbArgs some = args;
    some.rows = std::min(args.rows - row, most);
    some.logits = static_cast<const unsigned char*>(args.logits) + row * args.ld * eb;
    if (args.ids) some.ids += row;
    if (args.logp) some.logp += row;
    if (args.lse) some.lse += row;
    if (args.entropy) some.entropy += row;
    if (args.n_top) {
      some.top_ids += row * args.n_top;
      some.top_logp += row * args.n_top;
    }
    const hipError_t e = dtype == CLEAVE_BF16 ? launch_of<Bf16>(some, stream) : launch_of<float>(some, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_log_probs_backward(const LogProbBackwardArgs& args, int dtype, hipStream_t stream) {
  const int64_t eb = dtype == CLEAVE_BF16 ? 2 : 4, n = dtype == CLEAVE_BF16 ? Group16<Bf16>::N : Group16<float>::N;
  const int64_t of_workgroup = kGradThreads * kGradGroups * n, parts = (args.cols + of_workgroup - 1) / of_workgroup;
  const int64_t most = std::max<int64_t>(1, (int64_t{1} << 23) / parts);
  for (int64_t row = 0; row < args.rows; row += most) {
    LogProbBackwardArgs some = args;
    some.rows = std::min(args.rows - row, most);
    some.parts = static_cast<int>(parts);
    some.logits = static_cast<const unsigned char*>(args.logits) + row * args.ld * eb;
    some.dlogits = static_cast<unsigned char*>(args.dlogits) + row * args.ldd * eb;
    some.lse += row;
    if (args.ids) {
      some.ids += row;
      some.dlogp += row;
    }
    if (args.entropy) {
      some.entropy += row;
      some.dentropy += row;
    }
    const dim3 g(static_cast<uint32_t>(some.rows * parts)), b(kGradThreads);
    if (dtype == CLEAVE_BF16) hipLaunchKernelGGL((log_probs_backward_kernel<Bf16>), g, b, 0, stream, some);
    else hipLaunchKernelGGL((log_probs_backward_kernel<float>), g, b, 0, stream, some);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace cleave
