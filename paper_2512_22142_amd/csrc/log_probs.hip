// Log probabilities of given tokens, with the distribution's entropy and its most likely tokens, and the gradient of the logits
// (what a step does behind its last product; the paper keeps such operators on the parameter server, Sec. 4.1).
//
//   l = a x;  lse = log sum e^l;  logp = l[id] - lse;  H = -sum p log p,  p = e^(l - lse)
// over the columns of each row, a being the scale.  One pass: a thread keeps the largest x so far, m, and, with d = a (x - m),
//   s = sum e^d,  w = sum e^d d     (m -> m': with f = e^(a (m - m')), s' = f s, w' = f (w + a (m - m') s))
// so lse = a m + log s and H = log s - w / s.  An x of minus infinity counts nothing (0 times minus infinity is 0 here).
//
// Gradient:  dx_j = a (dlogp (1[j = id] - p_j) - dH p_j (log p_j + H)), p from lse where fp32 holds that well enough, else from the row.
//
// The most likely tokens: every thread also keeps its strip's first largest value.  Value and column make a 64-bit key, larger for a larger
// value or a lower column, so no two are equal.  The k-th largest of the keys of groups of threads is a bound that at least k elements
// reach, and only the strips of the few threads that reach it hold such: those are read again, and their elements ranked.
//
// Bound by memory, one read of the logits (the gradient: one read and one write), us:
//   8192 x 32000 bf16 with entropy 100-104 (5.2 TB/s), the gradient 178-190 (5.5-5.9), the one behind the other 275-284 (the second finds
//   a part of the logits in the Infinity Cache)
//   3001 x 50257 fp32 with five tokens 109 (5.5 TB/s)
//   1 x 32000 with twenty tokens 10.7, of them 3 a launch, 4 the row, the rest the order
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "kernels.h"
#include "operators.h"
#include "row_access.h"
#include "wave_reduce.h"

namespace cleave {

namespace {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
constexpr float kInf = __builtin_inff();

// Minus infinity becomes a number, so that zero times it is zero; below -150 the exponential beside it is zero already.  (NaN becomes one
// too: beside it the exponential is NaN.)
__device__ __forceinline__ float floored(float x) { return __builtin_fmaxf(x, -1e4f); }

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
__device__ __forceinline__ Key shuffle_xor(Key k, int d) {
  return static_cast<Key>(__shfl_xor(static_cast<uint32_t>(k >> 32), d)) << 32 | __shfl_xor(static_cast<uint32_t>(k), d);
}

constexpr int kCandidates = 1024;   // held in LDS at a time

template <int NT>
struct TopSpace {
  Key largest[64];           // the largest keys of 64 groups of neighbouring threads
  Key found[kCandidates];
  Key best[kMostTop];
  uint16_t reach[NT];        // threads whose strips reach the bound
  int count, reaching;
};

// How many of `list` (`count` keys, zeros behind them to a multiple of eight) are larger than `mine`.
__device__ __forceinline__ int larger_than(const Key* list, int count, Key mine) {
  int rank = 0;
  for (int j = 0; j < count; j += 8) {
#pragma unroll
    for (int i = 0; i < 8; ++i) rank += list[j + i] > mine;
  }
  return rank;
}

// space.best: the largest `n` keys of the workgroup's elements; zeros where there are fewer.  `mine`: this thread's largest;
// look(reaching, bound, take) calls take(key) once, from any thread, for every element that reaches the bound in the strips of the first
// `reaching` threads of space.reach.
//   The bound, which at least n elements reach: the n-th largest of the largest keys of 64 groups of threads; every wave finds it
// itself (the rank of a lane's key by 64 reads).  Random logits leave some 1.4 n candidates, in the strips of as many threads, which all
// threads share out among them.  Where more reach the bound than LDS holds (logits in an order that the strips follow), the n-th
// largest of those that were held is the next bound: each round leaves out all that the last one held but n.
template <int NT, typename Look>
__device__ __forceinline__ void find_top(TopSpace<NT>& space, Key mine, int n, Look look) {
  constexpr int kGroup = NT / 64;
  static_assert(kCandidates % 8 == 0 && kGroup >= 1, "whole eights");
  const int t = threadIdx.x, lane = t & 63;
  Key most = mine;
#pragma unroll
  for (int d = kGroup / 2; d > 0; d >>= 1) {
    const Key other = shuffle_xor(most, d);
    most = other > most ? other : most;
  }
  if (t % kGroup == 0) space.largest[t / kGroup] = most;
  if (t < n) space.best[t] = 0;
  if (t == 0) space.count = space.reaching = 0;
  __syncthreads();
  const Key group = space.largest[lane];
  const uint64_t is = __ballot(larger_than(space.largest, 64, group) == n - 1 && group != 0);
  Key bound = 1;   // fewer groups than n have an element: all of them
  if (is) {
    const int at = __builtin_ctzll(is);
    bound = static_cast<Key>(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<uint32_t>(group >> 32), at))) << 32 |
            static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<uint32_t>(group), at));
  }
  if (mine >= bound) space.reach[atomicAdd(&space.reaching, 1)] = static_cast<uint16_t>(t);
  __syncthreads();
  const int reaching = space.reaching;
  for (;;) {
    look(reaching, bound, [&](Key k) {
      const int at = atomicAdd(&space.count, 1);
      if (at < kCandidates) space.found[at] = k;
    });
    __syncthreads();
    const int all = space.count, count = min(all, kCandidates);
    if (t < (8 - (count & 7)) % 8) space.found[count + t] = 0;
    __syncthreads();
    for (int i = t; i < count; i += NT) {
      const Key k = space.found[i];
      const int rank = larger_than(space.found, count, k);
      if (rank < n) space.best[rank] = k;
    }
    if (t == 0) space.count = 0;
    __syncthreads();
    if (all <= kCandidates) return;
    bound = space.best[n - 1];
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

// The largest of three.  (As one instruction: the compiler would first make quiet NaN of what is loaded.  A signaling one may become the
// largest, beside which the sums are NaN; its neighbours' places in the order are then open.)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// U: groups of sixteen bytes of a thread that are taken together, while as many more are on their way.
template <typename T, int NT, int U, bool TOP, bool ENTROPY>
__global__ __launch_bounds__(NT) void log_probs_kernel(LogProbArgs args) {
  typedef Group16<T> G;
  constexpr int N = G::N, NW = NT / 64;
  __shared__ Stats slots[NW];
  const int t = threadIdx.x;
  const int64_t row = blockIdx.x / static_cast<uint32_t>(args.parts);
  const int part = static_cast<int>(blockIdx.x % static_cast<uint32_t>(args.parts));
  const int first = part * args.chunk;   // below cols
  const int len = static_cast<int>(min(static_cast<int64_t>(args.chunk), args.cols - first));
  const T* x = static_cast<const T*>(args.logits) + row * args.ld + first;
  const float c = args.scale * kLog2e;
  const int groups = (len + N - 1) / N, whole = len / N;
  // A row's last group, where it is not whole, is read so that it ends with the row; what the one before it has is left out.  (Fewer
  // elements than a group are read one by one.)
  const auto place = [&](int g) { return min(g * N, max(len - N, 0)); };
  const auto read = [&](int g) { return len >= N ? G::read(x + place(g), N) : G::read(x, len); };

  Stats own{-kInf, 0.0f, 0.0f};
  float best = -kInf;
  int best_at = t * N;   // the first one that counts
  const auto take = [&](const Raw16 (&raw)[U], int g, auto ragged_tag) {
    constexpr bool RAGGED = decltype(ragged_tag)::value;
    float v[U][N], most = -kInf;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      G::unpack(raw[u], v[u]);
      const int i = g + u * NT;
      int at = i * N;
      if constexpr (RAGGED) {
        at = place(i);
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (i >= groups || at + e < i * N || at + e >= len) v[u][e] = -kInf;
      }
      float here = max3(v[u][0], v[u][1], v[u][2]);
#pragma unroll
      for (int e = 3; e < N; e += 2) here = e + 1 < N ? max3(here, v[u][e], v[u][e + 1]) : __builtin_fmaxf(here, v[u][e]);
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
    float s[2] = {}, w[2] = {};
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float d = c * (v[u][e] - m), p = __builtin_amdgcn_exp2f(d);
        s[e % 2] += p;
        if constexpr (ENTROPY) w[e % 2] += p * floored(d);
      }
    own.s += s[0] + s[1];
    if constexpr (ENTROPY) own.w += w[0] + w[1];
  };
  constexpr std::true_type yes{};
  constexpr std::false_type no{};
  int g = t;
  const int rounds = whole / (U * NT);   // of whole groups in every thread
  Raw16 raw[U], next[U];
  const auto fetch = [&](int from, Raw16 (&to)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u) to[u] = G::read(x + static_cast<int64_t>(from + u * NT) * N, N);
  };
  const auto fetch_ragged = [&](int from, Raw16 (&to)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u) to[u] = read(min(from + u * NT, groups - 1));
  };
  const bool rest = rounds * U * NT < groups;
  if (rounds > 0) {
    fetch(g, raw);
    for (int r = 1; r < rounds; ++r) {
      fetch(g + U * NT, next);
      take(raw, g, no);
#pragma unroll
      for (int u = 0; u < U; ++u) raw[u] = next[u];
      g += U * NT;
    }
    if (rest) fetch_ragged(g + U * NT, next);
    take(raw, g, no);
    g += U * NT;
  } else {
    fetch_ragged(g, next);
  }
  if (rest) take(next, g, yes);

  // the wave's, then the waves'
  const float of_wave = wave_join(own.m, [](float a, float b) { return __builtin_fmaxf(a, b); });
  if (own.m != of_wave) move_to(own, of_wave, c);
  Stats all{of_wave, wave_total(own.s), ENTROPY ? wave_total(own.w) : 0.0f};
  if constexpr (NW > 1) {
    if ((t & 63) == 0) slots[t >> 6] = all;
    __syncthreads();
    all = slots[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) all = join(all, slots[w], c);
  }
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
    __shared__ TopSpace<NT> space;
    const Key mine = t < groups ? key_of(best, first + best_at) : 0;
    const uint32_t strip = (groups + NT - 1) / NT;
    find_top<NT>(space, mine, args.n_top, [&](uint32_t reaching, Key bound, auto take_key) {
      const float least = value_of(bound);   // (of a bound that nothing sets: NaN, which is no bound)
      const uint32_t count = reaching * strip;
      for (uint32_t i = t; i < count; i += U * NT) {
        int at_group[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const uint32_t k = min(i + u * NT, count - 1), j = k / reaching;
          at_group[u] = space.reach[k - j * reaching] + j * NT;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = read(min(at_group[u], groups - 1));
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (i + u * NT >= count || at_group[u] >= groups) continue;
          float v[N];
          G::unpack(raw[u], v);
          float here = v[0];
#pragma unroll
          for (int e = 1; e < N; ++e) here = __builtin_fmaxf(here, v[e]);
          if (here < least) continue;
          const int at = place(at_group[u]);
#pragma unroll
          for (int e = 0; e < N; ++e)
            if (at + e >= at_group[u] * N && at + e < len) {
              const Key k = key_of(v[e], first + at + e);
              if (k >= bound) take_key(k);
            }
        }
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
  __shared__ Key found[kMostParts * kMostTop + 8], best[kMostTop];
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
  if (threadIdx.x < 8) found[count + threadIdx.x] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < count; i += kJoinThreads) {
    const Key k = found[i];
    const int rank = larger_than(found, count, k);
    if (rank < args.n_top) best[rank] = k;
  }
  __syncthreads();
  if (static_cast<int>(threadIdx.x) < args.n_top) put_top(args, row, threadIdx.x, best[threadIdx.x], all, log_s);
}

template <typename T, int NT, int U = 4>
hipError_t launch_rows(const LogProbArgs& args, hipStream_t stream) {
  const dim3 g(static_cast<uint32_t>(args.rows * args.parts)), b(NT);
  if (args.n_top > 0) {
    if (args.entropy) hipLaunchKernelGGL((log_probs_kernel<T, NT, U, true, true>), g, b, 0, stream, args);
    else hipLaunchKernelGGL((log_probs_kernel<T, NT, U, true, false>), g, b, 0, stream, args);
  } else {
    if (args.entropy) hipLaunchKernelGGL((log_probs_kernel<T, NT, U, false, true>), g, b, 0, stream, args);
    else hipLaunchKernelGGL((log_probs_kernel<T, NT, U, false, false>), g, b, 0, stream, args);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || args.parts == 1) return e;
  hipLaunchKernelGGL((log_probs_join_kernel<T>), dim3(static_cast<uint32_t>(args.rows)), dim3(kJoinThreads), 0, stream, args);
  return hipGetLastError();
}

// Threads of a row.  Rows that fill the chip take few, whose sums are joined without a barrier (one wave) or a short one; few
// rows take more, whose latency counts.  us, 64, 128, 256, 512, 1024 threads:
//   bf16 with entropy   16384 x 1024 19, 33, 55, 106, 239; 8192 x 8192 27, 27, 29, 65, 146; 8192 x 32000 98, 103, 100, 117, 182
//                       1 x 8192 5.5, 4.8, 5.0, 6.2, 7.6; 1 x 32000 15, 10, 7.5, 7.3, 8.5; 256 x 32000 15, 10, 8.4, 8.9, 10
//   with twenty tokens  16384 x 4096 (five) 44, 50, 95, 217, 632; 1100 x 32000 45, 31, 29, 32, 64; 3001 x 50257 fp32 200, 175, 143, 124, 135
//                       1 x 8192 12.8, 8.9, 7.8, 9.7, 12.1; 1 x 32000 31, 18, 12.9, 11.7, 13.4
// Short rows take fewer groups together, since what is not there costs as much as what is: one up to 64 groups, two up to 128.  bf16, 64
// threads, four groups and as here (with eight tokens):
//                       16384 x 1024 15.3, 9.7 (36.9, 27.2); 16384 x 512 13.6, 7.2 (34.0, 24.0); 65536 x 128 43, 23.8 (123, 93)
template <typename T>
hipError_t launch_of(const LogProbArgs& args, hipStream_t stream) {
  const int64_t groups = (args.chunk + Group16<T>::N - 1) / Group16<T>::N;
  const bool many = args.rows * args.parts > 1024;
  if (many && groups <= 64) return launch_rows<T, 64, 1>(args, stream);
  if (many && groups <= 128) return launch_rows<T, 64, 2>(args, stream);
  if (many && groups <= 1024) return launch_rows<T, 64>(args, stream);
  if (groups <= (args.n_top > 0 && !many ? 1024 : 4096) || (many && args.n_top == 0)) return launch_rows<T, 256>(args, stream);
  return launch_rows<T, 512>(args, stream);
}

// ---- gradient ------------------------------------------------------------------

// Far rows.  p = e^(l - lse) is as good as the fp32 lse, which holds the less of log s the further it lies from zero: of a row masked by -1e9
// nothing.  From |lse| = kNear on, where it leaves p good to 2^-16, m and s are taken again from the row and p = e^(a (x - m) - log s).  All
// rows near, all far, us: 8192 x 32000 bf16 187, 378, fp32 386, 635; 16384 x 1024 bf16 16.2, 20.0; 1 x 32000 bf16 4.2, 16.1.
constexpr float kNear = 256.0f;
// Whose logits all lie below this has no token left: they are masked, by minus infinity or by the type's lowest value.  (Such rows are far at
// any scale from kLeastScale on; below it all are taken as far.)
constexpr float kMasked = -1e30f, kLeastScale = 0x1p-80f;
constexpr float kLargest = 0x1p100f;

// The gradient of such a row by NT threads, one workgroup's or a wave's.  A thread has the same groups in both passes, so that dx may lie over
// x.  give(log p, column, whether the row has tokens left): the gradient.
template <typename T, int NT, typename Give>
__device__ __forceinline__ void backward_far(const LogProbBackwardArgs& args, int64_t row, int t, Give give) {
  typedef Group16<T> G;
  constexpr int N = G::N, NW = RowGroup<NT>::kWaves;
  __shared__ float slots[2][NW];
  const T* x = static_cast<const T*>(args.logits) + row * args.ld;
  T* dx = static_cast<T*>(args.dlogits) + row * args.ldd;
  const int cols = static_cast<int>(args.cols);
  const auto walk = [&](auto visit) {   // visit(values, column of the first, how many there are)
#pragma unroll 1
    for (int at = t * N; at < cols; at += NT * N) {
      float v[N];
      G::unpack(G::read(x + at, cols - at), v);
      visit(v, at, cols - at);
    }
  };
  const auto larger = [](float a, float b) { return __builtin_fmaxf(a, b); };
  const auto power = [&](float d) { return __builtin_amdgcn_exp2f(kLog2e * (args.scale * d)); };
  float own = -kInf, s = 0.0f;
  walk([&](float (&v)[N], int, int left) {
    float most = v[0];
#pragma unroll
    for (int e = 1; e < N; ++e) {
      if (e >= left) v[e] = -kInf;
      most = larger(most, v[e]);
    }
    if (most > own) {
      s *= power(own - most);
      own = most;
    }
    const float from = own > -kInf ? own : 0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) s += power(v[e] - from);
  });
  const float m = join_waves<NW>(wave_join(own, larger), slots[0], larger);
  if (own != m) s *= power(own - m);   // (an infinite one stays: its sum is NaN)
  const float log_s = __builtin_logf(group_total<NT>(s, slots[1]));
  walk([&](float (&v)[N], int at, int left) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = give(args.scale * (v[e] - m) - log_s, at + e, !(m < kMasked));
    G::store(dx + at, left, v);
  });
}

// A thread takes U groups of sixteen bytes of a row, a workgroup of NT threads a part of one (a wave a short row of its own, four
// to a workgroup).  STREAM: non-temporal stores.  An output that the Infinity Cache cannot hold pushes the logits out of it, and the
// next launch waits for its write-backs; a smaller one is read from there next.  8192 x 32000 bf16 behind log_probs, both, us: plain 310,
// streamed 281, streamed and from the last row on 274; the launch alone 188, 181, 180 (5.8 TB/s).
template <typename T, int NT, int U, bool STREAM>
__global__ __launch_bounds__(RowGroup<NT>::kThreads) void log_probs_backward_kernel(LogProbBackwardArgs args) {
  typedef Group16<T> G;
  constexpr int N = G::N, kRows = RowGroup<NT>::kRows;
  const int t = threadIdx.x % NT;
  // (from the last row on: what log_probs read last is what the Infinity Cache still holds)
  const int64_t row = args.rows - 1 - (static_cast<int64_t>(blockIdx.x / static_cast<uint32_t>(args.parts)) * kRows + threadIdx.x / NT);
  if (row < 0) return;
  const int part = static_cast<int>(blockIdx.x % static_cast<uint32_t>(args.parts));
  const int cols = static_cast<int>(args.cols);
  const T* x = static_cast<const T*>(args.logits) + row * args.ld;
  T* dx = static_cast<T*>(args.dlogits) + row * args.ldd;
  const int first = part * (NT * U * N);   // below cols
  Raw16 raw[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int at = first + (u * NT + t) * N;
    raw[u] = G::read(x + at, max(cols - at, 0));
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
  // (the same for all threads of a row; beyond kLargest the sum that p multiplies may be infinite, and NaN times a masked token's p)
  if (__builtin_fabsf(lse) >= args.near || __builtin_fabsf(dh) >= kLargest || __builtin_fabsf(d) >= kLargest) {
    // one of the row's workgroups, chosen so that those of many rows lie on all XCDs (always the first: on every parts-th)
    if (part == static_cast<int>((blockIdx.x / static_cast<uint32_t>(args.parts)) / 4 % static_cast<uint32_t>(args.parts)))
      backward_far<T, NT>(args, row, t, [&](float logp, int j, bool left) {
        if (!left) return id >= cols ? __builtin_nanf("") : 0.0f;
        const float p = __builtin_amdgcn_exp2f(kLog2e * logp);
        return args.scale * ((j == id ? d : 0.0f) - (p * d + dh * (p * (floored(logp) + h))));
      });
    return;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int at = first + (u * NT + t) * N;
    if (at >= cols) break;
    float v[N];
    G::unpack(raw[u], v);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float logp = __builtin_fmaf(args.scale, v[e], -lse), p = __builtin_amdgcn_exp2f(kLog2e * logp);
      v[e] = -p * (d + dh * (floored(logp) + h));
    }
    if (id >= at && id < at + N) {
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] += at + e == id ? d : 0.0f;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] *= args.scale;
    if constexpr (STREAM) G::store_streamed(dx + at, cols - at, v);
    else G::store(dx + at, cols - at, v);
  }
}

}  // namespace

// A launch has fewer than 2^32 threads.
constexpr int64_t kLaunchWorkgroups = int64_t{1} << 21;

// Parts of a row: one, but for few long rows, whose parts a second launch joins.  us, 1, 2, 4, 8, 16 parts, bf16:
//   with entropy                               1 x 65536 8.4, 7.9, 7.2, 7.8, 9.8; 1 x 131072 12.7, 10.0, 8.7, 7.7, 8.7
//                                              16 x 262144 21.8, 15.0, 10.9, 9.4, 9.7; 64 x 131072 13.3, 11.2, 9.0, 9.5, 11.6
//   with twenty tokens, which every part ranks 1 x 65536 12.8, 13.5, 12.9, 14.9, 22.5; 1 x 131072 18.8, 16.5, 14.9, 15.4, 20.8
//                                              16 x 262144 30.6, 23.5, 18.3, 17.7, 23.5; 64 x 131072 19.7, 17.3, 16.7, 18.7, 25.6
int log_probs_parts(int64_t rows, int64_t cols, int64_t n_top) {
  if (rows > 64 || cols < 65536) return 1;
  return n_top > 0 || rows > 16 ? 4 : static_cast<int>(std::min<int64_t>(cols / 16384, kMostParts));
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

namespace {

template <typename T, int NT, int U>
hipError_t launch_backward(const LogProbBackwardArgs& args, bool stream_out, hipStream_t stream) {
  constexpr int kColumns = NT * U * Group16<T>::N, kRows = RowGroup<NT>::kRows;
  const int64_t parts = (args.cols + kColumns - 1) / kColumns;
  const int64_t most = std::max<int64_t>(1, (int64_t{1} << 23) / parts) * kRows;
  // (the last rows first, over launches too)
  for (int64_t end = args.rows; end > 0; end -= most) {
    const int64_t row = std::max<int64_t>(end - most, 0);
    LogProbBackwardArgs some = args;
    some.rows = end - row;
    some.parts = static_cast<int>(parts);
    some.near = args.scale < kLeastScale ? 0.0f : kNear;
    some.logits = static_cast<const T*>(args.logits) + row * args.ld;
    some.dlogits = static_cast<T*>(args.dlogits) + row * args.ldd;
    some.lse += row;
    if (args.ids) {
      some.ids += row;
      some.dlogp += row;
    }
    if (args.entropy) {
      some.entropy += row;
      some.dentropy += row;
    }
    const dim3 g(static_cast<uint32_t>((some.rows + kRows - 1) / kRows * parts)), b(RowGroup<NT>::kThreads);
    if (stream_out) hipLaunchKernelGGL((log_probs_backward_kernel<T, NT, U, true>), g, b, 0, stream, some);
    else hipLaunchKernelGGL((log_probs_backward_kernel<T, NT, U, false>), g, b, 0, stream, some);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T>
hipError_t launch_backward_of(const LogProbBackwardArgs& args, hipStream_t stream) {
  const bool stream_out = args.rows * args.cols * static_cast<int64_t>(sizeof(T)) >= kCacheBytes;
  if (args.cols <= 64 * 4 * Group16<T>::N) return launch_backward<T, 64, 4>(args, stream_out, stream);
  return launch_backward<T, 256, 4>(args, stream_out, stream);
}

}  // namespace

hipError_t launch_log_probs_backward(const LogProbBackwardArgs& args, int dtype, hipStream_t stream) {
  return dtype == CLEAVE_BF16 ? launch_backward_of<Bf16>(args, stream) : launch_backward_of<float>(args, stream);
}

}  // namespace cleave
