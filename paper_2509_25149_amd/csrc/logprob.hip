// Log probabilities of given tokens, with entropy and the best alternatives, and the gradient of the logits.
//   d_j = z_j - max z;  s = sum exp(scale d_j);  lse = scale max z + ln s;  p_j = exp(scale d_j) / s
//   logprob = scale d_t - ln s;  entropy H = ln s - sum p_j scale d_j
//   dz_j = scale (g [j = t] + p_j (g_lse - g - g_H (ln p_j + H)))
// One pass over a row: every thread keeps a running maximum, the sum of exponentials relative to it and (for H) the sum of d exp(d), rescaled when the maximum
// moves, a batch of 32 values at a time.  All of it FP32.  Memory bounds it: 8192 x 131072 bf16 with entropies 360 us, 6.0 TB/s read, with the vector
// pipe active in 82 to 93 % of the cycles by the counters (9.8 instructions a value), so that more work a value would show; its gradient 678 us, 6.3 TB/s.  Masked values may be -infinity (probability 0) or the type's lowest value: the maximum
// is kept apart from the logarithm of the sum, so that neither a large maximum nor a row of lowest values loses what the sum says.
#include <algorithm>

#include "nvfp4_internal.h"
#include "checkpoint8.h"

namespace nvfp4 {

namespace {

constexpr float kLog2E = 1.4426950408889634f, kLn2 = 0.69314718055994531f;
constexpr float kLowest = -3.4028234663852886e38f;
constexpr float kFar = -200.0f;   // 2^kFar is 0: exponents are held above it where they are factors, since 0 * -infinity is not 0
constexpr float kInfinity = __builtin_huge_valf();
constexpr int kMostThreads = 512, kMostParts = 64, kMostTop = 32, kCandidates = 1024;

__device__ __forceinline__ int64_t index_at(const void* p, bool i64, int64_t i) {
  return i64 ? static_cast<const int64_t*>(p)[i] : static_cast<const int32_t*>(p)[i];
}

// ---------------------------------------------------------------- a thread's piece of a row
// Eight columns, or four of FP32: 16 bytes, so that a wavefront's access covers whole lines.  FP32 logits whose gradient is bf16 are taken by eight all the same, for the sake of
// the stores (8192 x 20000: 225 us by four, 192 by eight).
template <bool kBf16>
constexpr int kGroup = kBf16 ? 8 : 4;
template <bool kBf16, int kN>
struct Group : Eight<kBf16> {
  static_assert(kN == 8);
  __device__ __forceinline__ void load(const void* row, int g) { Eight<kBf16>::load(row, static_cast<int64_t>(g) * 8); }
};
template <>
struct Group<false, 4> {
  float4v w;
  __device__ __forceinline__ void load(const void* row, int g) { w = static_cast<const float4v*>(row)[g]; }
  __device__ __forceinline__ void get(float (&v)[4]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = w[i];
  }
};
typedef uint32_t uint32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t uint32x4 __attribute__((ext_vector_type(4)));

// The results of a group.  kStream: no cache should keep them.
template <bool kStream, typename T>
__device__ __forceinline__ void put(T v, T* to) {
  if (kStream) __builtin_nontemporal_store(v, to);
  else *to = v;
}
template <bool kStream, bool kBf16>
__device__ __forceinline__ void put_group(void* row, int g, const float (&v)[8]) {
  if (kBf16) {
    put<kStream>(uint32x4{f32x2_to_bf16(v[0], v[1]), f32x2_to_bf16(v[2], v[3]), f32x2_to_bf16(v[4], v[5]), f32x2_to_bf16(v[6], v[7])}, static_cast<uint32x4*>(row) + g);
  } else {
    put<kStream>(float4v{v[0], v[1], v[2], v[3]}, static_cast<float4v*>(row) + 2 * static_cast<int64_t>(g));
    put<kStream>(float4v{v[4], v[5], v[6], v[7]}, static_cast<float4v*>(row) + 2 * static_cast<int64_t>(g) + 1);
  }
}
template <bool kStream, bool kBf16>
__device__ __forceinline__ void put_group(void* row, int g, const float (&v)[4]) {
  if (kBf16) put<kStream>(uint32x2{f32x2_to_bf16(v[0], v[1]), f32x2_to_bf16(v[2], v[3])}, static_cast<uint32x2*>(row) + g);
  else put<kStream>(float4v{v[0], v[1], v[2], v[3]}, static_cast<float4v*>(row) + g);
}

// ---------------------------------------------------------------- sums of exponentials relative to a maximum
// scale (z - m), to base e and to base 2.  Two logits may be further apart than FP32's largest number while a small scale makes the distance an ordinary one: with a scale below 1 half of
// the distance is formed, and taken twice as often.  Halves lose nothing (but 2^-150 where a distance is below FP32's normal numbers), and the fused product costs what the difference does:
// one operation.  At a scale of 1 and more a distance beyond FP32 is one after scaling too.
struct Exponent {
  float h, by, c;
  __device__ __forceinline__ explicit Exponent(float scale) : h(scale < 1.0f ? 0.5f : 1.0f), by(scale < 1.0f ? 2.0f * scale : scale), c(by * kLog2E) {}
  __device__ __forceinline__ float half(float z) const { return z * h; }   // (or the whole)
  __device__ __forceinline__ float base2(float z, float half_m) const { return __builtin_fmaf(z, h, -half_m) * c; }
  __device__ __forceinline__ float base_e(float z, float half_m) const { return __builtin_fmaf(z, h, -half_m) * by; }
};

// s = sum 2^t, e = sum t 2^t, t = scale (z - m) to base 2.  Nothing but -infinity: m = kLowest, s = 0.
// A NaN or +infinity makes s NaN, and s stays so.
struct Sum {
  float m, s, e;
};

__device__ __forceinline__ float far_at_most(float t) { return __builtin_fmaxf(t, kFar); }

template <bool kEntropy>
__device__ __forceinline__ void move_to(Sum& a, float m, const Exponent& c) {
  const float t = far_at_most(c.base2(a.m, c.half(m))), f = __builtin_amdgcn_exp2f(t);
  if (kEntropy) a.e = (a.e + a.s * t) * f;
  a.s *= f;
  a.m = m;
}

template <bool kEntropy>
__device__ __forceinline__ void join(Sum& a, Sum b, const Exponent& c) {
  const float m = __builtin_fmaxf(a.m, b.m);
  move_to<kEntropy>(a, m, c);
  move_to<kEntropy>(b, m, c);
  a.s += b.s;
  if (kEntropy) a.e += b.e;
}

template <bool kEntropy, int kN>
__device__ __forceinline__ void add(Sum& a, const float (&v)[kN], const Exponent& c) {
  float m = v[0];
#pragma unroll
  for (int i = 1; i < kN; ++i) m = __builtin_fmaxf(m, v[i]);
  move_to<kEntropy>(a, __builtin_fmaxf(a.m, m), c);
  const float half_m = c.half(a.m);
  float s[4] = {}, e[4] = {};   // four chains: shorter ones lose less
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const float t = c.base2(v[i], half_m), p = __builtin_amdgcn_exp2f(t);
    s[i & 3] += p;
    if (kEntropy) e[i & 3] = __builtin_fmaf(p, far_at_most(t), e[i & 3]);
  }
  a.s += (s[0] + s[1]) + (s[2] + s[3]);
  if (kEntropy) a.e += (e[0] + e[1]) + (e[2] + e[3]);
}

template <bool kEntropy>
__device__ __forceinline__ Sum wave_join(Sum a, const Exponent& c) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    Sum b;
    b.m = __shfl_xor(a.m, off, 64);
    b.s = __shfl_xor(a.s, off, 64);
    b.e = kEntropy ? __shfl_xor(a.e, off, 64) : 0.0f;
    join<kEntropy>(a, b, c);
  }
  return a;
}

// Of a workgroup's threads, the same in all of them.
template <bool kEntropy>
__device__ __forceinline__ Sum workgroup_join(Sum a, const Exponent& c, Sum* lds) {
  a = wave_join<kEntropy>(a, c);
  const int waves = blockDim.x >> 6;
  if (waves == 1) return a;
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = a;
  __syncthreads();
  a = lds[0];
  for (int w = 1; w < waves; ++w) join<kEntropy>(a, lds[w], c);
  return a;
}

template <bool kBf16>
__device__ __forceinline__ float value_at(const void* row, int64_t col) {
  return kBf16 ? __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(row)[col]) << 16) : static_cast<const float*>(row)[col];
}

// A group at the end of a row: columns past it are not there (-infinity).
template <bool kBf16, int kN>
__device__ __forceinline__ void rest_of_row(const void* row, int g, int cols, float (&v)[kN]) {
#pragma unroll
  for (int i = 0; i < kN; ++i) v[i] = g * kN + i < cols ? value_at<kBf16>(row, g * kN + i) : -kInfinity;
}

// A group, whole or not.
template <bool kBf16, int kN>
__device__ __forceinline__ void group_of(const void* row, int g, int cols, float (&v)[kN]) {
  if (g < cols / kN) {
    Group<kBf16, kN> x;
    x.load(row, g);
    x.get(v);
  } else {
    rest_of_row<kBf16>(row, g, cols, v);
  }
}

template <bool kEntropy, bool kBf16, int kN, int kGroups>
__device__ __forceinline__ void add_groups(Sum& a, const Group<kBf16, kN> (&x)[kGroups], const Exponent& c) {
  float v[kGroups * kN];
#pragma unroll
  for (int u = 0; u < kGroups; ++u) {
    float w[kN];
    x[u].get(w);
#pragma unroll
    for (int i = 0; i < kN; ++i) v[u * kN + i] = w[i];
  }
  add<kEntropy>(a, v, c);
}

// A thread's share of groups [g0, g1), 32 columns at a time.
template <bool kBf16, bool kEntropy, int kN>
__device__ __forceinline__ Sum sum_of_groups(const void* row, int g0, int g1, int cols, const Exponent& c) {
  constexpr int kBatch = 32 / kN;
  const int step = blockDim.x, whole = min(g1, cols / kN);
  Sum a{kLowest, 0.0f, 0.0f};
  int g = g0 + static_cast<int>(threadIdx.x);
  for (; g + (kBatch - 1) * step < whole; g += kBatch * step) {
    Group<kBf16, kN> x[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) x[u].load(row, g + u * step);
    add_groups<kEntropy>(a, x, c);
  }
  for (; g < g1; g += step) {
    float v[kN];
    group_of<kBf16>(row, g, cols, v);
    add<kEntropy>(a, v, c);
  }
  return a;
}

// What the backward pass starts from.  A row without a value above -infinity has no distribution: {0, +infinity} makes every probability 0 there.
struct RowStats {
  float m, logsum;
  __device__ __forceinline__ explicit RowStats(const Sum& a) : m(a.s == 0.0f ? 0.0f : a.m), logsum(a.s == 0.0f ? kInfinity : logf(a.s)) {}
  __device__ __forceinline__ float logprob(float z, const Exponent& c) const { return c.base_e(z, c.half(m)) - logsum; }
};

__device__ __forceinline__ void write_row(const LogprobForward& a, int64_t row, const Sum& sum, const RowStats& r, const Exponent& c, float at_target, bool counted) {
  const bool empty = sum.s == 0.0f;
  if (a.stats) a.stats[2 * row] = r.m, a.stats[2 * row + 1] = r.logsum;
  if (a.lse) a.lse[row] = empty ? -kInfinity : r.m * a.scale + r.logsum;
  if (a.entropy) a.entropy[row] = empty ? 0.0f : r.logsum - kLn2 * (sum.e / sum.s);
  if (a.logprob) a.logprob[row] = counted ? r.logprob(at_target, c) : 0.0f;
}

// ---------------------------------------------------------------- best alternatives
// A value and its column as one number, the greater the better: values in order (a NaN below -infinity; -0 is 0), the lower column first among equal ones.
__device__ __forceinline__ uint32_t order_of(float z) {
  const uint32_t u = __float_as_uint(z + 0.0f);
  return z != z ? 0u : u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ uint64_t place(float z, int col) { return static_cast<uint64_t>(order_of(z)) << 32 | (0xFFFFFFFFu - static_cast<uint32_t>(col)); }
__device__ __forceinline__ float value_of(uint64_t place) {
  const uint32_t k = static_cast<uint32_t>(place >> 32);
  return k == 0u ? __uint_as_float(0x7FC00000u) : __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ int column_of(uint64_t place) { return static_cast<int>(0xFFFFFFFFu - static_cast<uint32_t>(place)); }

struct TopShared {
  float group[kMostThreads / 64][64];
  uint64_t best[kMostThreads / 64];
  uint64_t found[kCandidates];
  uint8_t lanes[kMostThreads / 64][64];
  uint32_t n_found;
};

// The best of a thread's share of groups [g0, g1) that is worse than `last`.
template <bool kBf16>
__device__ __forceinline__ uint64_t best_of_share(const void* row, int g0, int g1, int cols, uint64_t last) {
  uint64_t best = 0ull;
#pragma unroll 4
  for (int g = g0 + static_cast<int>(threadIdx.x); g < g1; g += blockDim.x) {
    constexpr int kN = kGroup<kBf16>;
    float v[kN];
    group_of<kBf16>(row, g, cols, v);
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const uint64_t p = place(v[j], g * kN + j);
      if (g * kN + j < cols && p < last && p > best) best = p;
    }
  }
  return best;
}

// The k best of groups [g0, g1) to emit(rank, place).  `own`: the largest value that this thread has seen in sum_of_groups.
// The k-th largest of 64 maxima over disjoint columns bounds the k-th best from below; only threads whose maximum reaches it hold candidates, some
// k of them, and their wavefront reads their columns once more.  Candidates take their rank by counting the better ones.
// Where fewer than k values are above -infinity the first columns at -infinity follow.
// Where too many reach the bound (rows that are equal nearly everywhere) each thread keeps the best of its share, and the best of those is taken k times over.
template <bool kBf16, typename Emit>
__device__ __forceinline__ void take_best(const void* row, int g0, int g1, int cols, float own, int k, TopShared& s, Emit emit) {
  const int t = threadIdx.x, T = blockDim.x, waves = T >> 6;
  const int wave = t >> 6, lane = t & 63;
  s.group[wave][lane] = own;
  if (t == 0) s.n_found = 0u;
  __syncthreads();
  float m = s.group[0][lane];   // (kLowest, above -infinity, for groups of nothing else)
  for (int w = 1; w < waves; ++w) m = __builtin_fmaxf(m, s.group[w][lane]);
  int better = 0;
#pragma unroll
  for (int i = 0; i < 64; ++i) better += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(m), i)) > m;
  uint32_t bound = better < k ? order_of(m) : ~0u;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) bound = min(bound, static_cast<uint32_t>(__shfl_xor(bound, off, 64)));
  const bool holds = order_of(own) >= bound;
  const uint64_t holders = __ballot(holds);
  if (holds) s.lanes[wave][__popcll(holders & ((uint64_t{1} << lane) - 1))] = static_cast<uint8_t>(lane);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int turns = (g1 - g0 + T - 1) / T, items = __popcll(holders) * turns;
  constexpr int kN = kGroup<kBf16>;
  for (int i0 = lane; i0 < items; i0 += 4 * 64) {   // four groups asked for together
    Group<kBf16, kN> x[4];
    int g[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = i0 + u * 64;
      g[u] = i < items ? g0 + wave * 64 + s.lanes[wave][i / turns] + i % turns * T : g1;
      if (g[u] < min(g1, cols / kN)) x[u].load(row, g[u]);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (g[u] >= g1) continue;
      float v[kN];
      if (g[u] < cols / kN) x[u].get(v);
      else rest_of_row<kBf16>(row, g[u], cols, v);
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        if (g[u] * kN + j < cols && order_of(v[j]) >= bound) {
          const uint32_t at = atomicAdd(&s.n_found, 1u);
          if (at < kCandidates) s.found[at] = place(v[j], g[u] * kN + j);
        }
      }
    }
  }
  __syncthreads();
  int n = static_cast<int>(s.n_found);
  if (n < k) {   // everything above -infinity is among them: the first T >= k + 32 columns have enough others, unless they are NaN
    __syncthreads();
    const int col = g0 * kN + t;
    if (col < min(g1 * kN, cols) && value_at<kBf16>(row, col) == -kInfinity) {
      const uint32_t at = atomicAdd(&s.n_found, 1u);
      s.found[at] = place(-kInfinity, col);
    }
    __syncthreads();
    n = static_cast<int>(s.n_found);
  }
  if (n >= k && n <= kCandidates) {
    for (int i = t; i < n; i += T) {
      const uint64_t mine = s.found[i];
      int better = 0;
#pragma unroll 8
      for (int j = 0; j < n; ++j) better += s.found[j] > mine;
      if (better < k) emit(better, mine);
    }
    return;
  }
  uint64_t mine = best_of_share<kBf16>(row, g0, g1, cols, ~0ull);
  for (int r = 0; r < k; ++r) {
    uint64_t best = mine;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
      const uint64_t o = __shfl_xor(static_cast<unsigned long long>(best), off, 64);
      best = o > best ? o : best;
    }
    if ((t & 63) == 0) s.best[t >> 6] = best;
    __syncthreads();
    best = s.best[0];
    for (int w = 1; w < waves; ++w) best = s.best[w] > best ? s.best[w] : best;
    if (t == 0) emit(r, best);
    if (best != 0ull && mine == best) mine = best_of_share<kBf16>(row, g0, g1, cols, best);
    __syncthreads();
  }
}

__device__ __forceinline__ void write_alternative(const LogprobForward& a, int64_t row, int rank, uint64_t p, const RowStats& r, const Exponent& c) {
  a.top_index[row * a.top + rank] = column_of(p);
  a.top_logprob[row * a.top + rank] = r.logprob(value_of(p), c);
}

// ---------------------------------------------------------------- forward
// A workgroup takes a row, or one of `parts` pieces of it, whose sums and best go to the second launch.
template <bool kBf16, bool kEntropy, bool kTop>
__global__ __launch_bounds__(kMostThreads) void logprob_forward_kernel(LogprobForward a) {
  __shared__ Sum sums[kMostThreads / 64];
  const int part = static_cast<int>(blockIdx.x % static_cast<unsigned>(a.parts));
  const int64_t row = a.row0 + blockIdx.x / static_cast<unsigned>(a.parts);
  constexpr int kN = kGroup<kBf16>;
  const int cols = static_cast<int>(a.cols), groups = (cols + kN - 1) / kN, each = (groups + a.parts - 1) / a.parts;
  const int g0 = min(part * each, groups), g1 = min(g0 + each, groups);
  const void* z = static_cast<const char*>(a.z) + row * a.ld * (kBf16 ? 2 : 4);
  const Exponent c(a.scale);
  bool counted = false;
  float at_target = 0.0f;
  if (a.parts == 1 && threadIdx.x == 0 && a.targets) {   // (asked for ahead of the row)
    const int64_t target = index_at(a.targets, a.i64, row);
    counted = target >= 0 && target < cols;
    if (counted) at_target = value_at<kBf16>(z, target);
  }
  const Sum mine = sum_of_groups<kBf16, kEntropy, kN>(z, g0, g1, cols, c);
  const Sum all = workgroup_join<kEntropy>(mine, c, sums);
  if (a.parts > 1) {
    float* to = a.partial + (row * a.parts + part) * 4;
    if (threadIdx.x == 0) *reinterpret_cast<float4v*>(to) = float4v{all.m, all.s, kEntropy ? all.e : 0.0f, 0.0f};
    if constexpr (kTop) {
      __shared__ TopShared s;
      uint64_t* best = a.best + (row * a.parts + part) * a.top;
      take_best<kBf16>(z, g0, g1, cols, mine.m, a.top, s, [&](int rank, uint64_t p) { best[rank] = p; });
    }
    return;
  }
  const RowStats r(all);
  if (threadIdx.x == 0) write_row(a, row, all, r, c, at_target, counted);
  if constexpr (kTop) {
    __shared__ TopShared s;
    take_best<kBf16>(z, g0, g1, cols, mine.m, a.top, s, [&](int rank, uint64_t p) { write_alternative(a, row, rank, p, r, c); });
  }
}

// The pieces of a row together, one workgroup to a row.
template <bool kBf16, bool kEntropy, bool kTop>
__global__ __launch_bounds__(256) void logprob_join_kernel(LogprobForward a) {
  const int64_t row = a.row0 + blockIdx.x;
  const int t = threadIdx.x, parts = a.parts, k = a.top;
  const Exponent c(a.scale);
  const void* z = static_cast<const char*>(a.z) + row * a.ld * (kBf16 ? 2 : 4);
  bool counted = false;
  float at_target = 0.0f;
  if (t == 0 && a.targets) {
    const int64_t target = index_at(a.targets, a.i64, row);
    counted = target >= 0 && target < a.cols;
    if (counted) at_target = value_at<kBf16>(z, target);
  }
  Sum mine{kLowest, 0.0f, 0.0f};
  if ((t & 63) < parts) {   // (every wavefront the same)
    const float4v v = *reinterpret_cast<const float4v*>(a.partial + (row * parts + (t & 63)) * 4);
    mine = Sum{v[0], v[1], v[2]};
  }
  if constexpr (kTop) {
    __shared__ uint64_t best[kMostParts * kMostTop], found[kMostParts * kMostTop];
    __shared__ int n_found;
    const int n = parts * k, lane = t & 63;
#pragma unroll 4
    for (int i = t; i < n; i += 256) best[i] = a.best[row * n + i];
    if (t == 0) n_found = 0;
    const Sum all = wave_join<kEntropy>(mine, c);
    const RowStats r(all);
    if (t == 0) write_row(a, row, all, r, c, at_target, counted);
    __syncthreads();
    // With j = ceil(k / parts), the ceil(k / j)-th largest of the pieces' j-th bounds the k-th best: so many pieces have j each that reach it.
    const int j = (k + parts - 1) / parts, enough = (k + j - 1) / j;
    const uint64_t jth = lane < parts ? best[lane * k + j - 1] : 0ull;
    int better = 0;
#pragma unroll 8
    for (int i = 0; i < parts; ++i) better += best[i * k + j - 1] > jth;
    const uint64_t in = __ballot(lane < parts && better < enough);
    uint64_t bound = in >> lane & 1 ? jth : ~0ull;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) bound = min(bound, static_cast<uint64_t>(__shfl_xor(static_cast<unsigned long long>(bound), off, 64)));
    for (int i = t; i < n; i += 256)
      if (best[i] >= bound && best[i] != 0ull) found[atomicAdd(&n_found, 1)] = best[i];
    __syncthreads();
    for (int i = t; i < n_found; i += 256) {
      const uint64_t p = found[i];
      int ahead = 0;
#pragma unroll 8
      for (int o = 0; o < n_found; ++o) ahead += found[o] > p;
      if (ahead < k) write_alternative(a, row, ahead, p, r, c);
    }
  } else {
    const Sum all = wave_join<kEntropy>(mine, c);
    if (t == 0) write_row(a, row, all, RowStats(all), c, at_target, counted);
  }
}

// ---------------------------------------------------------------- gradient of the logits

// What is the same for a row: dz_j = p_j (a - b log2 p_j), log2 p_j = scale (z_j - m) log2(e) - l; and what the target's column gets on top.
// scale times a gradient may be beyond FP32 where p_j makes a number of it again, and p_j = 0 has to make 0.  So where scale times the largest of the gradients is above 2^116, a, b and the target's part
// are held 2^-up of themselves, below 2^125 with all that is added up, and p_j is taken 2^up times by its exponent, which is no operation more at a column.  (The sum of the gradients that `a` holds is FP32 by
// itself.  up is 140 at most; above 127, scale times gradient above 2^242, 0 may come out as NaN.)
template <bool kEntropy>
struct RowGradient {
  float half_m, l, a, b, at_target;   // l and a for exponents raised by `up`
  int target;                         // -1: none
  int up;
  __device__ __forceinline__ RowGradient(float half_m_, float logsum, float scale, float g, float g_lse, float g_entropy, float entropy, int64_t target_, int cols) {
    const bool counted = target_ >= 0 && target_ < cols;
    if (!counted) g = 0.0f;
    float most = __builtin_fmaxf(__builtin_fabsf(g), __builtin_fabsf(g_lse));
    if (kEntropy) most = __builtin_fmaxf(most, __builtin_fabsf(g_entropy));
    up = __builtin_amdgcn_readfirstlane(max(0, exponent_of(scale) + exponent_of(most) - 115));   // (the same in a wavefront)
    scale = __builtin_ldexpf(scale, -up);
    const float raised = static_cast<float>(up);
    half_m = half_m_, l = logsum * kLog2E - raised;
    a = scale * (g_lse - g - (kEntropy && g_entropy != 0.0f ? g_entropy * entropy : 0.0f)), b = 0.0f;
    if (kEntropy) {
      b = scale * g_entropy * kLn2;
      a = up ? a + b * raised : a;
    }
    at_target = scale * g;
    target = counted && logsum != kInfinity ? static_cast<int>(target_) : -1;
  }
  // (128 for what is no number; it stays none)
  static __device__ __forceinline__ int exponent_of(float v) { return static_cast<int>(__float_as_uint(v) >> 23 & 255u) - 127; }
  // v: logits of group g, and then their gradients.
  template <int kN>
  __device__ __forceinline__ void of(float (&v)[kN], int g, const Exponent& c) const {
    const float raised = static_cast<float>(up);
    float z[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      z[i] = v[i];
      const float t = c.base2(v[i], half_m) - l, p = __builtin_amdgcn_exp2f(t);
      v[i] = p * (kEntropy ? a - b * __builtin_fmaxf(t, kFar + raised) : a);
    }
    if (g == target >> (kN == 8 ? 3 : 2)) {
      float at = z[0];
#pragma unroll
      for (int i = 1; i < kN; ++i) at = i == (target & (kN - 1)) ? z[i] : at;
      const float t = c.base2(at, half_m) - (l + raised), p = __builtin_amdgcn_exp2f(t);
      const float x = __builtin_ldexpf(p * (kEntropy ? (a - (up ? b * raised : 0.0f)) - b * far_at_most(t) : a) + at_target, up);
#pragma unroll
      for (int i = 0; i < kN; ++i) v[i] = i == (target & (kN - 1)) ? x : v[i];
    }
  }
};

template <bool kInBf16, bool kOutBf16>
constexpr int kGradientGroup = kInBf16 || kOutBf16 ? 8 : 4;

template <bool kInBf16, bool kOutBf16, bool kEntropy>
__device__ __forceinline__ void gradient_of_rest(const void* z, void* dz, int g, int cols, const RowGradient<kEntropy>& r, const Exponent& c) {
  constexpr int kN = kGradientGroup<kInBf16, kOutBf16>;
  float v[kN];
  rest_of_row<kInBf16>(z, g, cols, v);
  r.of(v, g, c);
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const int col = g * kN + i;
    if (col < cols) {
      if (kOutBf16) static_cast<uint16_t*>(dz)[col] = static_cast<uint16_t>(f32_to_bf16(v[i]));
      else static_cast<float*>(dz)[col] = v[i];
    }
  }
}

// Groups [g0, g1) of a row by the workgroup's threads, from the end to the front.
template <bool kInBf16, bool kOutBf16, bool kEntropy, bool kStream>
__device__ __forceinline__ void gradient_of_groups(const void* z, void* dz, int g0, int g1, int cols, const RowGradient<kEntropy>& r, const Exponent& c) {
  constexpr int kN = kGradientGroup<kInBf16, kOutBf16>;
  const int step = blockDim.x, whole = min(g1, cols / kN);
  if (whole < g1 && threadIdx.x == 0) gradient_of_rest<kInBf16, kOutBf16, kEntropy>(z, dz, whole, cols, r, c);
  int g = whole - 1 - static_cast<int>(threadIdx.x);
  for (; g - 3 * step >= g0; g -= 4 * step) {
    Group<kInBf16, kN> x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u].load(z, g - u * step);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      float v[kN];
      x[u].get(v);
      r.of(v, g - u * step, c);
      put_group<kStream, kOutBf16>(dz, g - u * step, v);
    }
  }
  for (; g >= g0; g -= step) {
    Group<kInBf16, kN> x;
    float v[kN];
    x.load(z, g);
    x.get(v);
    r.of(v, g, c);
    put_group<kStream, kOutBf16>(dz, g, v);
  }
}

// (Eight wavefronts to a SIMD, which FP32 to bf16 with entropy has to be told: 8192 x 20000 164 us, with seven 172.)
template <bool kInBf16, bool kOutBf16, bool kEntropy>
__global__ __launch_bounds__(256, 8) void logprob_backward_kernel(LogprobBackward a) {
  const int part = static_cast<int>(blockIdx.x % static_cast<unsigned>(a.parts));
  const int64_t row = a.row0 + blockIdx.x / static_cast<unsigned>(a.parts);
  constexpr int kN = kGradientGroup<kInBf16, kOutBf16>;
  const int cols = static_cast<int>(a.cols), groups = (cols + kN - 1) / kN, each = (groups + a.parts - 1) / a.parts;
  const int g0 = min(part * each, groups), g1 = min(g0 + each, groups);
  const Exponent c(a.scale);
  const RowGradient<kEntropy> r(c.half(a.stats[2 * row]), a.stats[2 * row + 1], a.scale, a.g_logprob ? a.g_logprob[row] : 0.0f, a.g_lse ? a.g_lse[row] : 0.0f,
                      kEntropy ? a.g_entropy[row] : 0.0f, kEntropy ? a.entropy[row] : 0.0f, a.targets ? index_at(a.targets, a.i64, row) : -1, cols);
  gradient_of_groups<kInBf16, kOutBf16, kEntropy, false>(static_cast<const char*>(a.z) + row * a.ld * (kInBf16 ? 2 : 4),
                                                         static_cast<char*>(a.dz) + row * a.ldd * (kOutBf16 ? 2 : 4), g0, g1, cols, r, c);
}

// Loss and gradient in one launch: a workgroup takes a row, sums over it and goes over it again from its end.  The last groups stay on the CU between the two --
// half in registers, half in LDS --, those in front are read again, from the L2 or the memory-side cache (8192 x 131072 bf16: by the counters 1.5 times the logits' bytes are
// fetched; 795 us, 5.4 TB/s of the bytes that have to move; two launches take 1050, without what stays on the CU 925, with one workgroup to a CU that keeps all of a row 875).
// Tried too: a workgroup that takes one row after the other and fetches the next one into the places that the gradient leaves, each byte once: 820.
constexpr int kKeepBytes = 64;   // of a thread, in either

template <int T, bool kInBf16, bool kOutBf16, bool kStream>
__global__ __launch_bounds__(T, 8) void logprob_loss_kernel(LogprobForward f, LogprobBackward b) {
  constexpr int kN = kGradientGroup<kInBf16, kOutBf16>, kKeep = kKeepBytes / static_cast<int>(sizeof(Group<kInBf16, kN>));
  __shared__ Sum sums[T / 64];
  __shared__ Group<kInBf16, kN> kept[kKeep * T];
  const int64_t row = f.row0 + blockIdx.x;
  const int t = threadIdx.x, cols = static_cast<int>(f.cols), whole = cols / kN;
  const void* z = static_cast<const char*>(f.z) + row * f.ld * (kInBf16 ? 2 : 4);
  void* dz = static_cast<char*>(b.dz) + row * b.ldd * (kOutBf16 ? 2 : 4);
  const Exponent c(f.scale);
  const int64_t target = index_at(f.targets, f.i64, row);
  const bool counted = target >= 0 && target < cols;
  const float at_target = counted ? value_at<kInBf16>(z, target) : 0.0f, g = b.g_logprob[row];

  const int again = max(0, whole - 2 * kKeep * T), first = again + t;   // groups [0, again) are read twice
  Sum mine = sum_of_groups<kInBf16, false, kN>(z, 0, again, again * kN, c);
#pragma unroll
  for (int u = 0; u < kKeep; ++u) {
    Group<kInBf16, kN> x[1];
    if (first + u * T < whole) {
      x[0].load(z, first + u * T);
      kept[u * T + t] = x[0];
      add_groups<false>(mine, x, c);
    }
  }
  Group<kInBf16, kN> x[kKeep][1];
#pragma unroll
  for (int u = 0; u < kKeep; ++u)
    if (first + (kKeep + u) * T < whole) x[u][0].load(z, first + (kKeep + u) * T);
#pragma unroll
  for (int u = 0; u < kKeep; ++u)
    if (first + (kKeep + u) * T < whole) add_groups<false>(mine, x[u], c);
  if (cols % kN && t == T - 1) {
    float v[kN];
    rest_of_row<kInBf16>(z, whole, cols, v);
    add<false>(mine, v, c);
  }
  const Sum all = workgroup_join<false>(mine, c, sums);
  const RowStats r(all);
  if (t == 0) write_row(f, row, all, r, c, at_target, counted);
  const RowGradient<false> d(c.half(r.m), r.logsum, f.scale, g, 0.0f, 0.0f, 0.0f, target, cols);
  auto store = [&](const Group<kInBf16, kN>& x, int group) {
    float v[kN];
    x.get(v);
    d.of(v, group, c);
    put_group<kStream, kOutBf16>(dz, group, v);
  };
  if (cols % kN && t == T - 1) gradient_of_rest<kInBf16, kOutBf16, false>(z, dz, whole, cols, d, c);
#pragma unroll
  for (int u = kKeep - 1; u >= 0; --u)
    if (first + (kKeep + u) * T < whole) store(x[u][0], first + (kKeep + u) * T);
#pragma unroll
  for (int u = kKeep - 1; u >= 0; --u)
    if (first + u * T < whole) store(kept[u * T + t], first + u * T);
  gradient_of_groups<kInBf16, kOutBf16, false, kStream>(z, dz, 0, again, again * kN, d, c);
}

// ---------------------------------------------------------------- launches

// A launch holds 2^32 threads: rows of one, with `each` threads to a row.
int64_t rows_at_once(int64_t each) { return std::max<int64_t>(1, 0xfffffff0 / each); }

constexpr int64_t kCUs = 256;

struct ForwardShape {
  int parts, threads;
};
// A row to a workgroup, but for few long rows, which are cut into pieces (us on the GPU, whole / in pieces, bf16 with entropy, 1, 16, 64 and 90 rows: of 50257 6.3 / 5.6, 6.7 / 6.9, 6.8 / 8.1, 6.8 / 8.6;
// of 65536 7.3 / 5.6, 7.6 / 6.9, 8.1 / 8.1, 8.3 / 9.2; of 131072 11.2 / 5.6, 11.5 / 7.4, 12.1 / 9.2, 12.8 / 11.9.  With 20 alternatives, which are searched in every piece and then joined: of 65536
// 11.2 / 12.7, 11.8 / 15.1, 11.9 / 15.4, 12.5 / 16.2; of 100000 14.1 / 12.5, 15.2 / 15.6, 15.2 / 17.0, 16.1 / 17.3; of 131072 16.3 / 12.6, 17.3 / 15.6, 18.3 / 17.0, 19.4 / 19.3.  The second launch costs the
// host 3 more).  Threads by the bytes of a row; 64 where alternatives are looked for in up to 2 KB, which is as many as take_best needs for 32.
ForwardShape forward_shape(int64_t rows, int64_t cols, bool bf16, bool top) {
  if (rows < 96 && cols >= 65536) return {static_cast<int>(std::min<int64_t>(kMostParts, 4 * kCUs / std::max<int64_t>(rows, 1))), 256};
  const int64_t bytes = cols * (bf16 ? 2 : 4);
  return {1, bytes <= (top ? 2 << 10 : 16 << 10) ? 64 : bytes <= 64 << 10 || (rows >= kCUs && rows < 8 * kCUs) ? 256 : 512};
}

template <bool... kFlags>
hipError_t forward_with(const LogprobForward& a, int threads, hipStream_t s) {
  if constexpr (sizeof...(kFlags) == 3) {
    const int64_t most = rows_at_once(static_cast<int64_t>(a.parts) * std::max(threads, 256));
    LogprobForward p = a;
    for (p.row0 = 0; p.row0 < a.rows; p.row0 += most) {
      const unsigned rows = static_cast<unsigned>(std::min(most, a.rows - p.row0));
      hipLaunchKernelGGL((logprob_forward_kernel<kFlags...>), dim3(rows * static_cast<unsigned>(a.parts)), dim3(threads), 0, s, p);
      hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      if (a.parts == 1) continue;
      hipLaunchKernelGGL((logprob_join_kernel<kFlags...>), dim3(rows), dim3(256), 0, s, p);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  } else {
    const bool flags[] = {a.bf16, a.entropy != nullptr, a.top > 0};
    return flags[sizeof...(kFlags)] ? forward_with<kFlags..., true>(a, threads, s) : forward_with<kFlags..., false>(a, threads, s);
  }
}

template <bool... kFlags>
hipError_t backward_with(const LogprobBackward& a, int threads, hipStream_t s) {
  if constexpr (sizeof...(kFlags) == 3) {
    const int64_t most = rows_at_once(static_cast<int64_t>(a.parts) * threads);
    LogprobBackward p = a;
    for (p.row0 = 0; p.row0 < a.rows; p.row0 += most) {
      const unsigned rows = static_cast<unsigned>(std::min(most, a.rows - p.row0));
      hipLaunchKernelGGL((logprob_backward_kernel<kFlags...>), dim3(rows * static_cast<unsigned>(a.parts)), dim3(threads), 0, s, p);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  } else {
    const bool flags[] = {a.bf16, a.out_bf16, a.g_entropy != nullptr};
    return flags[sizeof...(kFlags)] ? backward_with<kFlags..., true>(a, threads, s) : backward_with<kFlags..., false>(a, threads, s);
  }
}

// By bytes of a row, in whose second pass the part that stays on the CU counts, against rows in flight.  us for 8192 rows with 64 / 256 / 512 / 1024 threads: 8 KB 27 / 31 / 46 / 97,
// 20 KB 91 / 69 / 75 / 124, 40 KB 185 / 135 / 126 / 169, 80 KB 368 / 295 / 252 / 245, 262 KB 1214 / 1123 / 1054 / 873; 1040 rows of 100 KB 72 / 57 / 55 / 61 (1040 of
// them do not fit the chip's 512 places for 1024 threads), of 200 KB 147 / 139 / 120 / 108.  (Of 131072 FP32 values, 524 KB, three quarters are read twice: by the counters 1.75 times their bytes.)
int loss_threads(int64_t rows, int64_t cols, bool bf16) {
  const int64_t bytes = cols * (bf16 ? 2 : 4);
  return bytes <= 8 << 10 ? 64 : bytes <= 36 << 10 ? 256 : bytes <= (rows >= 8 * kCUs ? 72 << 10 : 160 << 10) ? 512 : 1024;
}

template <int T, bool kStream>
hipError_t loss_of(const LogprobForward& f, const LogprobBackward& b, hipStream_t s) {
  const int64_t most = rows_at_once(T);
  LogprobForward p = f;
  for (p.row0 = 0; p.row0 < f.rows; p.row0 += most) {
    const unsigned rows = static_cast<unsigned>(std::min(most, f.rows - p.row0));
#define NVFP4_LOSS(I, O) hipLaunchKernelGGL((logprob_loss_kernel<T, I, O, kStream>), dim3(rows), dim3(T), 0, s, p, b)
    if (f.bf16) {
      if (b.out_bf16) NVFP4_LOSS(true, true); else NVFP4_LOSS(true, false);
    } else {
      if (b.out_bf16) NVFP4_LOSS(false, true); else NVFP4_LOSS(false, false);
    }
#undef NVFP4_LOSS
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

size_t logprob_workspace_bytes(int64_t rows, int64_t cols, int top) {
  const int parts = forward_shape(rows, cols, true, false).parts;
  // The pieces' sums, their best, and room for the statistics between the two passes of nvfp4_logprob_with_gradient.
  return parts == 1 ? 0 : static_cast<size_t>(rows) * (static_cast<size_t>(parts) * (16 + 8 * static_cast<size_t>(top)) + 8);
}

hipError_t launch_logprob_forward(const LogprobForward& all, void* workspace, hipStream_t s) {
  LogprobForward a = all;
  const ForwardShape shape = forward_shape(a.rows, a.cols, a.bf16, a.top > 0);
  a.parts = shape.parts;
  a.partial = static_cast<float*>(workspace);
  a.best = reinterpret_cast<uint64_t*>(a.partial + (a.parts > 1 ? a.rows * a.parts * 4 : 0));
  return forward_with<>(a, shape.threads, s);
}

// A workgroup takes 8 KB of the wider of logits and gradient, or a row that has fewer.  (us with 4 / 8 / 16 KB: 8192 x 131072 bf16 758 / 674 / 748, 1040 x 50257 FP32 86 / 76 / 84.)
hipError_t launch_logprob_backward(const LogprobBackward& all, hipStream_t s) {
  LogprobBackward a = all;
  const int64_t each = a.bf16 && a.out_bf16 ? 4096 : 2048;
  a.parts = static_cast<int>((a.cols + each - 1) / each);
  return backward_with<>(a, a.cols >= each / 2 ? 256 : 64, s);
}

hipError_t launch_logprob_with_gradient(const LogprobForward& f, const LogprobBackward& b, void* workspace, hipStream_t s) {
  if (forward_shape(f.rows, f.cols, f.bf16, false).parts == 1) {
    // The gradient passes the caches by where that pays: they are left to the rows that are read again (8192 x 131072 bf16 877 -> 797, 4096 x 131072 FP32 1075 -> 966), but stores of half lines
    // (FP32 from eight columns of bf16) lose by it (686 -> 980).
    const int threads = loss_threads(f.rows, f.cols, f.bf16);
    return threads == 64    ? loss_of<64, false>(f, b, s)
           : threads == 256 ? loss_of<256, false>(f, b, s)
           : threads == 512 ? (b.out_bf16 == f.bf16 ? loss_of<512, true>(f, b, s) : loss_of<512, false>(f, b, s))
                            : (b.out_bf16 == f.bf16 ? loss_of<1024, true>(f, b, s) : loss_of<1024, false>(f, b, s));
  }
  LogprobForward forward = f;
  LogprobBackward backward = b;
  if (!f.stats) backward.stats = forward.stats = static_cast<float*>(workspace) + f.rows * forward_shape(f.rows, f.cols, f.bf16, false).parts * 4;
  const hipError_t e = launch_logprob_forward(forward, workspace, s);
  return e == hipSuccess ? launch_logprob_backward(backward, s) : e;
}

}  // namespace nvfp4
