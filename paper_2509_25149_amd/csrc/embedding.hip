// Embedding: rows of a table by token, scaled, and the table's gradient.
//   forward   out[t] = scale table[id[t]], zeros for an id outside the table
//   backward  dtable[v] (+)= scale * sum of dout[t] over the tokens t with id[t] = v
// The gradient sorts the tokens by id (and by position among equal ids), so that every row's sum is taken in a fixed order without atomics and every row is
// written once.  Sums FP32.  Memory bounds both: 8192 x 5120 bf16 out of 131072 rows 24 us on the GPU; its gradient 444 us, of which the zeros of 2.7 GB are 380.
#include <algorithm>

#include "nvfp4_internal.h"
#include "checkpoint8.h"

namespace nvfp4 {

namespace {

__device__ __forceinline__ int64_t id_at(const void* ids, bool i64, int64_t t) {
  return i64 ? static_cast<const int64_t*>(ids)[t] : static_cast<const int32_t*>(ids)[t];
}

// ---------------------------------------------------------------- forward
// A workgroup takes 1024 consecutive groups of eight columns, of as many tokens as that is; a thread four of them.
constexpr int kGroupsEach = 4;

template <bool kTableBf16, bool kOutBf16>
__global__ __launch_bounds__(256) void embedding_forward_kernel(EmbeddingForward a) {
  const uint32_t groups = static_cast<uint32_t>(a.cols >> 3);
  const uint64_t first = static_cast<uint64_t>(blockIdx.x) * (256 * kGroupsEach);
  const int64_t token0 = a.token0 + static_cast<int64_t>(first / groups);
  const uint32_t group0 = static_cast<uint32_t>(first % groups);
  Eight<kTableBf16> x[kGroupsEach];
  int64_t token[kGroupsEach], id[kGroupsEach];
  int col[kGroupsEach];
#pragma unroll
  for (int u = 0; u < kGroupsEach; ++u) {
    const uint32_t g = group0 + threadIdx.x + 256u * u;
    token[u] = token0 + g / groups;
    col[u] = static_cast<int>(g % groups) * 8;
    id[u] = token[u] < a.tokens ? id_at(a.ids, a.i64, token[u]) : -1;
  }
#pragma unroll
  for (int u = 0; u < kGroupsEach; ++u) {
    if (id[u] < 0 || id[u] >= a.vocab) id[u] = -1;
    else x[u].load(static_cast<const char*>(a.table) + id[u] * a.ldt * (kTableBf16 ? 2 : 4), col[u]);
  }
#pragma unroll
  for (int u = 0; u < kGroupsEach; ++u) {
    if (token[u] >= a.tokens) continue;
    float v[8] = {};
    if (id[u] >= 0) {
      x[u].get(v);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= a.scale;
    }
    store8(static_cast<char*>(a.out) + token[u] * a.ldo * (kOutBf16 ? 2 : 4), col[u], kOutBf16, v);
  }
}

// ---------------------------------------------------------------- tokens in order of their ids
// A key is the id, or the number of rows for an id outside the table: those come last and belong to no row.
// kN of them, `step` tokens apart, asked for together; those behind the last token are not tokens (kNoKey).
constexpr uint32_t kNoKey = 0xFFFFFFFFu;
template <int kN, typename Id>
__device__ __forceinline__ void keys_of(const Id* ids, int t, int step, int n, int64_t vocab, uint32_t (&key)[kN]) {
  Id id[kN];
#pragma unroll
  for (int u = 0; u < kN; ++u) id[u] = ids[min(t + u * step, n - 1)];
#pragma unroll
  for (int u = 0; u < kN; ++u) key[u] = t + u * step >= n ? kNoKey : id[u] >= 0 && id[u] < vocab ? static_cast<uint32_t>(id[u]) : static_cast<uint32_t>(vocab);
}
template <int kN>
__device__ __forceinline__ void keys_of(const void* ids, bool i64, int t, int step, int n, int64_t vocab, uint32_t (&key)[kN]) {
  if (i64) keys_of(static_cast<const int64_t*>(ids), t, step, n, vocab, key);
  else keys_of(static_cast<const int32_t*>(ids), t, step, n, vocab, key);
}

// Up to kFewTokens: a token's place is the number of tokens before it, counted: two operations a pair.  A workgroup holds the keys and takes 32 tokens; a wavefront four of them, each
// lane against every 64th piece of four keys.  (us for the whole gradient of 8200 / 16384 tokens, 700 rows of 256, so 27 / 38 and by passes 33 / 33.)
constexpr int kFewTokens = 12288, kTile = 2048, kRankTokens = 32, kRankEach = 4;

constexpr int kRankThreads = kRankTokens / kRankEach * 64;

// Zeros into [vocab, cols] of FP32, 16 bytes a thread: waves that store once, neighbours on one XCD, write 2.7 GB at 6.9 TB/s (five or more stores to a thread at 5.6).
struct ZeroArgs {
  float* to;
  int64_t ld, pieces;   // of four columns, in all rows
  uint32_t across, groups;   // pieces of a row; workgroups
};
__device__ __forceinline__ void write_zeros(const ZeroArgs& z, uint32_t group) {
  for (int64_t i = static_cast<int64_t>(xcd_neighbours(group, z.groups)) * kRankThreads + threadIdx.x; i < z.pieces; i += static_cast<int64_t>(z.groups) * kRankThreads) {
    int64_t row;
    uint32_t part;
    if (i >> 32) row = i / z.across, part = static_cast<uint32_t>(i % z.across);
    else row = static_cast<uint32_t>(i) / z.across, part = static_cast<uint32_t>(i) % z.across;
    *reinterpret_cast<float4v*>(z.to + row * z.ld + static_cast<int64_t>(part) * 4) = float4v{0.0f, 0.0f, 0.0f, 0.0f};
  }
}

__global__ __launch_bounds__(kRankThreads) void zero_kernel(ZeroArgs z) { write_zeros(z, blockIdx.x); }

// Workgroups behind those of the tokens write zeros.
__global__ __launch_bounds__(kRankThreads) void rank_kernel(const void* ids, bool i64, int n, int64_t vocab, uint32_t* __restrict__ keys, uint32_t* __restrict__ order, ZeroArgs z) {
  const uint32_t ranking = static_cast<uint32_t>(n + kRankTokens - 1) / kRankTokens;
  if (blockIdx.x >= ranking) {
    write_zeros(z, blockIdx.x - ranking);
    return;
  }
  constexpr int T = kRankThreads;
  __shared__ __attribute__((aligned(16))) uint32_t all[kFewTokens];
  const int fours = (n + 3) >> 2;
  for (int base = 0; base < n; base += T * 8) {
    uint32_t k[8];
    keys_of(ids, i64, base + static_cast<int>(threadIdx.x), T, n, vocab, k);
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (base + u * T < fours * 4) all[base + u * T + threadIdx.x] = k[u];
  }
  __syncthreads();
  const int lane = threadIdx.x & 63, t0 = static_cast<int>(blockIdx.x) * kRankTokens + static_cast<int>(threadIdx.x >> 6) * kRankEach;
  const uint4* four = reinterpret_cast<const uint4*>(all);
  uint32_t key[kRankEach], before[kRankEach] = {};
#pragma unroll
  for (int e = 0; e < kRankEach; ++e) key[e] = t0 + e < n ? all[t0 + e] : 0u;
  // Among equal keys those in front come first: keys up to this token's in front of the wavefront's tokens (one piece, kRankEach being 4), less than it behind them.
  const int mid = t0 >> 2;
#pragma unroll 4
  for (int i = lane; i < mid; i += 64) {
    const uint4 k = four[i];
#pragma unroll
    for (int e = 0; e < kRankEach; ++e) before[e] += (k.x <= key[e]) + (k.y <= key[e]) + (k.z <= key[e]) + (k.w <= key[e]);
  }
#pragma unroll 4
  for (int i = mid + 1 + lane; i < fours; i += 64) {
    const uint4 k = four[i];
#pragma unroll
    for (int e = 0; e < kRankEach; ++e) before[e] += (k.x < key[e]) + (k.y < key[e]) + (k.z < key[e]) + (k.w < key[e]);
  }
#pragma unroll
  for (int e = 0; e < kRankEach; ++e) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) before[e] += __shfl_xor(before[e], off, 64);
#pragma unroll
    for (int o = 0; o < kRankEach; ++o) before[e] += o < e ? key[o] <= key[e] : o > e && t0 + o < n && key[o] < key[e];
    if (lane == 0 && t0 + e < n) keys[before[e]] = key[e], order[before[e]] = static_cast<uint32_t>(t0 + e);
  }
}

// More: passes over digits of up to nine bits, each stable: count the digits of a tile, sum up, put in place.  A tile of 2048 belongs to a workgroup, whose
// wavefronts have 512 consecutive keys each.  Counts of up to kFoldTiles tiles are summed up by every workgroup for itself, which saves a launch.
constexpr int kMostDigits = 512, kFoldTiles = 32;
struct SortPass {
  const void* ids;                      // first pass: keys are made from these
  const uint32_t *keys, *order;         // later ones
  uint32_t *counts, *to_keys, *to_order;
  int64_t vocab;
  int n, tiles, shift, digits;
  bool i64, first;
};

// Eight keys of a thread, `step` apart; kNoKey behind the last.
__device__ __forceinline__ void sort_keys(const SortPass& p, int i, int step, uint32_t (&key)[8]) {
  if (p.first) {
    keys_of(p.ids, p.i64, i, step, p.n, p.vocab, key);
  } else {
#pragma unroll
    for (int u = 0; u < 8; ++u) key[u] = p.keys[min(i + u * step, p.n - 1)];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (i + u * step >= p.n) key[u] = kNoKey;
  }
}

__global__ __launch_bounds__(256) void sort_count_kernel(SortPass p) {
  __shared__ uint32_t count[kMostDigits];
  for (int d = threadIdx.x; d < p.digits; d += 256) count[d] = 0u;
  __syncthreads();
  uint32_t key[8];
  sort_keys(p, static_cast<int>(blockIdx.x) * kTile + static_cast<int>(threadIdx.x), 256, key);
#pragma unroll
  for (int u = 0; u < 8; ++u)
    if (key[u] != kNoKey) atomicAdd(&count[(key[u] >> p.shift) & (p.digits - 1)], 1u);
  __syncthreads();
  for (int d = threadIdx.x; d < p.digits; d += 256) p.counts[static_cast<int64_t>(d) * p.tiles + blockIdx.x] = count[d];
}

// counts[i] <- sum of those before; one workgroup.
__global__ __launch_bounds__(1024) void sort_scan_kernel(uint32_t* counts, int n) {
  __shared__ uint32_t wave_total[16];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  uint32_t carry = 0u;
  for (int base = 0; base < n; base += 4096) {
    uint32_t v[4], sum = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = base + t * 4 + i;
      v[i] = at < n ? counts[at] : 0u;
      sum += v[i];
    }
    uint32_t up = sum;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const uint32_t o = __shfl_up(up, off, 64);
      if (lane >= off) up += o;
    }
    if (lane == 63) wave_total[wave] = up;
    __syncthreads();
    uint32_t before = carry + up - sum, total = 0u;
    for (int w = 0; w < 16; ++w) {
      if (w < wave) before += wave_total[w];
      total += wave_total[w];
    }
    carry += total;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = base + t * 4 + i;
      if (at < n) counts[at] = before;
      before += v[i];
    }
    __syncthreads();
  }
}

__global__ __launch_bounds__(256) void sort_place_kernel(SortPass p) {
  __shared__ uint32_t next[4][kMostDigits];   // where a wavefront's next key of a digit goes
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int d = threadIdx.x; d < 4 * kMostDigits; d += 256) next[0][d] = 0u;
  __syncthreads();
  const int base = static_cast<int>(blockIdx.x) * kTile + wave * 512;
  uint32_t key[8], order[8];
  sort_keys(p, base + lane, 64, key);
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const int i = base + r * 64 + lane;
    order[r] = p.first ? static_cast<uint32_t>(i) : p.order[min(i, p.n - 1)];
    if (key[r] != kNoKey) atomicAdd(&next[wave][(key[r] >> p.shift) & (p.digits - 1)], 1u);
  }
  __syncthreads();
  // Where this tile's first key of a digit goes: two digits to a thread.
  uint32_t at[2] = {};
  if (p.tiles > kFoldTiles) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int d = static_cast<int>(threadIdx.x) * 2 + e;
      if (d < p.digits) at[e] = p.counts[static_cast<int64_t>(d) * p.tiles + blockIdx.x];
    }
  } else {
    __shared__ uint32_t wave_total[4];
    uint32_t total[2] = {};
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int d = static_cast<int>(threadIdx.x) * 2 + e;
      if (d >= p.digits) continue;
#pragma unroll 8
      for (int i = 0; i < p.tiles; ++i) {
        const uint32_t n = p.counts[d * p.tiles + i];
        total[e] += n;
        at[e] += i < static_cast<int>(blockIdx.x) ? n : 0u;
      }
    }
    uint32_t up = total[0] + total[1];
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const uint32_t o = __shfl_up(up, off, 64);
      if (lane >= off) up += o;
    }
    if (lane == 63) wave_total[wave] = up;
    __syncthreads();
    uint32_t before = up - total[0] - total[1];
    for (int w = 0; w < wave; ++w) before += wave_total[w];
    at[0] += before;
    at[1] += before + total[0];
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int d = static_cast<int>(threadIdx.x) * 2 + e;
    if (d >= p.digits) continue;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t n = next[w][d];
      next[w][d] = at[e];
      at[e] += n;
    }
  }
  __syncthreads();
  volatile uint32_t* mine = next[wave];   // (a wavefront's own: its LDS operations are done in order)
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const bool in = key[r] != kNoKey;
    const uint32_t digit = (key[r] >> p.shift) & (p.digits - 1);
    uint64_t same = __ballot(in);
#pragma unroll
    for (int b = 0; b < 9; ++b) {
      const bool bit = (digit >> b) & 1u;
      const uint64_t with = __ballot(bit);
      same &= bit ? with : ~with;
    }
    const uint64_t below = same & ((uint64_t{1} << lane) - 1);
    uint32_t to = 0u;
    if (in) to = mine[digit] + static_cast<uint32_t>(__popcll(below));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (in && below == 0) mine[digit] = to + static_cast<uint32_t>(__popcll(same));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (in) {
      p.to_keys[to] = key[r];
      p.to_order[to] = order[r];
    }
  }
}

// ---------------------------------------------------------------- sums
struct SumArgs {
  EmbeddingBackward a;
  const uint32_t *keys, *order;   // n of them, in order
  float* partials;                // [chunks, 2, cols]: sum of a chunk's first row if that has begun before, of its last if that goes on behind
  int n, chunk, chunks, strips;   // strips of 512 columns
  uint32_t zero_groups;           // workgroups that write rows without a token
};

__device__ __forceinline__ int lower_bound(const uint32_t* keys, int n, uint32_t key) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (keys[mid] < key) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

constexpr int kZeroRows = 32, kAhead = 8;

// The first workgroups: a wavefront adds a chunk of consecutive tokens over 512 columns, eight to a lane, and stores each row as it ends.  The rest, if
// any, look for rows without a token, 32 each, and write zeros there.
template <bool kBf16>
__global__ __launch_bounds__(256) void embedding_sum_kernel(SumArgs s) {
  const EmbeddingBackward& a = s.a;
  const int lane = threadIdx.x & 63;
  const int64_t sums = (static_cast<int64_t>(s.chunks) * s.strips + 3) / 4;
  if (blockIdx.x >= sums) {
    for (int64_t row0 = (blockIdx.x - sums) * kZeroRows; row0 < a.vocab; row0 += static_cast<int64_t>(s.zero_groups) * kZeroRows) {
      bool absent = false;
      if (lane < kZeroRows && row0 + lane < a.vocab) {
        const int at = lower_bound(s.keys, s.n, static_cast<uint32_t>(row0 + lane));
        absent = at == s.n || s.keys[at] != static_cast<uint32_t>(row0 + lane);
      }
      for (uint64_t left = __ballot(absent); left; left &= left - 1) {
        float* to = a.dtable + (row0 + __builtin_ctzll(left)) * a.ldt;
        for (int64_t col = threadIdx.x * 4; col < a.cols; col += 1024) *reinterpret_cast<float4v*>(to + col) = float4v{0.0f, 0.0f, 0.0f, 0.0f};
      }
    }
    return;
  }
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (unit >= static_cast<int64_t>(s.chunks) * s.strips) return;
  const int chunk = static_cast<int>(unit / s.strips), first = chunk * s.chunk, last = min(first + s.chunk, s.n);
  const int64_t col = static_cast<int64_t>(unit % s.strips) * 512 + lane * 8, from = min(col, a.cols - 8);
  const bool in = col < a.cols;
  const uint32_t vocab = static_cast<uint32_t>(a.vocab);
  const uint32_t ahead = first > 0 ? s.keys[first - 1] : kNoKey, behind = last < s.n ? s.keys[last] : kNoKey;
  uint32_t key = s.keys[first];
  bool begun = ahead == key;
  float sum[8] = {};
  auto finish = [&](bool goes_on) {
    if (key >= vocab || !in) return;
    if (begun || goes_on) {
      store8(s.partials + (static_cast<int64_t>(chunk) * 2 + (begun ? 0 : 1)) * a.cols, col, false, sum);
      return;
    }
    float* row = a.dtable + static_cast<int64_t>(key) * a.ldt;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = a.scale * sum[i];
    if (a.accumulate) {
      Eight<false> old;
      float o[8];
      old.load(row, col);
      old.get(o);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += o[i];
    }
    store8(row, col, false, v);
  };
  for (int base = first; base < last; base += 64) {   // a lane holds one of the next 64 tokens
    const int mine = min(base + lane, last - 1), n = min(64, last - base);
    const uint32_t keys = s.keys[mine], order = s.order[mine];
    for (int at = 0; at < n; at += kAhead) {
      Eight<kBf16> x[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)   // (behind the last token the last once more)
        x[u].load(static_cast<const char*>(a.dout) + static_cast<int64_t>(__builtin_amdgcn_readlane(order, (at + u) & 63)) * a.ldd * (kBf16 ? 2 : 4), from);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (at + u >= n) break;
        const uint32_t k = __builtin_amdgcn_readlane(keys, at + u);
        if (k != key) {
          finish(false);
          key = k;
          begun = false;
#pragma unroll
          for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
        }
        float v[8];
        x[u].get(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += v[i];
      }
    }
  }
  finish(behind == key);
}

// What four wavefronts have of 512 (or 256) columns, in order; the first one gets the sum.
template <int kN>
__device__ __forceinline__ void add_wavefronts(float (&sum)[kN], float (*lds)[64][kN]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (wave > 0) {
#pragma unroll
    for (int i = 0; i < kN; ++i) lds[wave - 1][lane][i] = sum[i];
  }
  __syncthreads();
  if (wave > 0) return;
  for (int w = 0; w < 3; ++w) {
#pragma unroll
    for (int i = 0; i < kN; ++i) sum[i] += lds[w][lane][i];
  }
}

// Rows whose tokens reach over chunks: the workgroup of the chunk in which one begins adds up, in order, what the chunks have left of it, over 256 columns and a quarter of the chunks to
// each wavefront.
__global__ __launch_bounds__(256) void embedding_join_kernel(SumArgs s) {
  __shared__ float others[3][64][4];
  const EmbeddingBackward& a = s.a;
  const int chunk = static_cast<int>(blockIdx.x), first = chunk * s.chunk, last = first + s.chunk;
  if (last >= s.n) return;
  const uint32_t key = s.keys[last - 1];
  if (key >= static_cast<uint32_t>(a.vocab) || s.keys[last] != key || (first > 0 && s.keys[first - 1] == key)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int final_chunk = chunk;   // the last one that begins with the key: 64 looked at together
  for (uint64_t more = ~0ull; more == ~0ull; final_chunk += more == ~0ull ? 64 : __builtin_ctzll(~more)) {
    const int64_t at = static_cast<int64_t>(final_chunk + 1 + lane) * s.chunk;
    more = __ballot(at < s.n && s.keys[at] == key);
  }
  const int64_t col = static_cast<int64_t>(blockIdx.y) * 256 + lane * 4;
  const int parts = final_chunk - chunk + 1, each = (parts + 3) >> 2, p0 = wave * each, p1 = min(p0 + each, parts);
  // (The chunk in which the row begins has left its part in the second place, the others in the first.)
  const float* from = s.partials + static_cast<int64_t>(chunk) * 2 * a.cols + min(col, a.cols - 4);
  float4v part = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 16
  for (int p = p0; p < p1; ++p) part += *reinterpret_cast<const float4v*>(from + (static_cast<int64_t>(p) * 2 + (p == 0 ? 1 : 0)) * a.cols);
  float sum[4] = {part[0], part[1], part[2], part[3]};
  add_wavefronts(sum, others);
  if (wave > 0 || col >= a.cols) return;
  float4v* to = reinterpret_cast<float4v*>(a.dtable + static_cast<int64_t>(key) * a.ldt + col);
  const float4v v = a.scale * float4v{sum[0], sum[1], sum[2], sum[3]};
  *to = a.accumulate ? *to + v : v;
}

// ---------------------------------------------------------------- few tokens
// Up to kCountedTokens there is no sorting and, but for a large table's zeros, one launch: a workgroup takes a token and 512 columns, compares all ids with the token's, and goes on if it is
// the first one of its id: the others' places are bits in order, and each wavefront adds a quarter of their rows.  Tokens that are all the same are added by a few
// workgroups, which is why this ends at 512 of them.  (Ids by Zipf's law, us so / sorted, called from Python: 16 tokens, 700 rows of 256 8.3 / 15.6, 3000 of 5120
// 13.7 / 17.2; 128 tokens 8.3 / 16.0 and 15.2 / 18; 512 tokens 8.7 / 15.0 and 19 / 20; 512 times the same of 3000 rows of 5120 25 / 21.)
// The rest of the workgroups, if any, look for rows without a token, 64 each, and write zeros there.
constexpr int kCountedTokens = 512, kCountedZeroRows = 64;

template <bool kBf16, int kN>
__device__ __forceinline__ void add_listed(const EmbeddingBackward& a, const uint16_t* list, int n, int64_t col, float (&sum)[8]) {
  for (int i = 0; i < n; i += kN) {
    Eight<kBf16> x[kN];
#pragma unroll
    for (int u = 0; u < kN; ++u)   // (behind the last one the last once more)
      x[u].load(static_cast<const char*>(a.dout) + static_cast<int64_t>(list[min(i + u, n - 1)]) * a.ldd * (kBf16 ? 2 : 4), col);
#pragma unroll
    for (int u = 0; u < kN; ++u) {
      float v[8];
      x[u].get(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] = i + u < n ? sum[j] + v[j] : sum[j];
    }
  }
}

template <bool kBf16>
__global__ __launch_bounds__(256) void embedding_few_kernel(EmbeddingBackward a, int n, uint32_t across, uint32_t zero_groups) {
  __shared__ uint64_t same[kCountedTokens / 64];
  __shared__ uint16_t list[kCountedTokens];
  __shared__ float others[3][64][8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t sums = static_cast<uint32_t>(n) * across;
  uint32_t key[kCountedTokens / 256];
#pragma unroll
  for (int u = 0; u < kCountedTokens / 256; ++u) key[u] = kNoKey;
  if (n > 0) keys_of(a.ids, a.i64, static_cast<int>(threadIdx.x), 256, n, a.vocab, key);
  if (blockIdx.x >= sums) {
    uint32_t* present = reinterpret_cast<uint32_t*>(same);
    for (int64_t row0 = static_cast<int64_t>(blockIdx.x - sums) * kCountedZeroRows; row0 < a.vocab; row0 += static_cast<int64_t>(zero_groups) * kCountedZeroRows) {
      __syncthreads();
      if (threadIdx.x < 2) present[threadIdx.x] = 0u;
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kCountedTokens / 256; ++u) {
        const uint32_t r = key[u] - static_cast<uint32_t>(row0);
        if (r < kCountedZeroRows) atomicOr(&present[r >> 5], 1u << (r & 31));
      }
      __syncthreads();
      const int64_t left = a.vocab - row0;
      const uint64_t there = left < 64 ? (uint64_t{1} << left) - 1 : ~uint64_t{0};
      for (uint64_t absent = there & ~(static_cast<uint64_t>(present[1]) << 32 | present[0]); absent; absent &= absent - 1) {
        float* to = a.dtable + (row0 + __builtin_ctzll(absent)) * a.ldt;
        for (int64_t col = threadIdx.x * 4; col < a.cols; col += 1024) *reinterpret_cast<float4v*>(to + col) = float4v{0.0f, 0.0f, 0.0f, 0.0f};
      }
    }
    return;
  }
  const int t = static_cast<int>(blockIdx.x / across);
  uint32_t mine[1];
  keys_of(a.ids, a.i64, t, 1, n, a.vocab, mine);
  if (mine[0] >= static_cast<uint32_t>(a.vocab)) return;
#pragma unroll
  for (int u = 0; u < kCountedTokens / 256; ++u) {
    const uint64_t mask = __ballot(key[u] == mine[0]);
    if (lane == 0) same[u * 4 + wave] = mask;   // tokens 256 u + 64 wave on
  }
  __syncthreads();
  uint64_t m = lane < kCountedTokens / 64 ? same[lane] : 0ull;
  const int word = t >> 6;
  if (__ballot(lane < word ? m != 0 : lane == word && (m & ((uint64_t{1} << (t & 63)) - 1)) != 0)) return;   // not the first one
  int before = __popcll(m), total;
#pragma unroll
  for (int off = 1; off < kCountedTokens / 64; off <<= 1) {
    const int o = __shfl_up(before, off, 64);
    if (lane >= off) before += o;
  }
  total = __builtin_amdgcn_readlane(before, kCountedTokens / 64 - 1);
  before -= __popcll(m);
  const int64_t col = static_cast<int64_t>(blockIdx.x % across) * 512 + lane * 8, from = min(col, a.cols - 8);
  float sum[8] = {};
  if (total == 1) {
    if (wave > 0) return;
    Eight<kBf16> x;
    x.load(static_cast<const char*>(a.dout) + static_cast<int64_t>(t) * a.ldd * (kBf16 ? 2 : 4), from);
    x.get(sum);
  } else {
    if (wave == 0)
      for (; m; m &= m - 1) list[before++] = static_cast<uint16_t>(lane * 64 + __builtin_ctzll(m));
    __syncthreads();
    const int each = (total + 3) >> 2, first = wave * each, count = min(each, total - first);
    if (each <= 4) add_listed<kBf16, 4>(a, list + first, count, from, sum);
    else add_listed<kBf16, 16>(a, list + first, count, from, sum);
    add_wavefronts(sum, others);
  }
  if (wave > 0 || col >= a.cols) return;
  float* row = a.dtable + static_cast<int64_t>(mine[0]) * a.ldt;
#pragma unroll
  for (int i = 0; i < 8; ++i) sum[i] *= a.scale;
  if (a.accumulate) {
    Eight<false> old;
    float o[8];
    old.load(row, col);
    old.get(o);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] += o[i];
  }
  store8(row, col, false, sum);
}

// ---------------------------------------------------------------- launches

// Rows without a token: all rows written first, or those that have none looked for beside the sums (us on the GPU, first / looked for).  Up to 512 tokens by the table's bytes: 16 tokens into rows
// of 1024 columns, 8 MB 6.2 / 8.1, 16 MB 7.8 / 9.6, 64 MB 16.1 / 14.5, 256 MB 46 / 51, 1 GB 164 / 192; 512 tokens, 16 MB 9.3 / 10.1, 64 MB 17.9 / 14.6, 256 MB 50 / 55 -- where the launch more
// that writes them costs the host 2.5.  Beyond, by the rows to a token: 1040 tokens into rows of 2064, 1 15.0 / 16.7, 4 18.5 / 20.3, 8 23.2 / 25.7, 32 58 / 70; 8192 into rows of 2048, 1 37.5 / 36.0,
// 2 52.3 / 50.6, 4 77.5 / 79.5, 8 115 / 128, 16 192 / 218.
constexpr int64_t kFewTokensPerRow = 4, kZeroFirstBytes = 8 << 20;

struct SumPlan {
  int chunk, chunks, tiles, passes, digit_bits;
  size_t keys, order, counts, partials, bytes;   // places in the workspace, in words; two of keys and order each where there are passes
};
SumPlan plan(int64_t n, int64_t vocab, int64_t cols) {
  SumPlan p{};
  // 512 chunks, of eight tokens at least.  (us for the whole gradient from bf16 with 256 / 512 / 1024 chunks, 4000 x 5120: 8192 tokens 59 / 63 / 73, 16384 92 / 89 / 98, 32768 137 / 130 / 137, 65536
  // 216 / 213 / 216; with 4 / 8 / 16 tokens at least: 1040 into 5003 x 2064 19.4 / 19.3 / 20.8, 2048 into 3000 x 5120 34.9 / 30.5 / 27.5.)
  p.chunk = static_cast<int>(std::max<int64_t>(8, (n + 511) / 512));
  p.chunks = static_cast<int>((n + p.chunk - 1) / p.chunk);
  size_t at = 0;
  auto take = [&at](size_t words) {
    const size_t here = at;
    at += (words + 3) / 4 * 4;
    return here;
  };
  const bool few = n <= kFewTokens;
  p.keys = take(static_cast<size_t>(n) * (few ? 1 : 2));
  p.order = take(static_cast<size_t>(n) * (few ? 1 : 2));
  if (!few) {
    int bits = 1;
    while ((vocab >> bits) != 0) ++bits;
    p.passes = (bits + 8) / 9;
    p.digit_bits = (bits + p.passes - 1) / p.passes;
    p.tiles = static_cast<int>((n + kTile - 1) / kTile);
    p.counts = take(static_cast<size_t>(p.tiles) << p.digit_bits);
  }
  p.partials = take(static_cast<size_t>(p.chunks) * 2 * static_cast<size_t>(cols));
  p.bytes = at * 4;
  return p;
}

}  // namespace

size_t embedding_workspace_bytes(int64_t tokens, int64_t vocab, int64_t cols) { return tokens > kCountedTokens ? plan(tokens, vocab, cols).bytes : 0; }

hipError_t launch_embedding_forward(const EmbeddingForward& all, hipStream_t s) {
  EmbeddingForward a = all;
  const int64_t groups = a.cols / 8, most = std::max<int64_t>(1, (int64_t{1} << 33) / groups);   // tokens of a launch, which holds 2^32 threads
  for (; a.token0 < all.tokens; a.token0 += most) {
    a.tokens = std::min(all.tokens, a.token0 + most);
    const unsigned wgs = static_cast<unsigned>(((a.tokens - a.token0) * groups + 256 * kGroupsEach - 1) / (256 * kGroupsEach));
#define NVFP4_EMBED(T, O) hipLaunchKernelGGL((embedding_forward_kernel<T, O>), dim3(wgs), dim3(256), 0, s, a)
    if (a.table_bf16) {
      if (a.out_bf16) NVFP4_EMBED(true, true); else NVFP4_EMBED(true, false);
    } else {
      if (a.out_bf16) NVFP4_EMBED(false, true); else NVFP4_EMBED(false, false);
    }
#undef NVFP4_EMBED
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_embedding_backward(const EmbeddingBackward& a, void* workspace, hipStream_t s) {
  const int n = static_cast<int>(a.tokens);
  // Rows without a token: where tokens are few for the table all rows are written first, without looking; otherwise those that have none are looked for beside the sums.
  const bool few = n <= kCountedTokens, zero_first = !a.accumulate && (few ? a.vocab * a.cols * 4 > kZeroFirstBytes : a.tokens < a.vocab / kFewTokensPerRow);
  ZeroArgs z{};
  if (zero_first) {
    z.to = a.dtable, z.ld = a.ldt, z.across = static_cast<uint32_t>(a.cols / 4), z.pieces = a.vocab * z.across;
    z.groups = static_cast<uint32_t>(std::min<int64_t>((z.pieces + kRankThreads - 1) / kRankThreads, 1 << 22));   // (a launch holds 2^32 threads)
  }
  hipError_t e;
  if (zero_first && (few || n > kFewTokens)) {   // (otherwise in one launch with the ranking)
    hipLaunchKernelGGL(zero_kernel, dim3(z.groups), dim3(kRankThreads), 0, s, z);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (few) {
    const uint32_t across = static_cast<uint32_t>((a.cols + 511) / 512);
    const uint32_t zeros = a.accumulate || zero_first ? 0u : static_cast<uint32_t>(std::min<int64_t>((a.vocab + kCountedZeroRows - 1) / kCountedZeroRows, 1 << 16));
    if (n * across + zeros == 0) return hipSuccess;
    if (a.bf16) hipLaunchKernelGGL(embedding_few_kernel<true>, dim3(n * across + zeros), dim3(256), 0, s, a, n, across, zeros);
    else hipLaunchKernelGGL(embedding_few_kernel<false>, dim3(n * across + zeros), dim3(256), 0, s, a, n, across, zeros);
    return hipGetLastError();
  }
  const SumPlan p = plan(n, a.vocab, a.cols);
  uint32_t* words = static_cast<uint32_t*>(workspace);
  uint32_t *keys = words + p.keys, *order = words + p.order;
  if (n <= kFewTokens) {
    hipLaunchKernelGGL(rank_kernel, dim3((n + kRankTokens - 1) / kRankTokens + z.groups), dim3(kRankThreads), 0, s, a.ids, a.i64, n, a.vocab, keys, order, z);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  } else {
    SortPass q{};
    q.ids = a.ids, q.i64 = a.i64, q.vocab = a.vocab, q.n = n, q.tiles = p.tiles, q.digits = 1 << p.digit_bits, q.counts = words + p.counts;
    for (int pass = 0; pass < p.passes; ++pass) {
      q.first = pass == 0, q.shift = pass * p.digit_bits;
      q.keys = keys, q.order = order;
      keys = words + p.keys + (pass & 1 ? n : 0), order = words + p.order + (pass & 1 ? n : 0);
      q.to_keys = keys, q.to_order = order;
      hipLaunchKernelGGL(sort_count_kernel, dim3(p.tiles), dim3(256), 0, s, q);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      if (p.tiles > kFoldTiles) {
        hipLaunchKernelGGL(sort_scan_kernel, dim3(1), dim3(1024), 0, s, q.counts, p.tiles << p.digit_bits);
        if ((e = hipGetLastError()) != hipSuccess) return e;
      }
      hipLaunchKernelGGL(sort_place_kernel, dim3(p.tiles), dim3(256), 0, s, q);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  SumArgs u{};
  u.a = a, u.keys = keys, u.order = order, u.partials = reinterpret_cast<float*>(words + p.partials);
  u.n = n, u.chunk = p.chunk, u.chunks = p.chunks, u.strips = static_cast<int>((a.cols + 511) / 512);
  u.zero_groups = a.accumulate || zero_first ? 0u : static_cast<uint32_t>(std::min<int64_t>((a.vocab + kZeroRows - 1) / kZeroRows, 1 << 16));
  const int64_t wgs = (static_cast<int64_t>(u.chunks) * u.strips + 3) / 4 + u.zero_groups;
  if (a.bf16) hipLaunchKernelGGL(embedding_sum_kernel<true>, dim3(static_cast<unsigned>(wgs)), dim3(256), 0, s, u);
  else hipLaunchKernelGGL(embedding_sum_kernel<false>, dim3(static_cast<unsigned>(wgs)), dim3(256), 0, s, u);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (u.chunks > 1) hipLaunchKernelGGL(embedding_join_kernel, dim3(u.chunks, static_cast<unsigned>((a.cols + 255) / 256)), dim3(256), 0, s, u);
  return hipGetLastError();
}

}  // namespace nvfp4
