// What the 4-wavefront GEMM kernels for gfx950 share besides their loops: the walk over the tiles, and the
// output stage: one wavefront's block of FP32 sums (128 x 128, say),
// held as 8 x 8 results of 16x16 MFMAs, or kMB x kNB of them (acc[i][j][r] = D[m = 16 i + (lane & 15)][n = 16 j + 4 (lane >> 4) + r]),
// times the tensor-level decode scales (App. B.3, after Eq. 5), to FP32 (optionally added into D) or bf16.
// Device code only.
#pragma once

#include <type_traits>

#include "checkpoint8.h"
#include "nvfp4_device.h"
#include "nvfp4_internal.h"

namespace nvfp4 {

// row0 / col0: the block's first row / column in D; rows / cols: how many of its 128 x 128 exist (multiples of 16,
// possibly <= 0).  Stored from the registers, 64 contiguous bytes per row and instruction:
//   FP32  a lane writes its 4 consecutive columns of one row (16 bytes; the four lanes of a row 64 bytes);
//   bf16  a lane's 4 columns are only 8 bytes, so two neighbouring 16-column blocks are stored together: lanes
//         16 apart (column groups 4q.. and 4(q+1)..) trade halves with v_permlane16_swap_b32, after which an
//         even group holds 8 consecutive columns of the first block and an odd group 8 of the second.
// Ordinary stores throughout.  Non-temporal ones were measured both ways: for bf16 results (activations and their
// gradients, which the caller reads next) they made the amax pass behind Fprop a third faster (96 -> 62 us) but Fprop
// itself 4 % slower; for FP32 results (weight gradients) they took 3 us off the quantizer call that follows a Wgrad,
// but a wavefront's output stage issues them at two thirds of the rate (11.7 against 8.2 us for its 64 stores, by
// timestamps inside the kernel; the Wgrad call 1.359 against 1.347 ms).  A wavefront's stores leave at about 1 KiB per
// 150 cycles whatever else the chip does (the four wavefronts of a CU share one path to the L2: 128 KiB of bf16 per
// tile take 2.3 us, another 2.6 us go to reading, scaling and converting the 256 sums), so what bounds
// the output stage is what a wavefront has to issue, not memory bandwidth.  Must be called by all 64 lanes.  (Reordering the bf16 block through LDS into 256-byte row pieces was tried
// with ordinary stores and measured no faster.)
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));

// The lane's number within its wavefront, asked of the hardware at the place of the call: the compiler can neither
// move the question nor keep an earlier answer in a register.
__device__ __forceinline__ int lane_id() {
  int lane;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(lane));
  return lane;
}

// Tile number pid of the tiling -> tile row and column: the tiles are walked in bands of 8 tile rows, column by
// column within a band.
__device__ __forceinline__ void tile_coordinates(int pid, int tiles_m, int tiles_n, int& tm, int& tn) {
  constexpr int kBand = 8;
  const int band = pid / (kBand * tiles_n);
  const int band_rows = min(kBand, tiles_m - band * kBand);
  const int in_band = pid - band * kBand * tiles_n;
  tm = band * kBand + in_band % band_rows;
  tn = in_band / band_rows;
}


// The two operands' tensor-level decode scales.  Per tensor: a[0] * b[0] for every output.  With a scale per row of an
// operand (App. B.1, last sentence) output (m, n) takes a[m] * b[n]: still constant along k, so still outside the sum.
struct TensorScales {
  const float* a;
  const float* b;
  bool a_per_row, b_per_row;
};

// scale of the four outputs (row m, columns n .. n + 3); m, n global indices inside the matrix (used by the kernels
// with small tiles; the 128 x 128 wave block below loads its scale vectors once)
__device__ __forceinline__ float4v scale4(const TensorScales& ts, float uniform, bool vec, bool in, int64_t m, int64_t n) {
  float4v s = {uniform, uniform, uniform, uniform};
  if (vec && in) {
    const float sa = ts.a[ts.a_per_row ? m : 0];
#pragma unroll
    for (int r = 0; r < 4; ++r) s[r] = sa * ts.b[ts.b_per_row ? n + r : 0];
  }
  return s;
}

// What a lane needs to know to store its part of a 128 x 128 block: kVec: an operand carries one scale per row; the
// lane's 8 x 4 columns (n = 16 j + 4 lq + r) then take their factors from sb, loaded once, and its 8 rows
// (m = 16 i + l16) one factor each.  Otherwise the product a[0] * b[0] serves every output.
// A lane's addresses are one pointer (its row l16, its first column) plus i * 16 rows plus a constant per j, which the
// stores carry as their immediate offsets.
// kNB: how many 16-column blocks a lane holds of its rows (8 for a 128-column block; an odd number's last one is paired with
// nothing).
template <bool kBf16Out, bool kVec, int kNB = 8>
struct WaveBlockStore {
  void* d;
  int64_t ldd, lane_first;
  int l16, nl, rows, cols;
  bool accumulate;
  float out_scale;
  float4v sb[kVec ? kNB : 1];

  __device__ __forceinline__ WaveBlockStore(const TensorScales ts, void* Dv, int64_t ldd_, bool accumulate_, int64_t row0, int64_t col0,
                                            int rows_, int cols_, int lane)
      : d(Dv), ldd(ldd_), l16(lane & 15), rows(rows_), cols(cols_ < 16 * kNB ? cols_ : 16 * kNB), accumulate(accumulate_), out_scale(ts.a[0] * ts.b[0]) {
    const int lq = lane >> 4;
    // bf16: after the exchange a lane of an even column group holds 8 consecutive columns of block j, a lane of an odd
    // group 8 of block j + 1: column 16 j + nl, nl = 0, 16, 8, 24 for lq = 0 .. 3.
    nl = kBf16Out ? (lq & 1) * 16 + (lq >> 1) * 8 : lq * 4;
    lane_first = (row0 + l16) * ldd + col0 + nl;
    if (kVec) {
#pragma unroll
      for (int j = 0; j < kNB; ++j) {
        if (ts.b_per_row && j * 16 + lq * 4 < cols) {
          sb[kVec ? j : 0] = *reinterpret_cast<const float4v*>(ts.b + col0 + j * 16 + lq * 4);
        } else {
          const float b0 = ts.b[0];
          sb[kVec ? j : 0] = float4v{b0, b0, b0, b0};
        }
      }
    }
  }

  // the factor of the lane's row in 16-row block i (kVec only)
  __device__ __forceinline__ float row_scale(const TensorScales ts, int64_t row0, int i) const {
    return ts.a[ts.a_per_row && i * 16 + l16 < rows ? row0 + i * 16 + l16 : 0];
  }

  // The lane's 8 x 4 sums of 16-row block i: row m = 16 i + l16, columns 16 j + 4 lq + r.
  __device__ __forceinline__ void store_rows(const float4v (&sums)[kNB], int i, float sa) const {
    auto scale = [&](int j) -> float4v {
      if (kVec) return sb[kVec ? j : 0] * sa;
      return float4v{out_scale, out_scale, out_scale, out_scale};
    };
    const bool row_in = i * 16 + l16 < rows;
    if (kBf16Out) {
      uint16_t* d_row = static_cast<uint16_t*>(d) + lane_first + i * 16 * ldd;
#pragma unroll
      for (int j = 0; j < kNB; j += 2) {
        const float4v va = sums[j] * scale(j), vb = j + 1 < kNB ? sums[j + 1 < kNB ? j + 1 : j] * scale(j + 1 < kNB ? j + 1 : j) : float4v{0.0f, 0.0f, 0.0f, 0.0f};
        const uint32_t a0 = f32x2_to_bf16(va[0], va[1]), a1 = f32x2_to_bf16(va[2], va[3]);
        const uint32_t b0 = f32x2_to_bf16(vb[0], vb[1]), b1 = f32x2_to_bf16(vb[2], vb[3]);
        // first result: lanes of odd groups now hold the second block's dword of the group below; second result: lanes of
        // even groups now hold the first block's dword of the group above
        const auto s0 = __builtin_amdgcn_permlane16_swap(a0, b0, false, false);
        const auto s1 = __builtin_amdgcn_permlane16_swap(a1, b1, false, false);
        const u32x4v o = {s0[0], s1[0], s0[1], s1[1]};
        // columns come in multiples of 16, so the 8 columns are in or out together
        if (row_in && j * 16 + nl < cols) *reinterpret_cast<u32x4v*>(d_row + j * 16) = o;
      }
    } else {
      float* d_row = static_cast<float*>(d) + lane_first + i * 16 * ldd;
#pragma unroll
      for (int j = 0; j < kNB; ++j) {
        if (row_in && j * 16 + nl < cols) {  // columns come in multiples of 16, so the 4 columns are in or out together
          float4v v = sums[j] * scale(j);
          float* p = d_row + j * 16;
          if (accumulate) v += *reinterpret_cast<const float4v*>(p);
          *reinterpret_cast<float4v*>(p) = v;
        }
      }
    }
  }
};

// A wavefront's whole 128 x 128 block.  (A variant without the predicates for blocks that exist whole measured no
// faster.)  A kernel should contain this once: where a second use of the sums sits in another branch, the compiler
// reads all 256 out of the accumulation registers ahead of the branch, into registers it does not have.
template <bool kBf16Out, bool kVec, int kMB, int kNB>
__device__ __forceinline__ void store_wave_block_impl(float4v (&acc)[kMB][kNB], const TensorScales ts, void* __restrict__ Dv, int64_t ldd,
                                                      bool accumulate, int64_t row0, int64_t col0, int rows, int cols, int lane) {
  const WaveBlockStore<kBf16Out, kVec, kNB> out(ts, Dv, ldd, accumulate, row0, col0, rows, cols, lane);
  float sa[kVec ? kMB : 1] = {};
  if (kVec) {
#pragma unroll
    for (int i = 0; i < kMB; ++i) sa[kVec ? i : 0] = out.row_scale(ts, row0, i);
  }
#pragma unroll
  for (int i = 0; i < kMB; ++i) out.store_rows(acc[i], i, sa[kVec ? i : 0]);
}

// The per-tensor form, for kernels that have no other.
template <bool kBf16Out, int kNB = 8>
__device__ __forceinline__ void store_wave_block(float4v (&acc)[8][kNB], const TensorScales ts, void* __restrict__ Dv, int64_t ldd,
                                                 bool accumulate, int64_t row0, int64_t col0, int rows, int cols, int lane) {
  store_wave_block_impl<kBf16Out, false, 8, kNB>(acc, ts, Dv, ldd, accumulate, row0, col0, rows, cols, lane);
}


// ---------------------------------------------------------------- what nvfp4_gemm_epilogue does to the scaled sums
//   z = sum + bias;  8 bits of z are kept;  D = act(z) + residual             (kForward; kResidualF32, kResidualBf16: with a residual)
//   D = sum * act'(z), z from its 8 bits                                       (kGrad)
// All of it in FP32 in registers, D rounded once.  The kinds are instances of their own because all but the first load as much as they store, and the
// compiler waits for the right loads only where it knows how many follow them; bias, activation, what is kept and D's type are decided at run time, alike
// for the whole launch.
enum EpilogueKind { kNoEpilogue = 0, kForward = 1, kResidualF32 = 2, kResidualBf16 = 3, kGrad = 4 };
template <int kKind>
struct EpilogueArg : GemmEpilogue {
  __host__ __device__ EpilogueArg(const GemmEpilogue& e) : GemmEpilogue(e) {}
};
template <>
struct EpilogueArg<kNoEpilogue> {};
inline EpilogueKind epilogue_kind(const GemmEpilogue* e) { return !e ? kNoEpilogue : e->grad_codes ? kGrad : !e->residual ? kForward : e->residual_bf16 ? kResidualBf16 : kResidualF32; }

// Lanes 16 apart hold the rows of a 4 x 4 matrix of words, each lane a row: lane group q gets column q (its own inverse).
__device__ __forceinline__ void transpose4(uint32_t (&w)[4]) {
  const auto a = __builtin_amdgcn_permlane16_swap(w[0], w[1], false, false), b = __builtin_amdgcn_permlane16_swap(w[2], w[3], false, false);
  const auto c = __builtin_amdgcn_permlane32_swap(a[0], b[0], false, false), d = __builtin_amdgcn_permlane32_swap(a[1], b[1], false, false);
  w[0] = c[0], w[1] = d[0], w[2] = c[1], w[3] = d[1];
}
// The words of the four lane groups, in every lane.
__device__ __forceinline__ void gather4(uint32_t v, uint32_t (&w)[4]) {
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  const auto c = __builtin_amdgcn_permlane32_swap(a[0], a[0], false, false), d = __builtin_amdgcn_permlane32_swap(a[1], a[1], false, false);
  w[0] = c[0], w[1] = d[0], w[2] = c[1], w[3] = d[1];
}
// Largest of the lane groups' values (16x16 results), or of the two halves' (32x32 results), in all of them.
__device__ __forceinline__ uint32_t max_over_halves(uint32_t v) {
  const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(a[0], a[1]);
}
__device__ __forceinline__ uint32_t max_over_groups(uint32_t v) {
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return max_over_halves(max(a[0], a[1]));
}

// One 16-column block, for the kernels that store block by block: the lane holds kGroups groups of four columns of row m, n0 + first + 8 g .. + 3 (one
// group for 16x16 results, first = 4 (lane >> 4); two for 32x32, first = 4 (lane >> 5)).  The lanes that share a row's block come together; `in`: the row
// exists.  fetch() what is added or multiplied, of several blocks before the first is finished; finish() stores D too.  kLoads: whether there can be a residual
// or a derivative.
template <int kGroups, bool kLoads>
struct EpilogueOfBlock {
  float4v bias[kGroups];
  u32x4v residual[kGroups];   // as loaded (bf16: in the first two words)
  uint32_t codes[kGroups], byte;

  __device__ __forceinline__ void fetch(const GemmEpilogue& e, int64_t m, int64_t n0, int first, bool in) {
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      bias[g] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
      codes[g] = 0u;
    }
    byte = 0u;
    if (e.bias) {
#pragma unroll
      for (int g = 0; g < kGroups; ++g) bias[g] = *reinterpret_cast<const float4v*>(e.bias + n0 + first + 8 * g);
    }
    if (kLoads && e.residual && in) {
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        const int64_t at = m * e.ldr + n0 + first + 8 * g;
        if (e.residual_bf16) {
          const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(e.residual) + at);
          residual[g][0] = w.x, residual[g][1] = w.y;
        } else {
          residual[g] = *reinterpret_cast<const u32x4v*>(static_cast<const float*>(e.residual) + at);
        }
      }
    }
    if (kLoads && e.grad_codes && in) {
      const int64_t at = m * e.cols + n0;
      byte = e.grad_scales[at / 16];
#pragma unroll
      for (int g = 0; g < kGroups; ++g) codes[g] = *reinterpret_cast<const uint32_t*>(e.grad_codes + at + first + 8 * g);
    }
  }

  __device__ __forceinline__ void finish(const float4v (&v)[kGroups], const GemmEpilogue& e, void* __restrict__ Dv, int64_t ldd, int64_t m, int64_t n0, int first, bool in) const {
    float z[kGroups * 4];
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
#pragma unroll
      for (int r = 0; r < 4; ++r) z[4 * g + r] = v[g][r] + bias[g][r];
    if (kLoads && e.grad_codes) {
      float slope[kGroups * 4];
#pragma unroll
      for (int g = 0; g < kGroups; ++g) checkpoint_values4(codes[g], byte, slope + 4 * g);
      activation_slope(slope, e.act);
#pragma unroll
      for (int i = 0; i < kGroups * 4; ++i) z[i] *= slope[i];
    } else {
      if (e.keep_codes) {
        const int64_t at = m * e.cols + n0;
        const uint32_t b = checkpoint_scale(kGroups == 1 ? max_over_groups(max_magnitude(z)) : max_over_halves(max_magnitude(z)));
        if (in) {
#pragma unroll
          for (int g = 0; g < kGroups; ++g)
            *reinterpret_cast<uint32_t*>(e.keep_codes + at + first + 8 * g) = checkpoint_codes4(z[4 * g], z[4 * g + 1], z[4 * g + 2], z[4 * g + 3], b);
          if (first == 0) e.keep_scales[at / 16] = static_cast<uint8_t>(b);
        }
      }
      activate(z, e.act);
    }
    if (!in) return;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int64_t n = n0 + first + 8 * g;
      float4v d = {z[4 * g], z[4 * g + 1], z[4 * g + 2], z[4 * g + 3]};
      if (kLoads && e.residual) {
        const u32x4v w = residual[g];
#pragma unroll
        for (int r = 0; r < 4; ++r) d[r] += !e.residual_bf16 ? __uint_as_float(w[r]) : r % 2 ? bf16_hi(w[r / 2]) : bf16_lo(w[r / 2]);
      }
      if (e.out_bf16) *reinterpret_cast<uint2*>(static_cast<uint16_t*>(Dv) + m * ldd + n) = make_uint2(f32x2_to_bf16(d[0], d[1]), f32x2_to_bf16(d[2], d[3]));
      else *reinterpret_cast<float4v*>(static_cast<float*>(Dv) + m * ldd + n) = d;
    }
  }
};

// A wavefront's whole block of kMB x kNB 16x16 results, 16 rows of four blocks (64 columns) at a time, row by row: a row's lines fill up at once.  (Column
// group by column group, which needs the bias of one group only, MXFP4 8192 x 20480 x 5120 takes 432 us instead of 418 without anything to do, 528 instead of
// 472 with the 8 bits.)  What such a unit loads (residual, or 8 bits) is asked for kAhead units before it is needed; addresses past the end are
// replaced by the last in range rather than skipped, so that the number of loads in flight is known to the compiler.  (Asked for earlier still, during the loop's
// last steps and into LDS that nobody reads, so that the output stage finds it in the L2: the loop's own loads wait behind these; 1.12 ms plus 50 us became plus 70.)  The 8 bits move as 16 bytes of one block to a
// lane, bf16 as in WaveBlockStore.
template <int kKind, int kMB, int kNB>
struct EpilogueBlock {
  static constexpr int kGroups = (kNB + 3) / 4, kUnits = kGroups * kMB, kAhead = kKind == kResidualF32 ? 5 : kKind == kGrad ? 12 : 8;
  static constexpr bool kResidual = kKind == kResidualF32 || kKind == kResidualBf16, kLoads = kResidual || kKind == kGrad;
  struct Loads {
    u32x4v w[kKind == kResidualF32 ? 4 : kKind == kResidualBf16 ? 2 : 1];
    uint32_t byte;
  };
  const GemmEpilogue& e;
  const float* ts_b;
  int64_t ldd, row0, col0;
  int rows, cols, l16, lq, nl;   // nl: the lane's first column in a pair of bf16 blocks
  bool a_per_row, b_per_row;
  // The lane's place in the block's first 16 rows; 16-row block i is i * 16 leading dimensions on, the same for all lanes.
  char* d;
  const char* residual;
  uint8_t *codes, *scales;       // of block lq

  __device__ __forceinline__ EpilogueBlock(const GemmEpilogue& e_, const TensorScales& ts, void* Dv, int64_t ldd_, int64_t row0_, int64_t col0_, int rows_, int cols_, int lane)
      : e(e_), ts_b(ts.b), ldd(ldd_), row0(row0_), col0(col0_), rows(rows_), cols(cols_), l16(lane & 15), lq(lane >> 4), nl((lq & 1) * 16 + (lq >> 1) * 8),
        a_per_row(ts.a_per_row), b_per_row(ts.b_per_row) {
    const int64_t row = row0 + l16;
    d = static_cast<char*>(Dv) + (e.out_bf16 ? (row * ldd + col0 + nl) * 2 : (row * ldd + col0 + 4 * lq) * 4);
    if constexpr (kKind == kResidualF32) residual = static_cast<const char*>(e.residual) + (row * e.ldr + col0 + 4 * lq) * 4;
    if constexpr (kKind == kResidualBf16) residual = static_cast<const char*>(e.residual) + (row * e.ldr + col0 + (nl & 15)) * 2;
    const int64_t at = row * e.cols + col0;
    codes = (kKind == kGrad ? const_cast<uint8_t*>(e.grad_codes) : e.keep_codes) + at;
    scales = (kKind == kGrad ? const_cast<uint8_t*>(e.grad_scales) : e.keep_scales) + at / 16;
  }

  // 16-row block i and column block j, or the last that exist (rows and columns come in multiples of 16; a block past the end may start behind them all).
  __device__ __forceinline__ int row_block(int i) const { return min(i, (rows >> 4) - 1); }
  __device__ __forceinline__ int col_block(int j) const { return min(j, (cols >> 4) - 1); }

  __device__ __forceinline__ void fetch(Loads& l, int i, int jg) const {
    const int64_t down = static_cast<int64_t>(row_block(i)) * 16;
    if constexpr (kKind == kResidualF32) {
      const char* p = residual + down * e.ldr * 4;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (4 * jg + k < kNB) l.w[k] = *reinterpret_cast<const u32x4v*>(p + col_block(4 * jg + k) * 64);
    }
    if constexpr (kKind == kResidualBf16) {
      const char* p = residual + down * e.ldr * 2;
#pragma unroll
      for (int k = 0; k < 4; k += 2)
        if (4 * jg + k < kNB) l.w[k / 2] = *reinterpret_cast<const u32x4v*>(p + col_block(min(4 * jg + k + (nl >> 4), kNB - 1)) * 32);
    }
    if constexpr (kKind == kGrad) {
      const int j = col_block(min(4 * jg + lq, kNB - 1));
      l.w[0] = *reinterpret_cast<const u32x4v*>(codes + down * e.cols + j * 16);
      l.byte = scales[down * (e.cols >> 4) + j];
    }
  }

  // The bias of the lane's columns.
  __device__ __forceinline__ void columns(float4v (&bias)[kKind == kGrad ? 1 : kNB]) const {
    if constexpr (kKind != kGrad) {
#pragma unroll
      for (int j = 0; j < kNB; ++j) {
        bias[j] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
        if (e.bias) bias[j] = *reinterpret_cast<const float4v*>(e.bias + col0 + col_block(j) * 16 + 4 * lq);
      }
    }
  }

  // The operands' factors: their product where neither has one per row; otherwise A's of each of the lane's rows, and B's first.  (B's are read where they are
  // used, which waits for all that is in flight: 8192 x 20480 x 5120 with a residual 1228 us instead of 1136.)
  struct Factors {
    float uniform, a[kMB], b0;
  };

  // sums: the unit's blocks, unscaled: four of them, or what is left at the end of a row.
  template <int kBlocks>
  __device__ __forceinline__ void finish(float4v (&sums)[kBlocks], const Loads& l, int i, int jg, const Factors& f, const float4v (&bias)[kKind == kGrad ? 1 : kNB]) const {
    const bool row_in = i * 16 < rows;
    const int64_t down = static_cast<int64_t>(i) * 16;
    if (a_per_row || b_per_row) {
#pragma unroll
      for (int k = 0; k < kBlocks; ++k) {
        float4v sb = {f.b0, f.b0, f.b0, f.b0};
        if (b_per_row) sb = *reinterpret_cast<const float4v*>(ts_b + col0 + col_block(4 * jg + k) * 16 + 4 * lq);
        sums[k] *= sb * f.a[i];
      }
    } else {
#pragma unroll
      for (int k = 0; k < kBlocks; ++k) sums[k] *= f.uniform;
    }
    float z[4 * kBlocks];
#pragma unroll
    for (int t = 0; t < 4 * kBlocks; ++t) z[t] = sums[t / 4][t % 4] + (kKind == kGrad ? 0.0f : bias[kKind == kGrad ? 0 : 4 * jg + t / 4][t % 4]);
    if constexpr (kKind == kGrad) {
      uint32_t codes4[4] = {l.w[0][0], l.w[0][1], l.w[0][2], l.w[0][3]}, bytes[4];
      transpose4(codes4);
      gather4(l.byte, bytes);
      float slope[4 * kBlocks];
#pragma unroll
      for (int k = 0; k < kBlocks; ++k) checkpoint_values4(codes4[k], bytes[k], slope + 4 * k);
      activation_slope(slope, e.act);
#pragma unroll
      for (int t = 0; t < 4 * kBlocks; ++t) z[t] *= slope[t];
    } else {
      if (e.keep_codes) {
        uint32_t m[4], w[4], bytes[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int t = k < kBlocks ? 4 * k : 0;
          m[k] = k < kBlocks ? max(max(magnitude(z[t]), magnitude(z[t + 1])), max(magnitude(z[t + 2]), magnitude(z[t + 3]))) : 0u;
        }
        transpose4(m);
        const uint32_t byte = checkpoint_scale(max(max(m[0], m[1]), max(m[2], m[3])));   // of block 4 jg + lq
        gather4(byte, bytes);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int t = k < kBlocks ? 4 * k : 0;
          w[k] = k < kBlocks ? checkpoint_codes4(z[t], z[t + 1], z[t + 2], z[t + 3], bytes[k]) : 0u;
        }
        transpose4(w);
        const int c = 16 * (4 * jg + lq);
        if (row_in && lq < kBlocks && c < cols) {
          *reinterpret_cast<u32x4v*>(codes + down * e.cols + c) = u32x4v{w[0], w[1], w[2], w[3]};
          scales[down * (e.cols >> 4) + (c >> 4)] = static_cast<uint8_t>(byte);
        }
      }
      activate(z, e.act);
      if constexpr (kKind == kResidualF32) {
#pragma unroll
        for (int t = 0; t < 4 * kBlocks; ++t) z[t] += __uint_as_float(l.w[t / 4][t % 4]);
      }
      if constexpr (kKind == kResidualBf16) {
#pragma unroll
        for (int k = 0; k < kBlocks; ++k) {
          // (the exchange of the stores below, backwards)
          const u32x4v p = l.w[k / 2];
          const auto s0 = __builtin_amdgcn_permlane16_swap(p[0], p[2], false, false), s1 = __builtin_amdgcn_permlane16_swap(p[1], p[3], false, false);
          z[4 * k] += bf16_lo(s0[k % 2]), z[4 * k + 1] += bf16_hi(s0[k % 2]);
          z[4 * k + 2] += bf16_lo(s1[k % 2]), z[4 * k + 3] += bf16_hi(s1[k % 2]);
        }
      }
    }
    if (e.out_bf16) {
      uint16_t* to = reinterpret_cast<uint16_t*>(d) + down * ldd;
#pragma unroll
      for (int k = 0; k < kBlocks; k += 2) {
        constexpr int kEnd = 4 * kBlocks;
        const uint32_t a0 = f32x2_to_bf16(z[4 * k], z[4 * k + 1]), a1 = f32x2_to_bf16(z[4 * k + 2], z[4 * k + 3]);
        const uint32_t b0 = 4 * k + 4 < kEnd ? f32x2_to_bf16(z[(4 * k + 4) % kEnd], z[(4 * k + 5) % kEnd]) : 0u;
        const uint32_t b1 = 4 * k + 4 < kEnd ? f32x2_to_bf16(z[(4 * k + 6) % kEnd], z[(4 * k + 7) % kEnd]) : 0u;
        const auto s0 = __builtin_amdgcn_permlane16_swap(a0, b0, false, false), s1 = __builtin_amdgcn_permlane16_swap(a1, b1, false, false);
        const int c = 16 * (4 * jg + k);
        if (row_in && c + nl < cols && (k + 1 < kBlocks || nl < 16)) *reinterpret_cast<u32x4v*>(to + c) = u32x4v{s0[0], s1[0], s0[1], s1[1]};
      }
    } else {
      float* to = reinterpret_cast<float*>(d) + down * ldd;
#pragma unroll
      for (int k = 0; k < kBlocks; ++k) {
        const int c = 16 * (4 * jg + k);
        if (row_in && c < cols) *reinterpret_cast<float4v*>(to + c) = float4v{z[4 * k], z[4 * k + 1], z[4 * k + 2], z[4 * k + 3]};
      }
    }
  }
};

template <int kBegin, int kEnd, class F>
__device__ __forceinline__ void each(F&& f) {
  if constexpr (kBegin < kEnd) {
    f(std::integral_constant<int, kBegin>{});
    each<kBegin + 1, kEnd>(f);
  }
}

// A result in accumulation registers, read where it is used: left to itself the compiler moves reads up until the registers do not suffice.
__device__ __forceinline__ float4v read_acc(const float4v& a) {
  float4v v;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    float x;
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(a[r]));
    v[r] = x;
  }
  return v;
}

// kInAcc: how many of the results, counted row by row, are in accumulation registers.
template <int kKind, int kInAcc, int kMB, int kNB>
__device__ __forceinline__ void store_wave_block_epilogue(float4v (&acc)[kMB][kNB], const TensorScales& ts, const GemmEpilogue& e, void* __restrict__ Dv, int64_t ldd,
                                                          int64_t row0, int64_t col0, int rows, int cols, int lane) {
  using Block = EpilogueBlock<kKind, kMB, kNB>;
  const Block b(e, ts, Dv, ldd, row0, col0, rows, cols, lane);
  constexpr int kAhead = Block::kAhead, kUnits = Block::kUnits, kGroups = Block::kGroups;
  constexpr bool kLoads = Block::kLoads;
  typename Block::Factors factors;
  factors.uniform = ts.a[0] * ts.b[0], factors.b0 = ts.b[0];
#pragma unroll
  for (int i = 0; i < kMB; ++i) factors.a[i] = ts.a[b.a_per_row ? row0 + b.row_block(i) * 16 + b.l16 : 0];
  float4v bias[kKind == kGrad ? 1 : kNB];
  b.columns(bias);
  typename Block::Loads ring[kLoads ? kAhead : 1];
  if constexpr (kLoads) each<0, (kAhead < kUnits ? kAhead : kUnits)>([&](auto u) { b.fetch(ring[decltype(u)::value], decltype(u)::value / kGroups, decltype(u)::value % kGroups); });
  each<0, kUnits>([&](auto uc) {
    constexpr int u = decltype(uc)::value, i = u / kGroups, jg = u % kGroups, kBlocks = 4 * jg + 4 <= kNB ? 4 : kNB - 4 * jg;
    float4v sums[kBlocks];
#pragma unroll
    for (int k = 0; k < kBlocks; ++k) sums[k] = i * kNB + 4 * jg + k < kInAcc ? read_acc(acc[i][4 * jg + k]) : acc[i][4 * jg + k];
    b.template finish<kBlocks>(sums, ring[kLoads ? u % kAhead : 0], i, jg, factors, bias);
    if constexpr (kLoads && u + kAhead < kUnits) b.fetch(ring[u % kAhead], (u + kAhead) / kGroups, (u + kAhead) % kGroups);
    __builtin_amdgcn_sched_barrier(0);
  });
}

}  // namespace nvfp4
