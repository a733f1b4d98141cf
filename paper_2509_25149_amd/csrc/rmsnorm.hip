// Root-mean-square norm with the residual's addition in front of it, and its gradient.
//   forward   h = x + r;  rstd = 1 / sqrt(mean(h^2) + eps);  xhat = h rstd;  y = xhat gamma;  optionally 8 bits of xhat or y
//   backward  g = dy gamma;  dx = rstd (g - xhat mean(g xhat)) + dres;  dgamma = sum over rows of dy xhat
// Sums, statistics and all arithmetic in FP32; every output is rounded once, from the FP32 value (the norm sees x + r before it is rounded for h).
// One pass: a row stays in registers between its sum and its output, eight columns to a lane and chunk.  Memory bounds both.  8192 x 5120, bf16 with residual
// and 8-bit output: 70 us for 380 MB (5.4 TB/s; a large copy runs at 5.1).
#include <algorithm>
#include <type_traits>

#include "nvfp4_internal.h"
#include "checkpoint8.h"

namespace nvfp4 {

namespace {

// Sum over the row's threads: a wavefront, or the workgroup through LDS (`red`: a float per wavefront, not reused before the next barrier).
template <bool kWaveRow>
__device__ __forceinline__ float row_sum(float v, float* red) {
  v = wave_sum(v);
  if (kWaveRow) return v;
  const int waves = blockDim.x >> 6;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = red[0];
  for (int w = 1; w < waves; ++w) s += red[w];
  return s;
}

// kWaveRow: a wavefront per row, otherwise a workgroup.  A lane holds columns (ch * threads + t) * 8 .. + 7 of chunk ch.
template <bool kXBf16, bool kHBf16, int kChunks, bool kWaveRow>
__global__ __launch_bounds__(kWaveRow ? 256 : 1024) void rmsnorm_forward_kernel(RmsNormForward a) {
  __shared__ float red[16];
  const int threads = kWaveRow ? 64 : blockDim.x, t = kWaveRow ? threadIdx.x & 63 : threadIdx.x;
  const int64_t row = kWaveRow ? static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6) : blockIdx.x;
  if (kWaveRow && row >= a.rows) return;
  const int cols = static_cast<int>(a.cols);
  const void* x = static_cast<const char*>(a.x) + row * a.ldx * (kXBf16 ? 2 : 4);
  const void* r = static_cast<const char*>(a.residual) + row * a.ldr * (kHBf16 ? 2 : 4);

  float h[kChunks][8];
  float sum = 0.0f;
  Eight<kXBf16> ex[kChunks];
  Eight<kHBf16> er[kChunks];
#pragma unroll
  for (int ch = 0; ch < kChunks; ++ch) {
    const int col = (ch * threads + t) * 8;
    if (col < cols) {
      ex[ch].load(x, col);
      if (a.residual) er[ch].load(r, col);
    }
  }
#pragma unroll
  for (int ch = 0; ch < kChunks; ++ch) {
    const int col = (ch * threads + t) * 8;
    if (col < cols) {
      ex[ch].get(h[ch]);
      if (a.residual) {
        float v[8];
        er[ch].get(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[ch][i] += v[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(h[ch][i], h[ch][i], sum);
    }
  }
  sum = row_sum<kWaveRow>(sum, red);
  const float rstd = 1.0f / __builtin_sqrtf(sum / static_cast<float>(cols) + a.eps);
  if (t == 0 && a.rstd) a.rstd[row] = rstd;

#pragma unroll
  for (int ch = 0; ch < kChunks; ++ch) {
    const int col = (ch * threads + t) * 8;
    if (col < cols) {
      if (a.h) store8(static_cast<char*>(a.h) + row * a.ldh * (kHBf16 ? 2 : 4), col, kHBf16, h[ch]);
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) h[ch][i] *= rstd;
      if (a.gamma) {
        const float4v *gp = reinterpret_cast<const float4v*>(a.gamma + col), g0 = gp[0], g1 = gp[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = h[ch][i] * g0[i], y[4 + i] = h[ch][4 + i] * g1[i];
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = h[ch][i];
      }
      if (a.y) store8(static_cast<char*>(a.y) + row * a.ldy * (a.y_bf16 ? 2 : 4), col, a.y_bf16, y);
      if (a.codes) {
        if (a.codes_of_y) {
#pragma unroll
          for (int i = 0; i < 8; ++i) h[ch][i] = y[i];
        }
        uint32_t m = max_magnitude(h[ch]);
        m = max(m, lane_xor1(m));   // (columns come in multiples of 16: both lanes of a block are here)
        const uint32_t byte = checkpoint_scale(m);
        *reinterpret_cast<uint2*>(a.codes + row * a.cols + col) = make_uint2(checkpoint_codes4(h[ch][0], h[ch][1], h[ch][2], h[ch][3], byte),
                                                                             checkpoint_codes4(h[ch][4], h[ch][5], h[ch][6], h[ch][7], byte));
        if ((t & 1) == 0) a.scales[row * (a.cols / 16) + col / 16] = static_cast<uint8_t>(byte);
      }
    }
  }
}

// What a lane holds of a row of the backward pass, as loaded: dy, xhat (h, or its 8 bits), dres.
template <bool kDyBf16, bool kSBf16, bool kSaved8, bool kDres>
struct BackwardEight {
  Eight<kDyBf16> dy;
  Eight<kSBf16> h, dres;
  uint2 codes;
  uint32_t byte;
  __device__ __forceinline__ void load(const RmsNormBackward& a, int64_t row, int col, bool with_dres) {
    dy.load(static_cast<const char*>(a.dy) + row * a.lddy * (kDyBf16 ? 2 : 4), col);
    if (kSaved8) {
      codes = *reinterpret_cast<const uint2*>(a.codes + row * a.cols + col);
      byte = a.scales[row * (a.cols / 16) + col / 16];
    } else {
      h.load(static_cast<const char*>(a.h) + row * a.ldh * (kSBf16 ? 2 : 4), col);
    }
    if (with_dres) load_dres(a, row, col);
  }
  __device__ __forceinline__ void load_dres(const RmsNormBackward& a, int64_t row, int col) {
    if (kDres) dres.load(static_cast<const char*>(a.dres) + row * a.lddr * (kSBf16 ? 2 : 4), col);
  }
  __device__ __forceinline__ void get_xhat(float rstd, float (&xhat)[8]) const {
    if (kSaved8) {
      checkpoint_values4(codes.x, byte, xhat);
      checkpoint_values4(codes.y, byte, xhat + 4);
    } else {
      h.get(xhat);
#pragma unroll
      for (int i = 0; i < 8; ++i) xhat[i] *= rstd;
    }
  }
  // dx = rstd (g - xhat c) + dres
  __device__ __forceinline__ void get_dx(const float (&g)[8], const float (&xhat)[8], float rstd, float c, float (&d)[8]) const {
    if (kDres) dres.get(d);
#pragma unroll
    for (int i = 0; i < 8; ++i) d[i] = rstd * (g[i] - xhat[i] * c) + (kDres ? d[i] : 0.0f);
  }
  __device__ __forceinline__ void forget() {
    dy.forget();
    if (kSaved8) asm volatile("" : "+v"(codes.x), "+v"(codes.y));
    else h.forget();
  }
};

__device__ __forceinline__ void load_gamma(const float* gamma, int col, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = 1.0f;
  if (gamma) {
    Eight<false> e;
    e.load(gamma, col);
    e.get(v);
  }
}

// Workgroup w takes rows w, w + parts, ... and leaves its sum of dy xhat in row w of the partial sums (kWaveRow: a wavefront per row, four of them
// in a workgroup add theirs through LDS).  The next row's loads are issued before the row in hand is worked on (kAhead): a workgroup waits for memory once
// a row otherwise, and few are resident.  For that nothing else may be loaded in the loop -- memory answers in order -- so gamma stays in registers, and
// columns and rows past the end are replaced by the last instead of being skipped.  8192 x 5120, bf16, from 8 bits, with dres: 57 us = 5.2 TB/s with the second launch's
// 4 us; 80 with twice as many workgroups that load a row, work on it and store it in turn.
// Four chunks (more than 16384 columns), and workgroups of more than 512 threads, have no registers for that; with four the sums are kept in LDS too (each
// lane its own) and dres is loaded where it is added.
template <bool kDyBf16, bool kSBf16, bool kSaved8, bool kDres, int kChunks, int kMaxThreads, bool kWaveRow>
__global__ __launch_bounds__(kMaxThreads) void rmsnorm_backward_kernel(RmsNormBackward a, float* __restrict__ partials, bool add) {
  constexpr bool kAhead = kMaxThreads <= 512, kLate = kChunks > 2;
  extern __shared__ __attribute__((aligned(16))) float lds[];   // a wavefront's sums in two halves, used in turn; kWaveRow: four rows of partial sums
  const int threads = kWaveRow ? 64 : blockDim.x, t = kWaveRow ? threadIdx.x & 63 : threadIdx.x;
  const int wave = threadIdx.x >> 6;
  const int cols = static_cast<int>(a.cols);
  const int64_t first = kWaveRow ? static_cast<int64_t>(blockIdx.x) * 4 + wave : blockIdx.x, step = kWaveRow ? static_cast<int64_t>(gridDim.x) * 4 : gridDim.x;
  const float inv = 1.0f / static_cast<float>(cols);
  int col[kChunks];   // of the lane's eight columns, or the row's last eight
  bool in[kChunks];
#pragma unroll
  for (int ch = 0; ch < kChunks; ++ch) {
    col[ch] = (ch * threads + t) * 8;
    in[ch] = col[ch] < cols;
    col[ch] = min(col[ch], cols - 8);
  }

  float dgamma[kLate ? 1 : kChunks][8] = {}, gamma[kAhead ? kChunks : 1][8];
  float* const kept = lds + 32;
#pragma unroll
  for (int ch = 0; ch < kChunks; ++ch) {
    if (kAhead) load_gamma(a.gamma, col[ch], gamma[kAhead ? ch : 0]);
    if (kLate && in[ch]) store8(kept, col[ch], false, dgamma[0]);
  }

  using Loaded = BackwardEight<kDyBf16, kSBf16, kSaved8, kDres>;
  Loaded row_in[kChunks], next_in[kAhead ? kChunks : 1];
  float rstd = 0.0f, next_rstd = 0.0f;
  if (kAhead && first < a.rows) {
#pragma unroll
    for (int ch = 0; ch < kChunks; ++ch) row_in[ch].load(a, first, col[ch], true);
    rstd = a.rstd[first];
  }
  int turn = 0;
  for (int64_t row = first; row < a.rows; row += step, turn ^= 16) {
    const int64_t from = kAhead ? min(row + step, a.rows - 1) : row;
#pragma unroll
    for (int ch = 0; ch < kChunks; ++ch) (kAhead ? next_in[kAhead ? ch : 0] : row_in[ch]).load(a, from, col[ch], !kLate);
    (kAhead ? next_rstd : rstd) = a.rstd[from];
    float sum = 0.0f;
#pragma unroll
    for (int ch = 0; ch < kChunks; ++ch) {
      if (in[ch]) {
        float g[8], xhat[8];
        row_in[ch].get_xhat(rstd, xhat);
        row_in[ch].dy.get(g);
        float(&into)[8] = dgamma[kLate ? 0 : ch];
        float(&gm)[8] = gamma[kAhead ? ch : 0];
        if (!kAhead) load_gamma(a.gamma, col[ch], gm);
        Eight<false> k;
        if (kLate) {
          k.load(kept, col[ch]);
          k.get(into);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          into[i] = __builtin_fmaf(g[i], xhat[i], into[i]);
          sum = __builtin_fmaf(g[i] * gm[i], xhat[i], sum);
        }
        if (kLate) store8(kept, col[ch], false, into);
      }
    }
    const float c = row_sum<kWaveRow>(sum, lds + turn) * inv;
#pragma unroll
    for (int ch = 0; ch < kChunks; ++ch) {
      if (in[ch] && a.dx) {
        float g[8], xhat[8], d[8];
        if (kLate) row_in[ch].forget();
        row_in[ch].get_xhat(rstd, xhat);
        row_in[ch].dy.get(g);
        float(&gm)[8] = gamma[kAhead ? ch : 0];
        if (!kAhead) load_gamma(a.gamma, col[ch], gm);
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] *= gm[i];
        if (kLate) row_in[ch].load_dres(a, row, col[ch]);
        row_in[ch].get_dx(g, xhat, rstd, c, d);
        store8(static_cast<char*>(a.dx) + row * a.lddx * (kSBf16 ? 2 : 4), col[ch], kSBf16, d);
      }
    }
    if (kAhead) {
#pragma unroll
      for (int ch = 0; ch < kChunks; ++ch) row_in[ch] = next_in[kAhead ? ch : 0];
      rstd = next_rstd;
    }
  }
  if (!partials) return;
  float* to = partials + static_cast<int64_t>(blockIdx.x) * a.cols;
  if (kWaveRow) {
#pragma unroll
    for (int ch = 0; ch < kChunks; ++ch)
      if (in[ch]) store8(lds + wave * cols, col[ch], false, dgamma[kLate ? 0 : ch]);
    __syncthreads();
    for (int c = threadIdx.x; c < cols; c += 256) {
      const float s = (lds[c] + lds[cols + c]) + (lds[2 * cols + c] + lds[3 * cols + c]);
      to[c] = add ? to[c] + s : s;
    }
  } else {
#pragma unroll
    for (int ch = 0; ch < kChunks; ++ch) {
      if (in[ch]) {
        float(&sums)[8] = dgamma[kLate ? 0 : ch];
        if (kLate) {
          Eight<false> k;
          k.load(kept, col[ch]);
          k.get(sums);
        }
        if (add) {
#pragma unroll
          for (int i = 0; i < 8; ++i) sums[i] += to[col[ch] + i];
        }
        store8(to, col[ch], false, sums);
      }
    }
  }
}

// Threads of a row and chunks of each: a wavefront up to 1024 columns, then a workgroup of as few threads as hold the row in 1 (up to 2048 columns),
// 2 (up to 16384) or 4 chunks.
struct RowShape {
  bool wave;
  int chunks, threads;
};
RowShape row_shape(int64_t cols) {
  const int eights = static_cast<int>(cols / 8);
  if (eights <= 64) return {true, 1, 64};
  if (eights <= 128) return {true, 2, 64};
  const int chunks = eights <= 256 ? 1 : eights <= 2048 ? 2 : 4;
  return {false, chunks, (eights + 64 * chunks - 1) / (64 * chunks) * 64};
}

template <bool kXBf16, bool kHBf16>
hipError_t forward_of(const RmsNormForward& a, hipStream_t s) {
  const RowShape p = row_shape(a.cols);
#define NVFP4_NORM(CH, WAVE) \
  hipLaunchKernelGGL((rmsnorm_forward_kernel<kXBf16, kHBf16, CH, WAVE>), dim3(static_cast<unsigned>(WAVE ? (a.rows + 3) / 4 : a.rows)), dim3(WAVE ? 256 : p.threads), 0, s, a)
  if (p.wave) {
    if (p.chunks == 1) NVFP4_NORM(1, true); else NVFP4_NORM(2, true);
  } else if (p.chunks == 1) {
    NVFP4_NORM(1, false);
  } else if (p.chunks == 2) {
    NVFP4_NORM(2, false);
  } else {
    NVFP4_NORM(4, false);
  }
#undef NVFP4_NORM
  return hipGetLastError();
}

constexpr int kMostCols = 32768;
// Workgroups of the backward pass: one to a CU where a row has 4096 columns or more, otherwise as many as have that many columns on their way together.  More
// of them write more partial sums (5120 columns: 5 MB from 256, 10 from 512) and get fewer rows each to overlap.  us with 2048 / 4096 / 8192 / 16384 columns:
// 8192 x 5120 60 / 60 / 63 / 69, x 2560 44 / 35 / 34 / 40, x 2048 37 / 28 / 30 / 36, x 1024 16 / 16 / 17 / 19, 1040 x 2064 13.1 / 12.9 / 15.9 / 17 (there 496 of the 512
// workgroups have two rows and 16 three).
// A few rows take one workgroup and no second launch (5120 columns, us on the GPU / called from Python: a row 3.4 / 6.9, four 7.3 / 7.1 so and 5.7 / 8.9 in two launches).
constexpr int64_t kColsOnTheWay = 4096, kCUs = 256, kFew = 3;
int backward_parts(int64_t rows, int64_t cols) {
  const int64_t each = row_shape(cols).wave ? 4 : 1, groups = (rows + each - 1) / each;
  if (groups <= kFew) return groups > 0 ? 1 : 0;
  const int64_t most = kCUs * ((kColsOnTheWay + cols * each - 1) / (cols * each));
  return static_cast<int>(groups < most ? groups : most);
}

template <bool kDyBf16, bool kSBf16, bool kSaved8, bool kDres>
hipError_t backward_of(const RmsNormBackward& a, int parts, float* partials, bool add, hipStream_t s) {
  const RowShape p = row_shape(a.cols);
  const unsigned lds = p.wave ? static_cast<unsigned>(a.cols) * 16 : 128 + (p.chunks == 4 ? static_cast<unsigned>(a.cols) * 4 : 0);
#define NVFP4_NORM(CH, MOST, WAVE) \
  hipLaunchKernelGGL((rmsnorm_backward_kernel<kDyBf16, kSBf16, kSaved8, kDres, CH, MOST, WAVE>), dim3(parts), dim3(WAVE ? 256 : p.threads), lds, s, a, partials, add)
  if (p.wave) {
    if (p.chunks == 1) NVFP4_NORM(1, 256, true); else NVFP4_NORM(2, 256, true);
  } else if (p.chunks == 1) {
    NVFP4_NORM(1, 256, false);
  } else if (p.chunks == 2) {
    if (p.threads <= 512) NVFP4_NORM(2, 512, false); else NVFP4_NORM(2, 1024, false);
  } else {
    static PerDeviceOnce once;
    const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void*>(&rmsnorm_backward_kernel<kDyBf16, kSBf16, kSaved8, kDres, 4, 1024, false>), 128 + kMostCols * 4, once);
    if (e != hipSuccess) return e;
    NVFP4_NORM(4, 1024, false);
  }
#undef NVFP4_NORM
  return hipGetLastError();
}

template <bool... kFlags>
hipError_t backward_with(const RmsNormBackward& a, int parts, float* partials, bool add, hipStream_t s) {
  if constexpr (sizeof...(kFlags) == 4) {
    return backward_of<kFlags...>(a, parts, partials, add, s);
  } else {
    const bool flags[] = {a.dy_bf16, a.s_bf16, a.codes != nullptr, a.dres != nullptr};
    return flags[sizeof...(kFlags)] ? backward_with<kFlags..., true>(a, parts, partials, add, s) : backward_with<kFlags..., false>(a, parts, partials, add, s);
  }
}

}  // namespace

// The same call from row r on, for at most `rows` of them.
static RmsNormForward rows_from(RmsNormForward a, int64_t r, int64_t rows) {
  auto on = [r](auto*& p, int64_t bytes) {
    if (p) p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(reinterpret_cast<uintptr_t>(p) + r * bytes);
  };
  on(a.x, a.ldx * (a.x_bf16 ? 2 : 4));
  on(a.residual, a.ldr * (a.h_bf16 ? 2 : 4));
  on(a.h, a.ldh * (a.h_bf16 ? 2 : 4));
  on(a.y, a.ldy * (a.y_bf16 ? 2 : 4));
  on(a.rstd, 4);
  on(a.codes, a.cols);
  on(a.scales, a.cols / 16);
  a.rows = std::min(a.rows - r, rows);
  return a;
}

hipError_t launch_rmsnorm_forward(const RmsNormForward& all, hipStream_t s) {
  const int64_t most = 0xfffffff0 / std::max(row_shape(all.cols).threads, 64) / 4 * 4;   // rows of a launch, which holds 2^32 threads
  for (int64_t r = 0; r < all.rows; r += most) {
    const RmsNormForward a = rows_from(all, r, most);
    const hipError_t e = a.x_bf16 ? (a.h_bf16 ? forward_of<true, true>(a, s) : forward_of<true, false>(a, s))
                                  : (a.h_bf16 ? forward_of<false, true>(a, s) : forward_of<false, false>(a, s));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

size_t rmsnorm_partial_bytes(int64_t rows, int64_t cols) {
  const int parts = backward_parts(rows, cols);
  return parts > 1 ? static_cast<size_t>(parts) * static_cast<size_t>(cols) * 4 : 0;
}

hipError_t launch_rmsnorm_backward(const RmsNormBackward& a, hipStream_t s) {
  const int parts = backward_parts(a.rows, a.cols);
  // One part is the sum itself.
  float* partials = a.dgamma ? (parts > 1 ? a.partials : a.dgamma) : nullptr;
  if (parts > 0) {
    const bool add = parts == 1 && a.accumulate;
    const hipError_t e = backward_with<>(a, parts, partials, add, s);
    if (e != hipSuccess) return e;
  }
  if (!a.dgamma || parts == 1) return hipSuccess;
  return launch_colsum(partials, parts, a.cols, a.dgamma, a.accumulate, s);
}

}  // namespace nvfp4
