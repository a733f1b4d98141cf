// Root-mean-square norm with the residual's addition in front of it, and its gradient.
//   forward   h = x + r;  rstd = 1 / sqrt(mean(h^2) + eps);  xhat = h rstd;  y = xhat gamma;  optionally 8 bits of xhat or y
//   backward  g = dy gamma;  dx = rstd (g - xhat mean(g xhat)) + dres;  dgamma = sum over rows of dy xhat
// Sums, statistics and all arithmetic in FP32; every output is rounded once, from the FP32 value (the norm sees x + r before it is rounded for h).
// One pass: a row stays in registers between its sum and its output, eight columns to a lane and chunk.
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
template <bool kDyBf16, bool kSBf16, bool kSaved8>
struct BackwardEight {
  Eight<kDyBf16> dy;
  Eight<kSBf16> h, dres;
  uint2 codes;
  uint32_t byte;
  // g = dy gamma and xhat
  __device__ __forceinline__ void get(const float* gamma, int col, float rstd, float (&g)[8], float (&xhat)[8]) const {
    if (kSaved8) {
      checkpoint_values4(codes.x, byte, xhat);
      checkpoint_values4(codes.y, byte, xhat + 4);
    } else {
      h.get(xhat);
#pragma unroll
      for (int i = 0; i < 8; ++i) xhat[i] *= rstd;
    }
    dy.get(g);
    if (gamma) {
      const float4v *gp = reinterpret_cast<const float4v*>(gamma + col), g0 = gp[0], g1 = gp[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) g[i] *= g0[i], g[4 + i] *= g1[i];
    }
  }
};

// Workgroup w takes rows w, w + parts, ... and leaves its sum of dy xhat in row w of the partial sums (kWaveRow: a wavefront per row, four of them
// in a workgroup add theirs through LDS).
template <bool kDyBf16, bool kSBf16, bool kSaved8, int kChunks, bool kWaveRow>
__global__ __launch_bounds__(kWaveRow ? 256 : 1024) void rmsnorm_backward_kernel(RmsNormBackward a, float* __restrict__ partials, bool add) {
  // Four chunks: there are no registers for everything; the sums are kept in LDS (each lane its own) and dres is loaded where it is added.
  constexpr bool kLate = kChunks > 2;
  extern __shared__ __attribute__((aligned(16))) float lds[];   // a wavefront's sums in two halves, used in turn; kWaveRow: four rows of partial sums
  const int threads = kWaveRow ? 64 : blockDim.x, t = kWaveRow ? threadIdx.x & 63 : threadIdx.x;
  const int wave = threadIdx.x >> 6;
  const int cols = static_cast<int>(a.cols);
  const int64_t first = kWaveRow ? static_cast<int64_t>(blockIdx.x) * 4 + wave : blockIdx.x, step = kWaveRow ? static_cast<int64_t>(gridDim.x) * 4 : gridDim.x;
  const float inv = 1.0f / static_cast<float>(cols);

  float dgamma[kLate ? 1 : kChunks][8] = {};
  float* const kept = lds + 32;
  if (kLate) {
#pragma unroll
    for (int ch = 0; ch < kChunks; ++ch) {
      const int col = (ch * threads + t) * 8;
      if (col < cols) store8(kept, col, false, dgamma[0]);
    }
  }

  int turn = 0;
  for (int64_t row = first; row < a.rows; row += step, turn ^= 16) {
    const void* dy = static_cast<const char*>(a.dy) + row * a.lddy * (kDyBf16 ? 2 : 4);
    const void* h = static_cast<const char*>(a.h) + row * a.ldh * (kSBf16 ? 2 : 4);
    const void* dres = static_cast<const char*>(a.dres) + row * a.lddr * (kSBf16 ? 2 : 4);
    BackwardEight<kDyBf16, kSBf16, kSaved8> in[kChunks];
#pragma unroll
    for (int ch = 0; ch < kChunks; ++ch) {
      const int col = (ch * threads + t) * 8;
      if (col < cols) {
        in[ch].dy.load(dy, col);
        if (kSaved8) {
          in[ch].codes = *reinterpret_cast<const uint2*>(a.codes + row * a.cols + col);
          in[ch].byte = a.scales[row * (a.cols / 16) + col / 16];
        } else {
          in[ch].h.load(h, col);
        }
        if (a.dres && !kLate) in[ch].dres.load(dres, col);
      }
    }
    const float rstd = a.rstd[row];
    float sum = 0.0f;
#pragma unroll
    for (int ch = 0; ch < kChunks; ++ch) {
      const int col = (ch * threads + t) * 8;
      if (col < cols) {
        float g[8], xhat[8], d[8];
        in[ch].get(a.gamma, col, rstd, g, xhat);
        in[ch].dy.get(d);
        float(&into)[8] = dgamma[kLate ? 0 : ch];
        Eight<false> k;
        if (kLate) {
          k.load(kept, col);
          k.get(into);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          into[i] = __builtin_fmaf(d[i], xhat[i], into[i]);
          sum = __builtin_fmaf(g[i], xhat[i], sum);
        }
        if (kLate) store8(kept, col, false, into);
      }
    }
    const float c = row_sum<kWaveRow>(sum, lds + turn) * inv;
#pragma unroll
    for (int ch = 0; ch < kChunks; ++ch) {
      const int col = (ch * threads + t) * 8;
      if (col < cols && a.dx) {
        float g[8], xhat[8], d[8] = {};
        if (kLate) {
          in[ch].dy.forget();
          if (kSaved8) asm volatile("" : "+v"(in[ch].codes.x), "+v"(in[ch].codes.y));
          else in[ch].h.forget();
        }
        in[ch].get(a.gamma, col, rstd, g, xhat);
        if (a.dres) {
          if (kLate) in[ch].dres.load(dres, col);
          in[ch].dres.get(d);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] += rstd * (g[i] - xhat[i] * c);
        store8(static_cast<char*>(a.dx) + row * a.lddx * (kSBf16 ? 2 : 4), col, kSBf16, d);
      }
    }
  }
  if (!partials) return;
  float* to = partials + static_cast<int64_t>(blockIdx.x) * a.cols;
  if (kWaveRow) {
#pragma unroll
    for (int ch = 0; ch < kChunks; ++ch) {
      const int col = (ch * threads + t) * 8;
      if (col < cols) store8(lds + wave * cols, col, false, dgamma[kLate ? 0 : ch]);
    }
    __syncthreads();
    for (int col = threadIdx.x; col < cols; col += 256) {
      const float s = (lds[col] + lds[cols + col]) + (lds[2 * cols + col] + lds[3 * cols + col]);
      to[col] = add ? to[col] + s : s;
    }
  } else {
#pragma unroll
    for (int ch = 0; ch < kChunks; ++ch) {
      const int col = (ch * threads + t) * 8;
      if (col < cols) {
        float(&sums)[8] = dgamma[kLate ? 0 : ch];
        if (kLate) {
          Eight<false> k;
          k.load(kept, col);
          k.get(sums);
        }
        if (add) {
#pragma unroll
          for (int i = 0; i < 8; ++i) sums[i] += to[col + i];
        }
        store8(to, col, false, sums);
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

constexpr int kMostParts = 512;
int backward_parts(int64_t rows, int64_t cols) {
  const int64_t groups = row_shape(cols).wave ? (rows + 3) / 4 : rows;
  return static_cast<int>(groups < kMostParts ? groups : kMostParts);
}

template <bool kDyBf16, bool kSBf16, bool kSaved8>
hipError_t backward_of(const RmsNormBackward& a, int parts, float* partials, bool add, hipStream_t s) {
  const RowShape p = row_shape(a.cols);
  const unsigned lds = p.wave ? static_cast<unsigned>(a.cols) * 16 : 128 + (p.chunks == 4 ? static_cast<unsigned>(a.cols) * 4 : 0);
  if (p.chunks == 4) {
    static PerDeviceOnce once;
    const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void*>(&rmsnorm_backward_kernel<kDyBf16, kSBf16, kSaved8, 4, false>), 128 + 32768 * 4, once);
    if (e != hipSuccess) return e;
  }
#define NVFP4_NORM(CH, WAVE) \
  hipLaunchKernelGGL((rmsnorm_backward_kernel<kDyBf16, kSBf16, kSaved8, CH, WAVE>), dim3(parts), dim3(WAVE ? 256 : p.threads), lds, s, a, partials, add)
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

}  // namespace

hipError_t launch_rmsnorm_forward(const RmsNormForward& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  if (a.x_bf16) return a.h_bf16 ? forward_of<true, true>(a, s) : forward_of<true, false>(a, s);
  return a.h_bf16 ? forward_of<false, true>(a, s) : forward_of<false, false>(a, s);
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
    const int kind = (a.dy_bf16 ? 4 : 0) | (a.s_bf16 ? 2 : 0) | (a.codes ? 1 : 0);
    hipError_t e;
    switch (kind) {
      case 0: e = backward_of<false, false, false>(a, parts, partials, add, s); break;
      case 1: e = backward_of<false, false, true>(a, parts, partials, add, s); break;
      case 2: e = backward_of<false, true, false>(a, parts, partials, add, s); break;
      case 3: e = backward_of<false, true, true>(a, parts, partials, add, s); break;
      case 4: e = backward_of<true, false, false>(a, parts, partials, add, s); break;
      case 5: e = backward_of<true, false, true>(a, parts, partials, add, s); break;
      case 6: e = backward_of<true, true, false>(a, parts, partials, add, s); break;
      default: e = backward_of<true, true, true>(a, parts, partials, add, s); break;
    }
    if (e != hipSuccess) return e;
  }
  if (!a.dgamma || parts == 1) return hipSuccess;
  return launch_colsum(partials, parts, a.cols, a.dgamma, a.accumulate, s);
}

}  // namespace nvfp4
