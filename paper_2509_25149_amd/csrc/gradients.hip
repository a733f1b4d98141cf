// The norm over all gradients of a model, and clipping.
//   sumsq = sum over all tensors of g^2 (binary64);  norm = sqrt(sumsq);  out = g * (norm > max_norm ? max_norm / norm : 1)
// Squares and sums are binary64: a square of an FP32 number neither overflows nor vanishes there, and the multiply-add costs no more than in FP32.
// One launch for all tensors, whatever their number: a unit of work is a piece of one tensor, and a table on the device says which.  Each unit leaves its
// sum, a second launch adds those in a fixed order.  Memory bounds both passes.
#include <algorithm>

#include "nvfp4_internal.h"
#include "checkpoint8.h"

namespace nvfp4 {

namespace {

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

// A unit: rows [0, rows) of `cols` columns from data and out.
struct Unit {
  const char* data;
  char* out;
  int64_t ld, ld_out;   // bytes
  int rows, cols, flags;
};
__device__ __forceinline__ Unit unit_of(const GradTensor* tensors, const int32_t* unit_tensor) {
  const GradTensor& t = tensors[unit_tensor[blockIdx.x]];
  const uint32_t u = blockIdx.x - static_cast<uint32_t>(t.first_unit);
  const uint32_t across = static_cast<uint32_t>((t.cols + t.unit_cols - 1) / t.unit_cols);
  const int64_t row = static_cast<int64_t>(u / across) * t.unit_rows, col = static_cast<int64_t>(u % across) * t.unit_cols;
  const int in = t.flags & kGradBf16 ? 2 : 4, to = t.flags & kGradOutBf16 ? 2 : 4;
  Unit n;
  n.ld = t.ld * in, n.ld_out = t.ld_out * to;
  n.data = static_cast<const char*>(t.data) + row * n.ld + col * in;
  n.out = static_cast<char*>(t.out) + row * n.ld_out + col * to;
  n.rows = static_cast<int>(min(static_cast<int64_t>(t.unit_rows), t.rows - row));
  n.cols = static_cast<int>(min(static_cast<int64_t>(t.unit_cols), t.cols - col));
  n.flags = t.flags;
  return n;
}

template <bool kBf16>
__device__ __forceinline__ float load1(const char* row, int col) {
  return kBf16 ? __uint_as_float(static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(row)[col]) << 16) : reinterpret_cast<const float*>(row)[col];
}

// wide(row, group of eight columns) and single(row, column) over a unit by its 256 threads.
template <typename Wide, typename Single>
__device__ __forceinline__ void for_unit(const Unit& n, Wide wide, Single single) {
  const uint32_t groups = n.flags & kGradWide ? static_cast<uint32_t>(n.cols) >> 3 : 0u, rest = static_cast<uint32_t>(n.cols) - groups * 8;
  if (groups) {
    if (n.rows == 1) {
#pragma unroll 4
      for (uint32_t i = threadIdx.x; i < groups; i += 256) wide(0, static_cast<int>(i));
    } else {
#pragma unroll 4
      for (uint32_t i = threadIdx.x; i < groups * static_cast<uint32_t>(n.rows); i += 256) wide(static_cast<int>(i / groups), static_cast<int>(i % groups));
    }
  }
  if (rest) {
#pragma unroll 4
    for (uint32_t i = threadIdx.x; i < rest * static_cast<uint32_t>(n.rows); i += 256) single(static_cast<int>(i / rest), static_cast<int>(groups * 8 + i % rest));
  }
}

template <bool kBf16>
__device__ __forceinline__ double squares(const Unit& n) {
  double s[2] = {};
  for_unit(
      n,
      [&](int row, int g) {
        Eight<kBf16> x;
        float v[8];
        x.load(n.data + row * n.ld, static_cast<int64_t>(g) * 8);
        x.get(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i & 1] = __builtin_fma(static_cast<double>(v[i]), static_cast<double>(v[i]), s[i & 1]);
      },
      [&](int row, int col) {
        const double v = load1<kBf16>(n.data + row * n.ld, col);
        s[0] = __builtin_fma(v, v, s[0]);
      });
  return s[0] + s[1];
}

__global__ __launch_bounds__(256) void grad_sumsq_kernel(const GradTensor* __restrict__ tensors, const int32_t* __restrict__ unit_tensor, double* __restrict__ partials) {
  __shared__ double waves[4];
  const Unit n = unit_of(tensors, unit_tensor);
  const double s = wave_sum64(n.flags & kGradBf16 ? squares<true>(n) : squares<false>(n));
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) partials[blockIdx.x] = (waves[0] + waves[1]) + (waves[2] + waves[3]);
}

__global__ __launch_bounds__(1024) void grad_fold_kernel(const double* __restrict__ partials, int64_t units, double* __restrict__ sumsq) {
  __shared__ double waves[16];
  double s = 0.0;
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < units; i += 1024) s += partials[i];
  s = wave_sum64(s);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 16; ++w) s += waves[w];
    *sumsq = s;
  }
}

template <bool kBf16, bool kOutBf16>
__device__ __forceinline__ void scaled(const Unit& n, float by) {
  for_unit(
      n,
      [&](int row, int g) {
        Eight<kBf16> x;
        float v[8];
        x.load(n.data + row * n.ld, static_cast<int64_t>(g) * 8);
        x.get(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= by;
        store8(n.out + row * n.ld_out, static_cast<int64_t>(g) * 8, kOutBf16, v);
      },
      [&](int row, int col) {
        const float v = load1<kBf16>(n.data + row * n.ld, col) * by;
        char* to = n.out + row * n.ld_out;
        if (kOutBf16) reinterpret_cast<uint16_t*>(to)[col] = static_cast<uint16_t>(f32_to_bf16(v));
        else reinterpret_cast<float*>(to)[col] = v;
      });
}

// The factor from the sum of squares, in every workgroup.  1 for a norm that is not finite, and then, as for any factor of 1, what stays in its place is not touched.
__global__ __launch_bounds__(256) void grad_clip_kernel(const GradTensor* __restrict__ tensors, const int32_t* __restrict__ unit_tensor, int64_t units,
                                                        const double* __restrict__ sumsq, float max_norm, float* __restrict__ norm) {
  const double total = __builtin_sqrt(*sumsq);
  const bool clips = total > static_cast<double>(max_norm) && total < __builtin_huge_val();
  const float by = clips ? static_cast<float>(static_cast<double>(max_norm) / total) : 1.0f;
  if (blockIdx.x == 0 && threadIdx.x == 0 && norm) *norm = static_cast<float>(total);
  if (units == 0) return;
  const Unit n = unit_of(tensors, unit_tensor);
  if (by == 1.0f && n.data == n.out && ((n.flags & kGradBf16) != 0) == ((n.flags & kGradOutBf16) != 0)) return;
  if (n.flags & kGradBf16) {
    if (n.flags & kGradOutBf16) scaled<true, true>(n, by); else scaled<true, false>(n, by);
  } else {
    if (n.flags & kGradOutBf16) scaled<false, true>(n, by); else scaled<false, false>(n, by);
  }
}

}  // namespace

hipError_t launch_grad_sumsq(const GradTensor* tensors, const int32_t* unit_tensor, int64_t units, double* sumsq, double* partials, hipStream_t s) {
  if (units) {
    hipLaunchKernelGGL(grad_sumsq_kernel, dim3(static_cast<unsigned>(units)), dim3(256), 0, s, tensors, unit_tensor, partials);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(grad_fold_kernel, dim3(1), dim3(1024), 0, s, partials, units, sumsq);
  return hipGetLastError();
}

hipError_t launch_grad_clip(const GradTensor* tensors, const int32_t* unit_tensor, int64_t units, const double* sumsq, float max_norm, float* norm, hipStream_t s) {
  hipLaunchKernelGGL(grad_clip_kernel, dim3(static_cast<unsigned>(std::max<int64_t>(units, 1))), dim3(256), 0, s, tensors, unit_tensor, units, sumsq, max_norm, norm);
  return hipGetLastError();
}

}  // namespace nvfp4
