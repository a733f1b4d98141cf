// The norm over all gradients of a model, and clipping.
//   sumsq = sum over all tensors of g^2 (binary64);  norm = sqrt(sumsq);  out = g * (norm > max_norm ? max_norm / norm : 1)
// Squares and sums are binary64: a square of an FP32 number neither overflows nor vanishes there, and the multiply-add costs no more than in FP32.
// One launch for all tensors, whatever their number: a unit of work is a piece of one tensor, and a table on the device says which.  Each unit leaves its
// sum, a second launch adds those in a fixed order.  Memory bounds both passes: 210 million FP32 values 169 us (5.0 TB/s; by
// itself, without a clipping pass in front of it, 151) and 273 (6.2 TB/s).
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
__device__ __forceinline__ Unit unit_of(const GradTensor* tensors, const int32_t* unit_tensor, uint32_t unit) {
  const GradTensor& t = tensors[unit_tensor[unit]];
  const uint32_t u = unit - static_cast<uint32_t>(t.first_unit);
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

// Pieces of 16 bytes of the wider type (four FP32 or eight bf16 values), wherever they start: an element's alignment is enough for a 16-byte access to global memory, and the
// address space is said since the pointers come out of a table.
#define NVFP4_GLOBAL __attribute__((address_space(1)))
typedef float float4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t uint4u __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t uint2u __attribute__((ext_vector_type(2), aligned(2)));
template <int kN>
struct Words {
  using type = uint4u;
};
template <>
struct Words<4> {
  using type = uint2u;
};

template <bool kBf16, int kN>
__device__ __forceinline__ void load_piece(const char* at, float (&v)[kN]) {
  if constexpr (kBf16) {
    const auto w = *reinterpret_cast<const NVFP4_GLOBAL typename Words<kN>::type*>(reinterpret_cast<uintptr_t>(at));
#pragma unroll
    for (int i = 0; i < kN / 2; ++i) v[2 * i] = bf16_lo(w[i]), v[2 * i + 1] = bf16_hi(w[i]);
  } else {
    const float4u w = *reinterpret_cast<const NVFP4_GLOBAL float4u*>(reinterpret_cast<uintptr_t>(at));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = w[i];
  }
}
template <bool kBf16, int kN>
__device__ __forceinline__ void store_piece(char* at, const float (&v)[kN]) {
  if constexpr (kBf16) {
    typename Words<kN>::type w;
#pragma unroll
    for (int i = 0; i < kN / 2; ++i) w[i] = f32x2_to_bf16(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<NVFP4_GLOBAL typename Words<kN>::type*>(reinterpret_cast<uintptr_t>(at)) = w;
  } else {
    *reinterpret_cast<NVFP4_GLOBAL float4u*>(reinterpret_cast<uintptr_t>(at)) = float4u{v[0], v[1], v[2], v[3]};
  }
}
template <bool kBf16>
__device__ __forceinline__ float load1(const char* at) {
  const uintptr_t p = reinterpret_cast<uintptr_t>(at);
  return kBf16 ? __uint_as_float(static_cast<uint32_t>(*reinterpret_cast<const NVFP4_GLOBAL uint16_t*>(p)) << 16) : *reinterpret_cast<const NVFP4_GLOBAL float*>(p);
}
template <bool kBf16>
__device__ __forceinline__ void store1(char* at, float v) {
  const uintptr_t p = reinterpret_cast<uintptr_t>(at);
  if (kBf16) *reinterpret_cast<NVFP4_GLOBAL uint16_t*>(p) = static_cast<uint16_t>(f32_to_bf16(v));
  else *reinterpret_cast<NVFP4_GLOBAL float*>(p) = v;
}

// wide(row, column) for pieces of kN columns and single(row, column) for what a row has behind them, over a unit by `step` threads of which this one is number `t`.
template <int kN, int kUnroll, typename Wide, typename Single>
__device__ __forceinline__ void for_unit(const Unit& n, uint32_t t, uint32_t step, Wide wide, Single single) {
  const uint32_t pieces = static_cast<uint32_t>(n.cols) / kN, rest = static_cast<uint32_t>(n.cols) - pieces * kN;
  if (n.rows == 1) {
#pragma unroll kUnroll
    for (uint32_t i = t; i < pieces; i += step) wide(0, static_cast<int>(i * kN));
  } else if (pieces) {
#pragma unroll kUnroll
    for (uint32_t i = t; i < pieces * static_cast<uint32_t>(n.rows); i += step) wide(static_cast<int>(i / pieces), static_cast<int>(i % pieces * kN));
  }
  if (rest) {
    for (uint32_t i = t; i < rest * static_cast<uint32_t>(n.rows); i += step) single(static_cast<int>(i / rest), static_cast<int>(pieces * kN + i % rest));
  }
}

template <bool kBf16>
__device__ __forceinline__ double squares(const Unit& n) {
  constexpr int kN = kBf16 ? 8 : 4, kSize = kBf16 ? 2 : 4;
  double s[2] = {};
  for_unit<kN, 4>(
      n, threadIdx.x, 256,
      [&](int row, int col) {
        float v[kN];
        load_piece<kBf16>(n.data + row * n.ld + static_cast<int64_t>(col) * kSize, v);
#pragma unroll
        for (int i = 0; i < kN; ++i) s[i & 1] = __builtin_fma(static_cast<double>(v[i]), static_cast<double>(v[i]), s[i & 1]);
      },
      [&](int row, int col) {
        const double v = load1<kBf16>(n.data + row * n.ld + static_cast<int64_t>(col) * kSize);
        s[0] = __builtin_fma(v, v, s[0]);
      });
  return s[0] + s[1];
}

__global__ __launch_bounds__(256) void grad_sumsq_kernel(const GradTensor* __restrict__ tensors, const int32_t* __restrict__ unit_tensor, double* __restrict__ partials) {
  __shared__ double waves[4];
  const Unit n = unit_of(tensors, unit_tensor, blockIdx.x);
  const double s = wave_sum64(n.flags & kGradBf16 ? squares<true>(n) : squares<false>(n));
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) partials[blockIdx.x] = (waves[0] + waves[1]) + (waves[2] + waves[3]);
}

__global__ __launch_bounds__(1024) void grad_fold_kernel(const double* __restrict__ partials, int64_t units, double* __restrict__ sumsq) {
  __shared__ double waves[16];
  double s = 0.0;
#pragma unroll 8
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
__device__ __forceinline__ void scaled(const Unit& n, uint32_t t, uint32_t step, float by, int up) {
  constexpr int kN = kBf16 && kOutBf16 ? 8 : 4, kSize = kBf16 ? 2 : 4, kOutSize = kOutBf16 ? 2 : 4;
  for_unit<kN, 4>(
      n, t, step,
      [&](int row, int col) {
        float v[kN];
        load_piece<kBf16>(n.data + row * n.ld + static_cast<int64_t>(col) * kSize, v);
#pragma unroll
        for (int i = 0; i < kN; ++i) v[i] = __builtin_ldexpf(v[i] * by, up);
        store_piece<kOutBf16>(n.out + row * n.ld_out + static_cast<int64_t>(col) * kOutSize, v);
      },
      [&](int row, int col) {
        const float v = __builtin_ldexpf(load1<kBf16>(n.data + row * n.ld + static_cast<int64_t>(col) * kSize) * by, up);
        store1<kOutBf16>(n.out + row * n.ld_out + static_cast<int64_t>(col) * kOutSize, v);
      });
}

// The factor from the sum of squares, in every workgroup.  1 for a norm that is not finite, and then, as for any factor of 1, what stays in its place is not touched.
// `splits` workgroups to a unit, so that each has 4096 elements: short waves, neighbours on one XCD.  (A plain copy of 2.7 GB is fastest with 16 bytes to a thread, 6.3 TB/s against 5.7 with
// four times that and 5.4 in a loop; but here three loads in turn lead to the data.  us for norm and clipping of 210 million FP32 values / 30 million bf16 with 1024, 2048, 4096, 8192 elements
// to a workgroup: 474 / 51, 437 / 36, 444 / 31, 461 / 31.)
constexpr int64_t kClipElements = 4096;
__global__ __launch_bounds__(256) void grad_clip_kernel(const GradTensor* __restrict__ tensors, const int32_t* __restrict__ unit_tensor, int64_t units, uint32_t splits,
                                                        const double* __restrict__ sumsq, float max_norm, float* __restrict__ norm) {
  const double total = __builtin_sqrt(*sumsq);
  const bool clips = total > static_cast<double>(max_norm) && total < __builtin_huge_val();
  // A factor below FP32's normal numbers (a norm beyond 2^126 times the bound) would have too few bits, or none: it is by 2^up, by in [0.5, 1).
  const double factor = clips ? static_cast<double>(max_norm) / total : 1.0;
  const int up = factor < 0x1p-126 ? __builtin_amdgcn_frexp_exp(factor) : 0;
  const float by = static_cast<float>(__builtin_ldexp(factor, -up));
  if (blockIdx.x == 0 && threadIdx.x == 0 && norm) *norm = static_cast<float>(total);
  if (units == 0) return;
  const uint32_t w = xcd_neighbours(blockIdx.x, gridDim.x), t = w % splits * 256 + threadIdx.x, step = splits * 256;
  const Unit n = unit_of(tensors, unit_tensor, w / splits);
  if (by == 1.0f && up == 0 && n.data == n.out && ((n.flags & kGradBf16) != 0) == ((n.flags & kGradOutBf16) != 0)) return;
  if (n.flags & kGradBf16) {
    if (n.flags & kGradOutBf16) scaled<true, true>(n, t, step, by, up); else scaled<true, false>(n, t, step, by, up);
  } else {
    if (n.flags & kGradOutBf16) scaled<false, true>(n, t, step, by, up); else scaled<false, false>(n, t, step, by, up);
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

hipError_t launch_grad_clip(const GradTensor* tensors, const int32_t* unit_tensor, int64_t units, int64_t unit_elements, const double* sumsq, float max_norm,
                            float* norm, hipStream_t s) {
  const int64_t most = std::max<int64_t>(1, (1 << 24) / std::max<int64_t>(units, 1) - 1), splits = std::min((unit_elements + kClipElements - 1) / kClipElements, most);   // (a launch holds 2^32 threads)
  hipLaunchKernelGGL(grad_clip_kernel, dim3(static_cast<unsigned>(std::max<int64_t>(units * splits, 1))), dim3(256), 0, s, tensors, unit_tensor, units,
                     static_cast<uint32_t>(splits), sumsq, max_norm, norm);
  return hipGetLastError();
}

}  // namespace nvfp4
