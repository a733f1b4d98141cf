// What the kernels around the linear layers share: eight columns of a row in FP32 or bf16, the 8-bit checkpoint format, and the activation
// functions with their derivatives.  Device code only.
#pragma once

#include "nvfp4_device.h"

namespace nvfp4 {

// ---------------------------------------------------------------- eight consecutive columns of a row, 16-byte pieces
template <bool kBf16>
struct Eight;
template <>
struct Eight<true> {
  uint4 w;
  __device__ __forceinline__ void load(const void* row, int64_t col) { w = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(row) + col); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = bf16_lo(w.x), v[1] = bf16_hi(w.x), v[2] = bf16_lo(w.y), v[3] = bf16_hi(w.y);
    v[4] = bf16_lo(w.z), v[5] = bf16_hi(w.z), v[6] = bf16_lo(w.w), v[7] = bf16_hi(w.w);
  }
  // No instruction; the compiler forgets what it has made of the words, so that it does not keep that in registers.
  __device__ __forceinline__ void forget() { asm volatile("" : "+v"(w.x), "+v"(w.y), "+v"(w.z), "+v"(w.w)); }
};
template <>
struct Eight<false> {
  float4v a, b;
  __device__ __forceinline__ void load(const void* row, int64_t col) {
    const float4v* p = reinterpret_cast<const float4v*>(static_cast<const float*>(row) + col);
    a = p[0], b = p[1];
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
  }
  __device__ __forceinline__ void forget() { asm volatile("" : "+v"(a), "+v"(b)); }
};
__device__ __forceinline__ void store8(void* row, int64_t col, bool bf16, const float (&v)[8]) {
  if (bf16) {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(row) + col) =
        make_uint4(f32x2_to_bf16(v[0], v[1]), f32x2_to_bf16(v[2], v[3]), f32x2_to_bf16(v[4], v[5]), f32x2_to_bf16(v[6], v[7]));
  } else {
    float4v* p = reinterpret_cast<float4v*>(static_cast<float*>(row) + col);
    p[0] = float4v{v[0], v[1], v[2], v[3]};
    p[1] = float4v{v[4], v[5], v[6], v[7]};
  }
}

// ---------------------------------------------------------------- 8-bit checkpoints
// Blocks of 16 columns of a row: E4M3 codes and one UE8M0 byte e + 127 for 2^e, e the smallest with amax <= 448 * 2^e.  One pass: no amax of the
// tensor is needed, and a power of two divides exactly.  A block that holds an infinity or a NaN has byte 255, which decodes to NaN.

// The byte, from the block's largest magnitude as bits (compared as integers, so that a NaN is the largest).  448 is 1.75 * 2^8.
__device__ __forceinline__ uint32_t checkpoint_scale(uint32_t amax_bits) {
  const uint32_t up = max((amax_bits + 0x1FFFFFu) >> 23, 8u) - 8u;
  return amax_bits >= 0x7F800000u ? 255u : up;
}
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
template <int kN>
__device__ __forceinline__ uint32_t max_magnitude(const float (&v)[kN]) {
  uint32_t m = magnitude(v[0]);
#pragma unroll
  for (int i = 1; i < kN; ++i) m = max(m, magnitude(v[i]));
  return m;
}

// Four values / 2^(byte - 127) -> four codes, round to nearest even.  (The conversion looks at the scale operand's exponent field alone.)
typedef short short2v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t checkpoint_codes4(float v0, float v1, float v2, float v3, uint32_t byte) {
  const float s = __uint_as_float(byte << 23);
  union {
    short2v h;
    uint32_t u;
  } w;
  w.u = 0u;
  w.h = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w.h, v0, v1, s, false);
  w.h = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w.h, v2, v3, s, true);
  return w.u;
}

// Four codes -> values; byte 255 gives NaN.
__device__ __forceinline__ void checkpoint_values4(uint32_t codes, uint32_t byte, float* v) {
  const float s = byte == 255u ? __uint_as_float(0x7FC00000u) : ue8m0_decode(byte);
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(codes), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(codes), true);
  v[0] = lo[0] * s, v[1] = lo[1] * s, v[2] = hi[0] * s, v[3] = hi[1] * s;
}

// ---------------------------------------------------------------- activations
// SiLU and GELU (in its tanh form) are both z s(z (c1 + c3 z^2)), s the logistic function: c1 = 1, c3 = 0, and c1 = 2 sqrt(2 / pi), c3 = 0.044715 c1.
// Numbers of include/nvfp4.h's NVFP4_ACT_*.
enum { kActNone = 0, kActRelu2 = 1, kActGelu = 2, kActSilu = 3 };

// The argument p = z (c1 + c3 z^2) times log2(e) / 2: with w = 2^-|that|, q = w^2 = exp(-|p|), and s = 1 / (1 + q), or q / (1 + q) below zero.  (A square, because the
// exponential instruction has no subnormal results and a product has: nothing is flushed to zero before it is below the smallest number.)
// kOfSum: z may be infinite, where SiLU's p, 0 * z * z * z, is NaN: the clamp takes w = 0 then (a modifier of the exponential, no instruction; w is in [0, 1] without it).  z's own
// NaN reaches the result through z s.  Without it z comes from a checkpoint, which has no infinities, and its NaN stays in q and r.
template <bool kOfSum>
struct Logistic {
  float z, q, r;   // r = 1 / (1 + q)
  __device__ __forceinline__ Logistic(float z_, float c1, float c3) : z(z_) {
    const float p = z * __builtin_fmaf(c3 * z, z, c1);
    const float w = __builtin_amdgcn_exp2f(-__builtin_fabsf(p)), in = kOfSum ? __builtin_amdgcn_fmed3f(w, 0.0f, 1.0f) : w;
    q = in * in;
    r = __builtin_amdgcn_rcpf(1.0f + q);
  }
  __device__ __forceinline__ float s() const { return z < 0.0f ? q * r : r; }   // (p has z's sign)
};
constexpr float kHalfLog2E = 0.72134752044448170f;
__device__ __forceinline__ float logistic_c1(int act) { return act == kActSilu ? kHalfLog2E : 1.5957691216057308f * kHalfLog2E; }
__device__ __forceinline__ float logistic_c3(int act) { return act == kActSilu ? 0.0f : 0.07135481282988394f * kHalfLog2E; }

template <int kN>
__device__ __forceinline__ void activate(float (&v)[kN], int act) {
  if (act == kActRelu2) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const float r = v[i] < 0.0f ? 0.0f : v[i];   // (a NaN stays one)
      v[i] = r * r;
    }
  } else if (act != kActNone) {
    const float c1 = logistic_c1(act), c3 = logistic_c3(act);
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] *= Logistic<true>(v[i], c1, c3).s();
  }
}

// v <- derivative at v: (z s(p))' = s + z s (1 - s) p'.
template <int kN>
__device__ __forceinline__ void activation_slope(float (&v)[kN], int act) {
  if (act == kActRelu2) {
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = v[i] < 0.0f ? 0.0f : 2.0f * v[i];
  } else if (act == kActNone) {
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = 1.0f;
  } else {
    const float c1 = logistic_c1(act), c3 = logistic_c3(act), d1 = c1 / kHalfLog2E, d3 = 3.0f * c3 / kHalfLog2E;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const float z = v[i];
      const Logistic<false> l(z, c1, c3);
      const float qr = l.q * l.r, t = qr * l.r;   // s (1 - s)
      v[i] = (z < 0.0f ? qr : l.r) + (t > 0.0f ? z * t * __builtin_fmaf(d3 * z, z, d1) : 0.0f);   // (far out t is 0 and the polynomial infinite)
    }
  }
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

}  // namespace nvfp4
