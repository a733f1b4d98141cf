// 8-bit checkpoints of activations (format: checkpoint8.h) and what the backward pass does with them:
//   save      codes and scales of a tensor
//   load      act(z) * column factor, FP32 or bf16: an activation's output made again from what went into it, or a normalised row times gamma
//   backward  dz = da act'(z) and the sum of dz over rows (the gradient of the bias in front of the activation)
// All of them read and write every byte once; memory bounds them: 8192 x 20480 bf16, save 91 us, load 88 (5.8 TB/s), activation gradient with the bias's
// 164 for squared ReLU and 175 for GELU (5.2 and 4.9 TB/s; a large copy runs at 5.1).
#include <algorithm>

#include "nvfp4_internal.h"
#include "checkpoint8.h"

namespace nvfp4 {

namespace {

// A workgroup covers 512 columns (eight to a lane) of some rows, its wavefronts taking every fourth row.  (A line of 128 scales belongs to four such strips, and is
// fetched by as many XCDs: 200 MiB instead of 170 for 8192 x 20480.  Four wavefronts side by side on 2048 columns read 170 and take longer: load 90 us instead of
// 88, activation gradient 181 instead of 164.)
constexpr int kStrip = 512;

template <bool kBf16>
__global__ __launch_bounds__(256) void checkpoint_save_kernel(const void* __restrict__ x, int64_t rows, int64_t cols, int64_t ldx, int rows_per_group,
                                                              uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, int strips) {
  const int strip = blockIdx.x % strips, lane = threadIdx.x & 63;
  const int64_t r0 = static_cast<int64_t>(blockIdx.x / strips) * rows_per_group, r1 = min(r0 + rows_per_group, rows);
  const int64_t col = static_cast<int64_t>(strip) * kStrip + lane * 8;
  if (col >= cols) return;
#pragma unroll 2
  for (int64_t row = r0 + (threadIdx.x >> 6); row < r1; row += 4) {
    Eight<kBf16> e;
    e.load(static_cast<const char*>(x) + row * ldx * (kBf16 ? 2 : 4), col);
    float v[8];
    e.get(v);
    uint32_t m = max_magnitude(v);
    m = max(m, lane_xor1(m));
    const uint32_t byte = checkpoint_scale(m);
    *reinterpret_cast<uint2*>(codes + row * cols + col) =
        make_uint2(checkpoint_codes4(v[0], v[1], v[2], v[3], byte), checkpoint_codes4(v[4], v[5], v[6], v[7], byte));
    if ((lane & 1) == 0) scales[row * (cols / 16) + col / 16] = static_cast<uint8_t>(byte);
  }
}

template <bool kBf16>
__global__ __launch_bounds__(256) void checkpoint_load_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t rows, int64_t cols,
                                                              int rows_per_group, int act, const float* __restrict__ col_scale, void* __restrict__ out,
                                                              int64_t ld_out, int strips) {
  const int strip = blockIdx.x % strips, lane = threadIdx.x & 63;
  const int64_t r0 = static_cast<int64_t>(blockIdx.x / strips) * rows_per_group, r1 = min(r0 + rows_per_group, rows);
  // FP32 columns are stored as they lie, four to a lane and half a strip: 16 bytes a lane without gaps (8192 x 20480 176 us; eight to a lane, in two stores with gaps, 238).
  constexpr int kHalves = kBf16 ? 1 : 2, kCols = kBf16 ? 8 : 4;
  const int64_t col = static_cast<int64_t>(strip) * kStrip + lane * kCols;
  float f[kHalves][kCols];
  bool in[kHalves];
#pragma unroll
  for (int h = 0; h < kHalves; ++h) {
    in[h] = col + h * 256 < cols;
#pragma unroll
    for (int i = 0; i < kCols; ++i) f[h][i] = col_scale && in[h] ? col_scale[col + h * 256 + i] : 1.0f;
  }
#pragma unroll 2
  for (int64_t row = r0 + (threadIdx.x >> 6); row < r1; row += 4) {
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      if (!in[h]) continue;
      const int64_t at = row * cols + col + h * 256;
      const uint32_t byte = scales[at / 16];
      float v[kCols];
      checkpoint_values4(*reinterpret_cast<const uint32_t*>(codes + at), byte, v);
      if constexpr (kBf16) checkpoint_values4(*reinterpret_cast<const uint32_t*>(codes + at + 4), byte, v + 4);
      activate(v, act);
#pragma unroll
      for (int i = 0; i < kCols; ++i) v[i] *= f[h][i];
      if constexpr (kBf16) store8(static_cast<uint16_t*>(out) + row * ld_out, col, true, v);
      else *reinterpret_cast<float4v*>(static_cast<float*>(out) + row * ld_out + col + h * 256) = float4v{v[0], v[1], v[2], v[3]};
    }
  }
}

// partials: row blockIdx.x / strips of them gets the group's sums, or null.
template <bool kBf16>
__global__ __launch_bounds__(256) void activation_backward_kernel(ActivationBackward a, int rows_per_group, float* __restrict__ partials, bool add, int strips) {
  __shared__ float sums[4][kStrip];
  const int strip = blockIdx.x % strips, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t group = blockIdx.x / strips, r0 = group * rows_per_group, r1 = min(r0 + rows_per_group, a.rows);
  const int64_t col = static_cast<int64_t>(strip) * kStrip + lane * 8;
  float s[8] = {};
  if (col < a.cols) {
#pragma unroll 2
    for (int64_t row = r0 + wave; row < r1; row += 4) {
      Eight<kBf16> e;
      e.load(static_cast<const char*>(a.da) + row * a.ldda * (kBf16 ? 2 : 4), col);
      float d[8], v[8];
      e.get(d);
      if (a.act != kActNone) {
        const uint2 c = *reinterpret_cast<const uint2*>(a.codes + row * a.cols + col);
        const uint32_t byte = a.scales[row * (a.cols / 16) + col / 16];
        checkpoint_values4(c.x, byte, v);
        checkpoint_values4(c.y, byte, v + 4);
        activation_slope(v, a.act);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] *= v[i];
      }
      if (a.dz) store8(static_cast<char*>(a.dz) + row * a.lddz * (kBf16 ? 2 : 4), col, kBf16, d);
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] += d[i];
    }
  }
  if (!partials) return;
  store8(sums[wave], lane * 8, false, s);
  __syncthreads();
  for (int c = threadIdx.x; c < kStrip; c += 256) {
    const int64_t to = static_cast<int64_t>(strip) * kStrip + c;
    if (to < a.cols) {
      const float v = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
      float* p = partials + group * a.cols + to;
      *p = add ? *p + v : v;
    }
  }
}

int strips_of(int64_t cols) { return static_cast<int>((cols + kStrip - 1) / kStrip); }

// Rows of a workgroup: as few as leave no more than kMostGroups workgroups, four at least, and with sums over rows no more than kMostParts of them to a strip.
// Workgroups start in order, so the shorter they are the closer together the chip reads and writes; the sums' second launch has their number to
// add up.  8192 x 20480, us with 1024 / 4096 / 8192 / 16384 / 32768 workgroups: save bf16 103 / 107 / 101 / 96 / 91, load bf16 107 / 105 / 99 / 93 / 88, activation gradient
// without sums 169 / 167 / 156 / 150 / 146; with sums, 128 / 256 / 512 parts: 170 / 165 / 164, 8192 x 1296 20 / 15.5 / 16.2.
// A few rows are one workgroup's to a strip, whose sums need no second launch (16 x 5120, us on the GPU / called from Python: 5.2 / 5.7, in two launches 5.3 / 8.6; 32 rows 8.0 /
// 7.9 and 5.3 / 8.4).
constexpr int64_t kMostGroups = 32768, kMostParts = 256, kFew = 16;
int rows_of(int64_t rows, int64_t cols, bool sums) {
  if (sums && rows <= kFew) return kFew;
  int64_t groups = std::max<int64_t>(kMostGroups / strips_of(cols), 1);
  if (sums) groups = std::min(groups, kMostParts);
  const int64_t each = (rows + groups - 1) / groups;
  return static_cast<int>(std::max<int64_t>((each + 3) / 4 * 4, 4));
}

}  // namespace

hipError_t launch_checkpoint_save(const void* x, bool bf16, int64_t rows, int64_t cols, int64_t ldx, uint8_t* codes, uint8_t* scales, hipStream_t s) {
  if (rows == 0) return hipSuccess;
  const int strips = strips_of(cols), each = rows_of(rows, cols, false);
  const dim3 grid(static_cast<unsigned>((rows + each - 1) / each * strips));
  if (bf16)
    hipLaunchKernelGGL(checkpoint_save_kernel<true>, grid, dim3(256), 0, s, x, rows, cols, ldx, each, codes, scales, strips);
  else
    hipLaunchKernelGGL(checkpoint_save_kernel<false>, grid, dim3(256), 0, s, x, rows, cols, ldx, each, codes, scales, strips);
  return hipGetLastError();
}

hipError_t launch_checkpoint_load(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, int act, const float* col_scale, void* out, bool bf16,
                                  int64_t ld_out, hipStream_t s) {
  if (rows == 0) return hipSuccess;
  const int strips = strips_of(cols), each = rows_of(rows, cols, false);
  const dim3 grid(static_cast<unsigned>((rows + each - 1) / each * strips));
  if (bf16)
    hipLaunchKernelGGL(checkpoint_load_kernel<true>, grid, dim3(256), 0, s, codes, scales, rows, cols, each, act, col_scale, out, ld_out, strips);
  else
    hipLaunchKernelGGL(checkpoint_load_kernel<false>, grid, dim3(256), 0, s, codes, scales, rows, cols, each, act, col_scale, out, ld_out, strips);
  return hipGetLastError();
}

size_t activation_partial_bytes(int64_t rows, int64_t cols) {
  const int each = rows_of(rows, cols, true);
  const int64_t groups = (rows + each - 1) / each;
  return groups > 1 ? static_cast<size_t>(groups) * static_cast<size_t>(cols) * 4 : 0;
}

hipError_t launch_activation_backward(const ActivationBackward& a, hipStream_t s) {
  const int strips = strips_of(a.cols), each = rows_of(a.rows, a.cols, a.dbias != nullptr);
  const int groups = static_cast<int>((a.rows + each - 1) / each);
  float* partials = a.dbias ? (groups > 1 ? a.partials : a.dbias) : nullptr;   // one group's sums are the result
  if (groups > 0) {
    const bool add = groups == 1 && a.accumulate;
    const dim3 grid(static_cast<unsigned>(groups) * static_cast<unsigned>(strips));
    if (a.bf16)
      hipLaunchKernelGGL(activation_backward_kernel<true>, grid, dim3(256), 0, s, a, each, partials, add, strips);
    else
      hipLaunchKernelGGL(activation_backward_kernel<false>, grid, dim3(256), 0, s, a, each, partials, add, strips);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!a.dbias || groups == 1) return hipSuccess;
  return launch_colsum(partials, groups, a.cols, a.dbias, a.accumulate, s);
}

}  // namespace nvfp4
