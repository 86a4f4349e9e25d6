// The 8-bit form of kept activations: 32 consecutive values of a row share a power-of-two scale
// 2^(s - 127), the smallest with which the largest of them is at most 448, E4M3's largest value; each
// value is the E4M3 code nearest to v / scale (ties to even). Powers of two make the division and the
// product exact, so a code is off by its own rounding only: 2^-4 of a value down to 2^-14 of the
// block's largest, an absolute step below. A block that holds an infinity or a NaN becomes all NaN
// (s = 255), as its gradients would; values from 1.9375 * 2^127 on round to 2^128, an infinity. Scales below 2^-126 are not used (s >= 1).
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"

namespace ckpt {

constexpr int kBlock = 32;  // values that share a scale

// Scale byte of a block from the largest of its values' bits without sign (NaN > infinity > finite).
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits) {
  const int e = int(amax_bits >> 23);                       // 448 = 1.75 * 2^8
  const int s = e - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e == 255 ? 255u : uint32_t(max(s, 1));
}
__device__ __forceinline__ float scale_inverse(uint32_t s) { return __uint_as_float((254u - s) << 23); }
__device__ __forceinline__ float scale_value(uint32_t s) { return __uint_as_float(s << 23); }

// Four values times `inv` as codes, the first in the lowest byte.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a * inv, b * inv), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c * inv, d * inv), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}
constexpr uint32_t kNanCodes = 0x7f7f7f7fu;

// The values of four codes times `scale`.
__device__ __forceinline__ void values4(uint32_t codes, float scale, float *v) {
  const __half2_raw lo = __nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t(codes & 0xffffu), __NV_E4M3);
  const __half2_raw hi = __nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t(codes >> 16), __NV_E4M3);
  const float2 a = __half22float2(__half2(lo)), b = __half22float2(__half2(hi));
  v[0] = a.x * scale;
  v[1] = a.y * scale;
  v[2] = b.x * scale;
  v[3] = b.y * scale;
}

// Kept [A|B] (rows x 2F) in the 32-row tiles of the GEMM epilogues, whose lanes own a row each: codes in
// runs of 16 columns (a lane's 16 bytes, a warp's 512), scales in runs of one block (a warp's 32 bytes).
__device__ __forceinline__ size_t ab_code_index(size_t row, int col, int F) {
  return ((row >> 5) * size_t(2 * F / 16) + size_t(col >> 4)) * 512 + (row & 31) * 16;
}
__device__ __forceinline__ size_t ab_scale_index(size_t row, int col, int F) {
  return ((row >> 5) * size_t(2 * F / kBlock) + size_t(col / kBlock)) * 32 + (row & 31);
}

}  // namespace ckpt
