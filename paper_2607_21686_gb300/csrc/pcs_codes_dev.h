// pcs_codes_dev.h -- what the codes of an 8-bit cache stand for, on the device.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "pcs_attend.h"

namespace pcs {

// 2^(b - 127); NaN for b = 255.  (b = 0 is the float of the largest bit below the
// normal ones, 255 would be infinity: both take that bit.)
__device__ __forceinline__ float scale_value(uint32_t b) {
  return __uint_as_float(b << 23 | (b == 0 || b == 255 ? 0x00400000u : 0u));
}

// Two codes (a 16-bit half each, as they lie in memory) to a pair of float16, exactly.
__device__ __forceinline__ uint32_t pair_e4m3(uint16_t x) {
  uint32_t y;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(y) : "h"(x));
  return y;
}
// Whole numbers: a code with its sign turned is c + 128, and 0x6400 with that in its
// low byte is 1024 + c + 128.  `sel` picks the two bytes of x.
__device__ __forceinline__ uint32_t pair_i8(uint32_t x, uint32_t sel) {
  const uint32_t y = __byte_perm(x, 0x64646464u, sel);
  const __half2 k = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));  // 1152
  const __half2 z = __hsub2(*reinterpret_cast<const __half2*>(&y), k);
  return *reinterpret_cast<const uint32_t*>(&z);
}
// Four codes of a word to two pairs of float16.
template <int CODES>
__device__ __forceinline__ void four_halves(uint32_t x, uint32_t& lo, uint32_t& hi) {
  if constexpr (CODES == kCodesE4M3) {
    lo = pair_e4m3(static_cast<uint16_t>(x));
    hi = pair_e4m3(static_cast<uint16_t>(x >> 16));
  } else {
    x ^= 0x80808080u;
    lo = pair_i8(x, 0x4140);
    hi = pair_i8(x, 0x4342);
  }
}
template <int CODES>
__device__ __forceinline__ void four_values(uint32_t x, float* y) {
  uint32_t lo, hi;
  four_halves<CODES>(x, lo, hi);
  const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo));
  const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  y[0] = a.x, y[1] = a.y, y[2] = b.x, y[3] = b.y;
}

// Rounded to T; float16 ends at its largest number (a head whose largest element is
// near it may stand for 65536, the next code).  NaN stays.
template <typename T>
__device__ __forceinline__ T rounded(float x);
template <>
__device__ __forceinline__ float rounded<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 rounded<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half rounded<__half>(float x) {
  return __float2half_rn(x > 65504.0f ? 65504.0f : x < -65504.0f ? -65504.0f : x);
}

}  // namespace pcs
