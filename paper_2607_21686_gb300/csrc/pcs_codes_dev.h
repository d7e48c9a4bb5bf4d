// pcs_codes_dev.h -- what the codes of an 8-bit cache stand for, on the device.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

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

// To float16's largest number (a head whose largest element is near it may stand for
// 65536, the next code); NaN stays.
__device__ __forceinline__ float limited(float x) {
  asm("min.NaN.f32 %0, %0, %1;" : "+f"(x) : "f"(65504.0f));
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(x) : "f"(-65504.0f));
  return x;
}
template <typename T>
__device__ __forceinline__ uint32_t pair_of(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pair_of<__half>(float lo, float hi) {
  const __half2 h = __floats2half2_rn(limited(lo), limited(hi));
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <>
__device__ __forceinline__ uint32_t pair_of<__nv_bfloat16>(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Four codes times their scale to four elements of 16 bits.
template <typename T, int CODES>
__device__ __forceinline__ uint2 four_elements(uint32_t x, float scale) {
  float y[4];
  if constexpr (CODES == kCodesI8) {
    x ^= 0x80808080u;  // 0x4b0000 and a byte u are 2^23 + u
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = (__uint_as_float(__byte_perm(x, 0x4b000000u, 0x7650 + i)) - 8388736.0f) * scale;
  } else {
    four_values<CODES>(x, y);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] *= scale;
  }
  return make_uint2(pair_of<T>(y[0], y[1]), pair_of<T>(y[2], y[3]));
}
// Two halves' operations on words.
__device__ __forceinline__ uint32_t mul_f16(uint32_t x, uint32_t y) {
  const __half2 z = __hmul2(*reinterpret_cast<const __half2*>(&x), *reinterpret_cast<const __half2*>(&y));
  return *reinterpret_cast<const uint32_t*>(&z);
}
__device__ __forceinline__ uint32_t fma_f16(uint32_t x, uint32_t y, uint32_t w) {
  const __half2 z = __hfma2(*reinterpret_cast<const __half2*>(&x), *reinterpret_cast<const __half2*>(&y), *reinterpret_cast<const __half2*>(&w));
  return *reinterpret_cast<const uint32_t*>(&z);
}
// Four codes times a scale that is a normal float16, by its own arithmetic, two at a time;
// less: -1152 times the scale (I8: codes come as 1024 + c + 128).
template <int CODES>
__device__ __forceinline__ void four_scaled(uint32_t x, uint32_t scale, uint32_t less, uint32_t& lo, uint32_t& hi) {
  if constexpr (CODES == kCodesE4M3) {
    lo = mul_f16(pair_e4m3(static_cast<uint16_t>(x)), scale);
    hi = mul_f16(pair_e4m3(static_cast<uint16_t>(x >> 16)), scale);
  } else {
    x ^= 0x80808080u;
    lo = fma_f16(__byte_perm(x, 0x64646464u, 0x4140), scale, less);
    hi = fma_f16(__byte_perm(x, 0x64646464u, 0x4342), scale, less);
  }
}
// Whether a scale is such a one, with nothing near float16's ends; to bfloat16 any is plain.
template <typename T>
__device__ __forceinline__ bool plain_scale(uint32_t b) {
  return !std::is_same<T, __half>::value || (b >= 127 - 14 && b <= 127 + 5);
}
// Sixteen codes times a plain scale, by its byte.  (To bfloat16 by way of floats: two at a time
// in its own arithmetic, codes put in place by their bits, took longer, 346 -> 384 us for
// trees of 60 nodes over contexts of 32 sessions.)
template <typename T, int CODES>
__device__ __forceinline__ void sixteen_plain(const uint4& x, uint32_t b, uint4& lo, uint4& hi) {
  if constexpr (std::is_same<T, __half>::value) {
    const uint32_t scale = (b - 112) * 0x04000400u, less = CODES == kCodesI8 ? mul_f16(scale, 0xe480e480u) : 0;  // -1152
    four_scaled<CODES>(x.x, scale, less, lo.x, lo.y);
    four_scaled<CODES>(x.y, scale, less, lo.z, lo.w);
    four_scaled<CODES>(x.z, scale, less, hi.x, hi.y);
    four_scaled<CODES>(x.w, scale, less, hi.z, hi.w);
  } else {
    const float s = scale_value(b);
    const uint2 a = four_elements<T, CODES>(x.x, s), d = four_elements<T, CODES>(x.y, s);
    const uint2 e = four_elements<T, CODES>(x.z, s), f = four_elements<T, CODES>(x.w, s);
    lo = make_uint4(a.x, a.y, d.x, d.y);
    hi = make_uint4(e.x, e.y, f.x, f.y);
  }
}
// Any scale.
template <typename T, int CODES>
__device__ __forceinline__ void sixteen_elements(const uint4& x, uint32_t b, uint4& lo, uint4& hi) {
  if (plain_scale<T>(b)) {
    sixteen_plain<T, CODES>(x, b, lo, hi);
    return;
  }
  const float s = scale_value(b);
  const uint2 a = four_elements<T, CODES>(x.x, s), d = four_elements<T, CODES>(x.y, s);
  const uint2 e = four_elements<T, CODES>(x.z, s), f = four_elements<T, CODES>(x.w, s);
  lo = make_uint4(a.x, a.y, d.x, d.y);
  hi = make_uint4(e.x, e.y, f.x, f.y);
}

}  // namespace pcs
