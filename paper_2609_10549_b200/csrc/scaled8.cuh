// 8-bit numbers with block scales, on the device: which scale a block gets, and conversions.
//
// A block's scale is the smallest power of two 2^e, e >= -127, with max|x| <= F 2^e, F the format's largest number (E4M3: 448 =
// 1.75 * 2^8, E5M2: 57344 = 1.75 * 2^15), stored as e + 127 (E8M0).  Dividing by a power of two is exact, so an element is rounded
// once, to the nearest number of the format.
#pragma once

#include <cstdint>

#include "internal.h"

namespace compass {

// Formats as the tensor core's instruction descriptor numbers them.
enum Format8 : int { E4M3 = 0, E5M2 = 1 };

// From the bits of max|x| (finite).  max|x| = m 2^k, 1 <= m < 2: e = k - 8 (or 15), and one more where m > 1.75, which is where
// adding 2^21 - 1 to the mantissa carries into the exponent.
template <int kFormat>
__device__ __forceinline__ uint32_t scale_byte_of(uint32_t top) {
  const int e = int((top + 0x1FFFFFu) >> 23) - (kFormat == E4M3 ? 8 : 15);
  return uint32_t(max(e, 0));
}
// 2^-(b - 127): what a block is multiplied by (b <= 247).
__device__ __forceinline__ float inverse_scale(uint32_t b) { return __uint_as_float((254u - b) << 23); }
// 2^(b - 127); 255 is NaN.
__device__ __forceinline__ float scale_value(uint32_t b) {
  return __uint_as_float(b == 0 ? 0x00400000u : b == 255 ? 0x7FC00000u : b << 23);
}

// Four numbers, lowest first, to nearest even.  (Their size fits; NaN stays NaN.)
template <int kFormat>
__device__ __forceinline__ uint32_t pack8x4(float a, float b, float c, float d) {
  uint16_t lo, hi;
  if constexpr (kFormat == E4M3) {
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  } else {
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  }
  return uint32_t(lo) | uint32_t(hi) << 16;
}
// Two numbers (the low 16 bits) in FP32, exactly.
template <int kFormat>
__device__ __forceinline__ float2 unpack8x2(uint32_t w) {
  uint32_t h;
  if constexpr (kFormat == E4M3) asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(uint16_t(w)));
  else asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(h) : "h"(uint16_t(w)));
  float2 f;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(f.x), "=f"(f.y) : "r"(h));
  return f;
}

inline int format_of(int dtype) { return dtype == COMPASS_DTYPE_E4M3 ? E4M3 : dtype == COMPASS_DTYPE_E5M2 ? E5M2 : -1; }
inline int64_t scale_blocks(int64_t n) { return (n + 127) / 128; }

}  // namespace compass
