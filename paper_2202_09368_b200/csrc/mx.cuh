// The 4-bit microscaled format on the device: a block's shared power of two and the codes of its values.
#pragma once
#include <stdint.h>

namespace ecmoe {

namespace {

constexpr unsigned kMxNan = 255;

// The block's scale byte s (it stands for 2^(s - 127)) from the bits of its largest magnitude: the largest lies in [4, 8) times the
// scale, unless it is below 2^-125 (s = 0).  An infinity or a NaN, whose bits are above every finite value's, makes it NaN.
__device__ __forceinline__ unsigned mx_scale_of(unsigned amax_bits) {
  const unsigned e = amax_bits >> 23;
  return e == 255 ? kMxNan : e > 2 ? e - 2 : 0;
}
// 2^(127 - s), by which the block's values are multiplied: exact, also where a value is subnormal (2^127 is its largest).  A NaN block's
// values become zeros of either sign or NaN here and mx_codes is not asked for them.
__device__ __forceinline__ float mx_inverse(unsigned s) { return __uint_as_float((254u - s) << 23); }
// The same straight from the largest magnitude's bits: 256 - e in the exponent's place, at most 254
__device__ __forceinline__ float mx_inverse_of(unsigned amax_bits) { return __uint_as_float(min(0x80000000u - (amax_bits & 0x7F800000u), 0x7F000000u)); }
// 2^(s - 127); s = 0 is subnormal
__device__ __forceinline__ float mx_scale_value(unsigned s) {
  return __uint_as_float(s == kMxNan ? 0x7fffffffu : s == 0 ? 0x00400000u : s << 23);
}

// Codes of eight scaled values, the first in the lowest four bits: to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to the even
// code), 6 beyond, the sign in the top bit.
__device__ __forceinline__ unsigned mx_codes8(const float* y) {
  unsigned r;
  asm("{\n .reg .b8 a, b, c, d;\n"
      " cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
      " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n"
      " mov.b32 %0, {a, b, c, d};\n}\n"
      : "=r"(r) : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
  return r;
}

}  // namespace

}  // namespace ecmoe
