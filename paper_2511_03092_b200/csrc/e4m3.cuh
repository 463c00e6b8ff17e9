// Numbers of 8 bits (e4m3: a sign, four bits of exponent, three of mantissa; 448 at most, a NaN, no infinity).
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

namespace snap {

// Two codes (low byte first) as two half-precision numbers, exactly.  65 lanes per clock and SM: registers of four codes come at 22.0 a clock
// (16.5 where a byte permutation goes before), by masks and shifts at 11.0 to 13.2.
__device__ __forceinline__ uint32_t halves_of_codes(uint32_t two) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((unsigned short)two));
  return r;
}
__device__ __forceinline__ float2 floats_of_codes(uint32_t two) {
  const uint32_t h = halves_of_codes(two);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
// Rounded to nearest even; 448 at most in size, NaN stays.
__device__ __forceinline__ uint32_t codes_of_floats(float lo, float hi) {
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

// A number that is to be rounded to a few bits, given as single precision holds it (to nearest) and the sign of what that leaves out: where it leaves
// anything out, the one of the two neighbours whose last bit is set, which lies on no border between codes and on the side where the number is.
__device__ __forceinline__ float to_odd(float x, float rest) {
  const uint32_t b = __float_as_uint(x);
  if (rest == 0.f || x == 0.f || (b & 1u)) return x;
  return __uint_as_float((rest > 0.f) == (x > 0.f) ? b + 1u : b - 1u);
}
// x * y of which few bits are kept, neither it nor its last bit too small for single precision
__device__ __forceinline__ float product_to_odd(float x, float y) {
  const float p = x * y;
  return to_odd(p, fmaf(x, y, -p));
}
// x / scale for a code, |x| <= 448 scale (or not finite)
__device__ __forceinline__ float quotient_to_odd(float x, float scale) {
  if (scale < 0x1p-60f) { x *= 0x1p64f; scale *= 0x1p64f; }              // (the remainders below stay above the smallest number)
  const float inv = 1.f / scale, q = x * inv;
  if (!(fabsf(q) <= 1024.f)) return q;
  const float p = fmaf(fmaf(-q, scale, x), inv, q);                      // nearest but for rounding's error of the correction
  return to_odd(p, fmaf(-p, scale, x));
}

// The exponent of a block's scale: the smallest e from -126 to 120 with `largest` <= 448 * 2^e, 448 being 1.75 * 2^8.
__device__ __forceinline__ int scale_exponent(float largest) {
  const uint32_t b = __float_as_uint(largest);                           // not negative
  const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u);
  return min(max(e, -126), 120);
}
__device__ __forceinline__ float exp2_of(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

}  // namespace snap
