// tt_e4m3.cuh -- elements of an 8-bit cache: e4m3 values times a power of two that 16
// slots of a page share in a head, held as its exponent and 127 (E8M0).
#pragma once

#include <cstdint>

#include "tt_device.cuh"

namespace tt {

// 2^(code - 127); 255 stands for NaN.
__device__ __forceinline__ float e8m0(uint32_t code) {
  return __uint_as_float(code == 0 ? 0x00400000u : code == 255 ? 0x7fc00000u : code << 23);
}
// Its inverse, for codes 1 .. 254.
__device__ __forceinline__ float e8m0_inverse(uint32_t code) {
  return __uint_as_float(code == 254 ? 0x00400000u : (254 - code) << 23);
}
// The least code from 1 on whose 448 2^(code - 127) is at least x >= 0, finite (448 =
// 1.75 2^8).
__device__ __forceinline__ uint32_t e8m0_for(float x) {
  const uint32_t bits = __float_as_uint(x), up = (bits & 0x7fffffu) > 0x600000u;
  return max(1, int(bits >> 23) - 8 + int(up));
}

// Two values rounded to e4m3 (the nearest, ties to even; beyond 448: 448; NaN: NaN),
// lo in the low byte, and back.
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// (as two fp16 values: each e4m3 value is one)
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t two) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(uint16_t(two)));
  return r;
}

}  // namespace tt
