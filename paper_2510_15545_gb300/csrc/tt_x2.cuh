// tt_x2.cuh -- fp32 arithmetic on pairs (one instruction for two values), and the
// logits of a 16-byte vector as pairs: for kernels that stream logits rows and
// would be held up by the number of their instructions.
#pragma once

#include "tt_device.cuh"

namespace tt {

using f32x2 = unsigned long long;

__device__ __forceinline__ f32x2 pair(float lo, float hi) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void split(f32x2 x, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x));
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 exp2_pair(f32x2 x) {
  float lo, hi;
  split(x, lo, hi);
  return pair(ex2_approx(lo), ex2_approx(hi));
}
__device__ __forceinline__ float sum_pair(f32x2 x) {
  float lo, hi;
  split(x, lo, hi);
  return lo + hi;
}

// Pair q of a vector's logits (2 pairs of fp32, 4 of bf16).
template <int DT>
__device__ __forceinline__ f32x2 logit_pair(const uint4& w, int q) {
  if constexpr (DT == TT_F32) {
    return q == 0 ? pair(__uint_as_float(w.x), __uint_as_float(w.y))
                  : pair(__uint_as_float(w.z), __uint_as_float(w.w));
  } else {
    const uint32_t x = q == 0 ? w.x : q == 1 ? w.y : q == 2 ? w.z : w.w;
    return pair(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
  }
}

// The larger of each logit and `low` (two bf16 in a word, or one fp32); NaN stays.
template <int DT>
__device__ __forceinline__ uint32_t at_least(uint32_t w, uint32_t low) {
  uint32_t r;
  if constexpr (DT == TT_F32)
    asm("max.NaN.f32 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(low));
  else
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(low));
  return r;
}
template <int DT>
__device__ __forceinline__ uint4 at_least(const uint4& w, uint32_t low) {
  return make_uint4(at_least<DT>(w.x, low), at_least<DT>(w.y, low), at_least<DT>(w.z, low),
                    at_least<DT>(w.w, low));
}

}  // namespace tt
