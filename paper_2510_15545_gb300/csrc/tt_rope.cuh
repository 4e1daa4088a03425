// tt_rope.cuh -- the angle of a rotary position, and what kernels that rotate heads
// share: elements of 16-bit and 32-bit types in 16-byte vectors.
#pragma once

#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "tt_device.cuh"

namespace tt {

struct Turn {
  float c, s;  // cosine and sine
};

// Position x of a pair that makes F 2^-64 turns per position. x F mod 2^64 is the
// angle in 2^-64 turns, exactly: far positions cost no digits, as they do when an
// angle of a million radians is formed in fp32 (its unit there is 0.06). What is
// left after the nearest quarter turn, |r| <= pi / 4, goes through the series of
// sine and cosine (first terms left out: r^11 / 11!, 1.8e-9, and r^12 / 12!,
// 1.2e-10); the quarters swap the two and their signs.
__device__ __forceinline__ Turn turn_of(int32_t x, uint64_t F) {
  const uint32_t p = uint32_t((uint64_t(int64_t(x)) * F) >> 32);
  const uint32_t quarter = (p + 0x20000000u) >> 30;
  const float r = float(int32_t(p - (quarter << 30))) * 1.46291807926715968e-9f;  // 2 pi 2^-32
  const float x2 = r * r;
  float s = fmaf(x2, 2.75573192e-6f, -1.98412698e-4f);
  s = fmaf(x2, s, 8.33333333e-3f);
  s = fmaf(x2, s, -1.66666667e-1f);
  s = fmaf(x2 * r, s, r);
  float c = fmaf(x2, -2.75573192e-7f, 2.48015873e-5f);
  c = fmaf(x2, c, -1.38888889e-3f);
  c = fmaf(x2, c, 4.16666667e-2f);
  c = fmaf(x2, c, -0.5f);
  c = fmaf(x2, c, 1.f);
  const float cc = quarter & 1 ? s : c, ss = quarter & 1 ? c : s;
  return {__uint_as_float(__float_as_uint(cc) ^ (((quarter + 1) & 2) << 30)),
          __uint_as_float(__float_as_uint(ss) ^ ((quarter & 2) << 30))};
}

// The pair (a, b) turned: rounded three times in fp32.
__device__ __forceinline__ void turn_pair(const Turn& t, float& a, float& b) {
  const float x = fmaf(a, t.c, -(b * t.s)), y = fmaf(b, t.c, a * t.s);
  a = x;
  b = y;
}

// Elements of a 16-byte vector as fp32, and back, each rounded once.
template <int DT>
struct Elems {
  static constexpr int kCount = DT == TT_F32 ? 4 : 8;
  static constexpr int kBytes = DT == TT_F32 ? 4 : 2;
};
template <int DT>
__device__ __forceinline__ void unpack16(const uint4& w, float (&e)[Elems<DT>::kCount]) {
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT == TT_F32) {
      e[i] = __uint_as_float(v[i]);
    } else if constexpr (DT == TT_BF16) {
      e[2 * i] = __uint_as_float(v[i] << 16);
      e[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    } else {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v[i]));
      e[2 * i] = f.x;
      e[2 * i + 1] = f.y;
    }
  }
}
template <int DT>
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {
  uint32_t r;
  if constexpr (DT == TT_F16)
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <int DT>
__device__ __forceinline__ uint4 pack16(const float (&e)[Elems<DT>::kCount]) {
  if constexpr (DT == TT_F32) {
    return make_uint4(__float_as_uint(e[0]), __float_as_uint(e[1]), __float_as_uint(e[2]),
                      __float_as_uint(e[3]));
  } else {
    return make_uint4(pack_pair<DT>(e[0], e[1]), pack_pair<DT>(e[2], e[3]),
                      pack_pair<DT>(e[4], e[5]), pack_pair<DT>(e[6], e[7]));
  }
}
// One element.
template <int DT>
__device__ __forceinline__ float load_elem(const char* p) {
  if constexpr (DT == TT_F32) return *reinterpret_cast<const float*>(p);
  const uint16_t x = *reinterpret_cast<const uint16_t*>(p);
  return DT == TT_BF16 ? __uint_as_float(uint32_t(x) << 16) : __half2float(__ushort_as_half(x));
}
template <int DT>
__device__ __forceinline__ void store_elem(char* p, float x) {
  if constexpr (DT == TT_F32)
    *reinterpret_cast<float*>(p) = x;
  else
    *reinterpret_cast<uint16_t*>(p) = uint16_t(pack_pair<DT>(x, 0.f));
}

}  // namespace tt
