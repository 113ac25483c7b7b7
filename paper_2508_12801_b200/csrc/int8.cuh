// Steps of 8-bit integers: rows, weights and blocks of kept activations.
//
// Values of largest magnitude amax become q = rint(x * inv), inv = 127 / amax, and stand for q * scale, scale = amax / 127, both in
// fp32.  One fused multiply-add does it: x * inv + 1.5 * 2^23 is rounded once, to the nearest whole number (ties to even), and that number is
// the sum's low byte.  Below amax = 2^-118, where inv would leave fp32's range, everything is zero; values that are not finite
// give a scale of NaN, so that whatever is computed from them is NaN.
#pragma once
#include "common.cuh"

namespace msr {

constexpr int kKeepBlock = 32;                       // columns of kept activations that share a scale
__host__ __device__ constexpr int keep_width(int d_ff) { return (d_ff + kKeepBlock - 1) / kKeepBlock * kKeepBlock; }

struct Step8 { float inv, scale; };                  // 1 / step and step
__device__ __forceinline__ Step8 step8(uint32_t amax_bits) {
  const float amax = __uint_as_float(amax_bits);
  Step8 s{0.f, 0.f};
  if (amax_bits >= 0x7f800000u) s.scale = __uint_as_float(0x7fc00000u);
  else if (amax >= 0x1p-118f) { s.inv = 127.f / amax; s.scale = amax / 127.f; }
  return s;
}
__device__ __forceinline__ uint32_t round8(float x, float inv) { return __float_as_uint(fmaf(x, inv, 12582912.f)); }      // the low byte
__device__ __forceinline__ uint32_t pack8(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
__device__ __forceinline__ uint32_t abs_bits(uint32_t u) { return u & 0x7fffffffu; }
// the larger of m and the magnitudes of a and b; NaN wins
__device__ __forceinline__ float max_abs(float m, float a, float b) {
  asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(fabsf(a)), "f"(fabsf(b)));
  return m;
}
// Integer i of a word of four, plus kByte8Zero, as a float: exact.  The word comes with its sign bits flipped (^ 0x80808080).
constexpr float kByte8Zero = 8388736.f;              // 2^23 + 128
__device__ __forceinline__ float byte8_raw(uint32_t flipped, int i) { return __uint_as_float(__byte_perm(flipped, 0x4b000000u, 0x7440 + i)); }

}  // namespace msr
