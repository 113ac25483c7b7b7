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
// What an integer sum stands for: sum * (row's scale * column's).  Scales of quantised bf16 lie anywhere from 2^-125 to 2^121, so the product of two
// can leave fp32's normal range where the result does not; the sum is then multiplied by the smaller scale first, which neither loses bits (a sum is a
// whole number below 2^31: where the product is subnormal, it is exact) nor overflows unless the result does.  NaN stays NaN.
__device__ __forceinline__ float value8(int sum, float row, float col) {
  const float both = row * col;
  if (fabsf(both) >= 0x1p-126f && fabsf(both) <= 3.402823466e38f) return (float)sum * both;
  const bool first = fabsf(row) < fabsf(col);
  return (float)sum * (first ? row : col) * (first ? col : row);
}
// Whether a scale needs that care: products of two others (2^-63 to 2^63, and 0) stay in range, and then value8 is sum * (row * col), bit for bit.
// Tiles without such a scale are multiplied that way, a vote a tile, in code of their own (E 128, C 4096, 1024 -> 4096: 2 050 us; 2 227 with the choice in
// one loop, which spilled).
__device__ __forceinline__ bool far8(float scale) {
  const uint32_t u = __float_as_uint(scale) & 0x7fffffffu;
  return u != 0 && u - 0x20000000u > 0x5f000000u - 0x20000000u;
}
__device__ __forceinline__ bool far8(float4 s) { return far8(s.x) || far8(s.y) || far8(s.z) || far8(s.w); }
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
