// Device helpers of the 8-bit key/value cache: e4m3 values with one power-of-two scale per (page, KV head), keys and values apart.
//
// Layout of one (page, head): keys [D / 16, 16 tokens, 16], values [D, 16 tokens], one byte each.  A lane's 16 bytes are then a
// piece of one matrix operand of the attention kernel as they lie: 16 dimensions of one key, one dimension of 16 values.
//
// Why powers of two: e4m3 is a floating-point format, so another mantissa in the scale buys nothing inside its range of normal values,
// while a page whose scale grows, or an entry that moves to a page of a larger scale, is rewritten exactly but for what becomes
// subnormal; and the conversion instructions apply the exponent for free.
#pragma once
#include "common.h"

namespace specv {

constexpr int kQuantPage = 16;
constexpr int kLeastScaleExp = -100;          // the smallest nonzero entry, 2^-109, is still a normal bf16 and fp32 number
constexpr int kMostScaleExp = 119;            // the largest entry, 448 * 2^119, is still finite in bf16 (inputs beyond it saturate)

typedef float f32x2 __attribute__((ext_vector_type(2)));

// The least 2^e of that range with amax <= 448 * 2^e (448 = 1.75 * 2^8, the largest e4m3 value).  amax finite.
__device__ __forceinline__ float page_scale(float amax) {
  const uint32_t w = __float_as_uint(amax);
  const int e = static_cast<int>(w >> 23) - 127 - 8 + ((w & 0x7fffffu) > 0x600000u ? 1 : 0);
  return __uint_as_float(static_cast<uint32_t>(min(max(e, kLeastScaleExp), kMostScaleExp) + 127) << 23);
}
// 1 / s of a power of two 2^-126 .. 2^126, exactly.
__device__ __forceinline__ float inverse_scale(float s) { return __uint_as_float((254u << 23) - (__float_as_uint(s) & 0x7f800000u)); }

// |x| where it is finite, 0 for infinities and NaN: what a scale is made from.
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;
}
// To the range of e4m3 (infinities become +-448); NaN stays NaN.
__device__ __forceinline__ float to_e4m3_range(float x) { return x == x ? __builtin_amdgcn_fmed3f(x, -448.f, 448.f) : x; }

// Four values, already divided by their scale, as e4m3 (nearest even) in one word, and back.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(to_e4m3_range(a), to_e4m3_range(b), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(to_e4m3_range(c), to_e4m3_range(d), w, true);
  return static_cast<uint32_t>(w);
}
// Four entries times `ratio` <= 1, a power of two.
__device__ __forceinline__ uint32_t rescale_e4m3(uint32_t w, float ratio) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false);
  const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), true);
  return pack_e4m3(lo[0] * ratio, lo[1] * ratio, hi[0] * ratio, hi[1] * ratio);
}
// Byte mask of a word of four slots, the first of them slot t: those in [from, to).
__device__ __forceinline__ uint32_t slot_mask(int t, int from, int to) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m |= (t + i >= from && t + i < to) ? 0xffu << (8 * i) : 0u;
  return m;
}

}  // namespace specv
