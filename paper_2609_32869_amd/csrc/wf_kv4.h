// Rounding to the 4-bit cache (internal): block scales and codes, as the store and the
// request-time product's epilogue write them.
#pragma once
#include "wf_common.h"
#include "wf_ops.h"

namespace wf {

// Smallest 2^e, e >= -120, with amax <= 6 * 2^e, as a biased exponent: amax = m 2^x with
// 1 <= m < 2 is <= 6 * 2^e = 1.5 * 2^(e + 2) for e = x - 2 where m <= 1.5, else x - 1.
// 0xff where amax is not finite.
__device__ __forceinline__ uint32_t scale_of(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - ((u & 0x7fffffu) <= 0x400000u ? 2 : 1);
  return (u >> 23) == 255u ? 255u : (uint32_t)max(e, 7);
}

// 8 values -> 8 codes, element i in nibble i.
__device__ __forceinline__ uint32_t codes8(const float* x, float s) {
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], s, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], s, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], s, 3);
}

// max |x| that keeps a NaN (fmaxf would drop it): |x| as integers, NaN above infinity
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ float scale_f(uint32_t byte) { return __uint_as_float(byte << 23); }

// 4 values -> 4 codes in the low half.
__device__ __forceinline__ uint32_t codes4(const float* x, float s) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(__builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], s, 0), x[2], x[3], s, 1) & 0xffffu;
}
// A group's key word: dims 8 i .. + 7 of frame f (of 32); its block's scale byte.
__device__ __forceinline__ uint8_t* key_word(uint8_t* group, int f, int i) {
  return group + 16 * (16 * (i >> 1) + (f & 15)) + 8 * (f >> 4) + 4 * (i & 1);
}
__device__ __forceinline__ uint8_t* key_scale(uint8_t* group, int f, int half) {
  return group + kKv4KeyScale + 32 * half + 2 * (f & 15) + (f >> 4);
}
// Its value word: frames 8 i .. + 7 of a dim; the scale byte lies at kKv4ValueScale + dim.
__device__ __forceinline__ uint8_t* value_word(uint8_t* group, int i, int dim) { return group + kKv4Values + 256 * i + 4 * dim; }

}  // namespace wf
