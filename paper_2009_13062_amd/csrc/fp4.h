// The 4-bit rows of a cache: 32 neighbouring features share a scale 2^(byte - 127), an element is sign, two bits of exponent and one of fraction:
// +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} times the scale.  Two codes to a byte, the lower feature in the lower half; a row of d features is G = ceil(d / 32) groups of 16 bytes, features
// past d as 0, and G scales, one more byte (0) behind an odd number of them.
//
// The scale is the smallest power of two with |x| <= 7 * scale in the whole group, exponents -125 ... 125: up to 7 an element rounds to 6, off by no more than elsewhere
// between two codes (1 / 7), and a smaller scale than the usual floor(log2 max) - 2 gives from 6 to 7 is never taken, so none is cut by more.  Multiplying by a power of two is
// exact, so rounding to the nearest code (halfway to the even one) has one answer, which the hardware's conversions give: all 256 scales and both directions were checked.  Of a
// scale they look at the exponent alone.
// A group that holds an infinity or NaN gets the byte 255, which reads as NaN throughout.
#pragma once
#include "nf_common.h"

namespace nf {

constexpr int kFp4Group = 32, kFp4Odd = 255;
__host__ __device__ constexpr int fp4_groups(int d) { return (d + kFp4Group - 1) / kFp4Group; }
__host__ __device__ constexpr int fp4_code_bytes(int d) { return fp4_groups(d) * (kFp4Group / 2); }
__host__ __device__ constexpr int fp4_scale_bytes(int d) { return fp4_groups(d) + fp4_groups(d) % 2; }

// Scale byte of a group whose largest magnitude has these bits (sign cleared).  Adding 0x1fffff carries into the exponent from 1.75 times a power of two up.
__device__ __forceinline__ uint32_t fp4_scale(uint32_t top) {
  const int e = (int)((top + 0x1fffffu) >> 23) - 2;
  return top >= 0x7f800000u ? kFp4Odd : (uint32_t)min(max(e, 2), 252);
}
__device__ __forceinline__ float fp4_scale_value(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight neighbouring features to a dword of codes
__device__ __forceinline__ uint32_t fp4_codes(const float (&x)[8], uint32_t scale) {
  const float s = fp4_scale_value(scale);
  uint32_t r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], s, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], s, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], s, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], s, 3);
  return scale == kFp4Odd ? 0u : r;
}
// The same of bfloat16 features, a pair to a dword
__device__ __forceinline__ uint32_t fp4_codes(const uint4& w, uint32_t scale) {
  const float s = fp4_scale_value(scale);
  uint32_t r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, __builtin_bit_cast(bf16x2_t, w.x), s, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2_t, w.y), s, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2_t, w.z), s, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2_t, w.w), s, 3);
  return scale == kFp4Odd ? 0u : r;
}

// Byte SEL of a dword of codes to two values: bfloat16 in a dword, or float32.  (NaN under the byte 255.)
template <int SEL> __device__ __forceinline__ uint32_t fp4_pair_bf16(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
}
template <int SEL> __device__ __forceinline__ f32x2_t fp4_pair_f32(uint32_t codes, float scale) { return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, SEL); }
// A dword of codes to eight values
__device__ __forceinline__ uint4 fp4_values_bf16(uint32_t codes, float scale) {
  return make_uint4(fp4_pair_bf16<0>(codes, scale), fp4_pair_bf16<1>(codes, scale), fp4_pair_bf16<2>(codes, scale), fp4_pair_bf16<3>(codes, scale));
}
// One element of a row, for the kernels that take any size
__device__ __forceinline__ float fp4_value(const uint8_t* codes, const uint8_t* scales, int t) {
  const f32x2_t v = fp4_pair_f32<0>(codes[t / 2], fp4_scale_value(scales[t / kFp4Group]));
  return t % 2 ? v.y : v.x;
}

}  // namespace nf
