// Device code of the 4-bit store (its format: mocap_cache.h).
//
// gfx950 converts between fp4 (e2m1) and bf16 or fp32 two values at a time, with a
// scale of which only the exponent bits 30:23 count and which may be NaN (exponent
// 255: both results are NaN); to fp4 it rounds to nearest even and saturates.  A
// scale byte is therefore its own exponent field, wherever the other bits come from.
#pragma once

#include "attn_device.h"
#include "cache.h"

namespace mocap {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kScaleNan = 255;

// Byte b (a constant) of a word of scale bytes as a scale.
__device__ __forceinline__ float scale_of(uint32_t word, int b) {
  return __uint_as_float(b == 3 ? word >> 1 : word << (23 - 8 * b));
}

// Byte b (a constant) of a word of codes: its low value in the low half.
template <int B>
__device__ __forceinline__ uint32_t two_values(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B));
}

// The low and the high halves of two words, as pairs.
__device__ __forceinline__ uint32_t low_halves(uint32_t first, uint32_t second) {
  return __builtin_amdgcn_perm(second, first, 0x05040100);
}
__device__ __forceinline__ uint32_t high_halves(uint32_t first, uint32_t second) {
  return __builtin_amdgcn_perm(second, first, 0x07060302);
}

// Scale byte of values of which the largest magnitude has these bits (fp32): the
// exponent, one more where the fraction is over 1.5.
__device__ __forceinline__ int scale_byte(uint32_t largest) {
  if (largest >= 0x7F800000u) return kScaleNan;
  return min(max((int)((largest + 0x3FFFFFu) >> 23) - 2, 2), 252);
}

// Eight values as codes; a block that is not finite has codes 0.
__device__ __forceinline__ uint32_t eight_codes(const float* x, int byte) {
  if (byte == kScaleNan) return 0;
  const float scale = __uint_as_float((uint32_t)byte << 23);
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], scale, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], scale, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], scale, 3);
}

// The largest magnitude of eight values, as bits (NaN above infinity above all others).
__device__ __forceinline__ uint32_t largest_bits(const float* x) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(x[j]) & 0x7FFFFFFFu);
  return m;
}

}  // namespace
}  // namespace mocap
