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

// Bytes of a word of scales that are kScaleNan, or more than any stored position's (253 and
// 254 make infinities): bits 7, 15, 23 and 31.
__device__ __forceinline__ uint32_t beyond_252(uint32_t x) { return ((x & 0x7F7F7F7Fu) + 0x03030303u) & x & 0x80808080u; }

// Calls found(block, slot) for the NaN blocks among a tile's value scales [B][64], a byte after the other:
// only tiles of which not all rows see all, and which hold such blocks, are searched, but there it
// is as long as several tiles.  One token with NaN values near the end: 137 tokens of 16/2/64
// heads in a window of 1000 8 -> 18 us, 300 of 32/8/128 in one of 4096 42 -> 61, 2048 of them 140 ->
// 150, 2048 behind 30720 933 -> 952; one in every tile 29, 83, 196, 1609.
template <int B, typename Found>
__device__ __forceinline__ void each_nan(const uint8_t* scales, Found found) {
#pragma unroll 1
  for (int i = 0; i < B * 64; ++i)
    if (scales[i] == kScaleNan) found(i / 64, i % 64);
}

__device__ __forceinline__ uint32_t div_by(uint32_t n, uint32_t magic, int shift) {
  return (__umulhi(n, magic) + n) >> shift;
}

// The tiles of a run of a chunk's rows at positions [first, last]: the sinks' [0, sinks),
// then [begin, end).
struct Tiles {
  int sinks, begin, end;
  __device__ __forceinline__ int count() const { return sinks + end - begin; }
  __device__ __forceinline__ int at(int i) const { return i < sinks ? i : i - sinks + begin; }
};
__device__ __forceinline__ Tiles tiles_of(const WindowLaunch& p, int first, int last) {
  const int low = max(0, first - p.window + 1);
  Tiles t;
  t.begin = low / kTileKeys;
  t.end = last / kTileKeys + 1;
  t.sinks = min((min(p.sinks, low) + kTileKeys - 1) / kTileKeys, t.begin);
  return t;
}
// Whether all of these rows see a whole tile.
__device__ __forceinline__ bool seen_in_full(const WindowLaunch& p, int tile, int first, int last) {
  const int k0 = tile * kTileKeys, k1 = k0 + kTileKeys;
  return k1 <= first + 1 && (k0 > last - p.window || k1 <= p.sinks);
}

}  // namespace
}  // namespace mocap
