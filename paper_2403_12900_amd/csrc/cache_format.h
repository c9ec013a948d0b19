// The 4-bit cache's tiles on the device: where a (block, head)'s bytes lie and
// how values become codes.
//
// A tile is 16 positions of one KV head: key codes, value codes, key scales,
// value scales (17 * HD bytes).  Lane l = r + 16 g of a wave finds what it
// feeds the matrix unit with in one piece: of the keys, position r and HD / 4
// consecutive dimensions; of the values, positions 4 g .. 4 g + 3 and
// dimensions r, r + 16, r + 32, ...  A code byte holds two dimensions of one
// position, so one conversion with that position's scale gives both, and codes
// with two significant bits are exact in bf16 at every scale.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_common.h"

namespace sprk {

template <int HD>
struct Mx4 {
  static constexpr int P = HD / 32;          // groups of 32 dimensions
  static constexpr int kTile = 17 * HD;      // bytes
  static constexpr int kV = 8 * HD, kKs = 16 * HD, kVs = 16 * HD + HD / 2;
  static __device__ __forceinline__ int key_code(int t, int d) { return (d / 32 * 16 + t) * 16 + d % 32 / 2; }
  static __device__ __forceinline__ int value_word(int g, int e, int p) { return kV + ((g * 16 + e) * P + p) * 4; }
  static __device__ __forceinline__ int key_scale(int t, int p) { return kKs + p * 16 + t; }
  static __device__ __forceinline__ int value_scales(int g, int p) { return kVs + (g * P + p) * 4; }
};

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

// Scale byte i of a word as the conversions take it: they read the exponent
// bits of an fp32 number and nothing else of it (2^(byte - 127); 255 is NaN).
template <int I>
__device__ __forceinline__ float scale_of(uint32_t w) {
  if constexpr (I == 0) return __uint_as_float(w << 23);
  else if constexpr (I == 1) return __uint_as_float(w << 15);
  else if constexpr (I == 2) return __uint_as_float(w << 7);
  else return __uint_as_float(w >> 1);
}

// Values of code byte I of w, low nibble first, in two bf16 or fp16 or fp32.
template <int I>
__device__ __forceinline__ uint32_t codes_to_bf16(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, I));
}
template <int I>
__device__ __forceinline__ uint32_t codes_to_f16(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, I));
}
template <int I>
__device__ __forceinline__ f32x2_t codes_to_f32(uint32_t w, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, I);
}

// Scale byte of a group whose largest element has the magnitude bits `top`:
// with top = 2^e (1 + m), the smallest s with top <= 7 * 2^s = 1.75 * 2^(s + 2).
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  const int e = static_cast<int>(top >> 23);
  if (e == 255) return 255;
  const int s = e - 129 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return static_cast<uint32_t>(min(max(s, -120), 125) + 127);
}

// Eight values as codes, the first in the lowest nibble.  The conversion
// rounds to nearest, ties to the even code, and saturates at 6.
__device__ __forceinline__ uint32_t to_codes(const float* x, float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
  return w;
}

// x in fp32, rounded to odd: cut, with the last bit set where anything was cut
// off.  Comparisons with numbers of fewer bits (the borders of scales and
// codes) come out as they would for x itself.  Finite x stay finite.
__device__ __forceinline__ float odd_f32(double x) {
  const float f = static_cast<float>(x);
  if (static_cast<double>(f) == x || !isfinite(x)) return f;
  uint32_t u = __float_as_uint(f);
  if (fabs(static_cast<double>(f)) > fabs(x)) u -= 1;
  return __uint_as_float(u | 1u);
}

}  // namespace sprk
