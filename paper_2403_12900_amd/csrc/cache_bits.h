// Bit masks over the four code bytes, or scale bytes, of a word of the 4-bit
// cache: positions 0 .. 3 of a group of dimensions.  Shared with the host test
// library.
#pragma once

#include <cstdint>

#ifdef __HIP__
#include <hip/hip_runtime.h>
#define SPRK_ANYWHERE __host__ __device__ __forceinline__
#else
#define SPRK_ANYWHERE inline
#endif

namespace sprk {

// Bytes whose bit of b (4 of them) is set, as a mask.
SPRK_ANYWHERE uint32_t byte_mask(uint32_t b) { return ((b * 0x00204081u) & 0x01010101u) * 255u; }

// Which of a word's scale bytes are 255 (NaN): the top bit of each.
SPRK_ANYWHERE uint32_t nan_bytes(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & w & 0x80808080u; }
SPRK_ANYWHERE uint32_t nan_bits(uint32_t w) {
  const uint32_t x = nan_bytes(w) >> 7;
  return (x | x >> 7 | x >> 14 | x >> 21) & 15u;
}

// Not 0: one of a word's scales is outside 2^-18 .. 2^13 (bytes 109 .. 140: a byte
// out of that range leaves a top bit, and the lowest such byte has no borrow from
// below).
SPRK_ANYWHERE uint32_t odd_scales(uint32_t scales) { return (scales - 0x6D6D6D6Du) & 0xE0E0E0E0u; }
// Whether a word's values are not all exact in fp16: a position with such a scale
// and a code that is not zero, or a NaN.  (A group of zeros has the lowest scale,
// and zeros are exact.)
SPRK_ANYWHERE bool beyond_f16(uint32_t w, uint32_t scales) {
  // byte - 109 without borrows, and whether it is past 31, in each byte's top bit.
  const uint32_t t = (((scales | 0x80808080u) - 0x6D6D6D6Du) ^ (~scales & 0x80808080u)) & 0xE0E0E0E0u;
  const uint32_t odd = t | t << 1 | t << 2, some = (w & 0x77777777u) + 0x7F7F7F7Fu;
  return ((odd & some & 0x80808080u) | nan_bytes(scales)) != 0;
}

}  // namespace sprk

#undef SPRK_ANYWHERE
