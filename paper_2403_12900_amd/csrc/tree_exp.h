// The fp64 exponential of the verification kernels, shared with the host test
// library.
#pragma once

#include <cstdint>

#ifdef __HIP__
#define SPRK_ANYWHERE __host__ __device__ __forceinline__
#else
#define SPRK_ANYWHERE inline
#endif

namespace sprk {

// exp(x) for x <= 0 to 2^-50 of its value, 0 below -708 (where the result
// would leave the normal range): x = n ln 2 + r, |r| <= ln 2 / 2, with ln 2 in
// two parts, and the Taylor polynomial of degree 12 of e^r.  Its rest is below
// r^13 / 13! < 1.7e-16, 2.4e-16 of the smallest e^r; the roundings of r and of
// the products add at most 3e-16 (degree 11 left 8.8e-15).  Adding 1.5 * 2^52
// leaves n, rounded, in the low bits of the sum, from where it goes into the
// exponent: no conversions, which run at a quarter of the rate of the products.
SPRK_ANYWHERE double exp_neg(double x) {
  constexpr double kShift = 6755399441055744.0;
  const double t = __builtin_fma(x, 1.4426950408889634, kShift), n = t - kShift;
  double r = __builtin_fma(n, -0x1.62e42fefa39efp-1, x);
  r = __builtin_fma(n, -0x1.abc9e3b39803fp-56, r);
  double p = 1.0 / 479001600.0;
  p = __builtin_fma(p, r, 1.0 / 39916800.0);
  p = __builtin_fma(p, r, 1.0 / 3628800.0);
  p = __builtin_fma(p, r, 1.0 / 362880.0);
  p = __builtin_fma(p, r, 1.0 / 40320.0);
  p = __builtin_fma(p, r, 1.0 / 5040.0);
  p = __builtin_fma(p, r, 1.0 / 720.0);
  p = __builtin_fma(p, r, 1.0 / 120.0);
  p = __builtin_fma(p, r, 1.0 / 24.0);
  p = __builtin_fma(p, r, 1.0 / 6.0);
  p = __builtin_fma(p, r, 0.5);
  p = __builtin_fma(p, r, 1.0);
  p = __builtin_fma(p, r, 1.0);
  const uint64_t bits = __builtin_bit_cast(uint64_t, p);
  const uint32_t hi = static_cast<uint32_t>(bits >> 32) + (static_cast<uint32_t>(__builtin_bit_cast(uint64_t, t)) << 20);
  const double e = __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | static_cast<uint32_t>(bits));
  return x < -708.0 ? 0.0 : e;
}

}  // namespace sprk

#undef SPRK_ANYWHERE
