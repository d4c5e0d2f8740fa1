// exp and log in 64 bits with few registers, for the few values per row that a kernel needs them
// for while it holds the row: the library's functions would take as many registers as the row.
#pragma once

#include <hip/hip_runtime.h>

namespace tfm {

// ln 2: its first 40 bits, whose products with exponents are exact, and the rest.
constexpr double LN2_HI = 0x1.62e42fefa2000p-1, LN2_LO = 0x1.9ef35793c7673p-41;

// exp(x) = 2^n exp(r), n = round(x / ln 2), |r| <= ln 2 / 2: Taylor's series to r^13 / 13!, whose
// remainder is below 2^-57, by Horner's rule.  Relative error below 2^-51; NaN for NaN.
__device__ __forceinline__ double exp64(double x) {
  if (x < -800.0) return 0.0;
  if (x > 800.0) return INFINITY;
  const double n = __builtin_rint(x * (1.0 / (LN2_HI + LN2_LO)));
  double r = __builtin_fma(n, -LN2_HI, x);
  r = __builtin_fma(n, -LN2_LO, r);
  double p = 1.0 / 6227020800.0;
  p = __builtin_fma(p, r, 1.0 / 479001600.0);
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
  return __builtin_amdgcn_ldexp(p, (int)n);
}

// log(x) = e ln 2 + log m, m in [1/sqrt 2, sqrt 2): 2 artanh(f), f = (m - 1) / (m + 1), by its
// series to f^21 (f^2 <= 0.0295: the remainder is below 2^-57 of it).
__device__ __forceinline__ double log64(double x) {
  if (!(x > 0.0)) return x == 0.0 ? -INFINITY : NAN;
  if (x == INFINITY) return x;
  int e = __builtin_amdgcn_frexp_exp(x);
  double m = __builtin_amdgcn_frexp_mant(x);
  if (m < 0.70710678118654752) {
    m *= 2.0;
    --e;
  }
  const double f = (m - 1.0) / (m + 1.0), s = f * f;
  double p = 1.0 / 21.0;
  p = __builtin_fma(p, s, 1.0 / 19.0);
  p = __builtin_fma(p, s, 1.0 / 17.0);
  p = __builtin_fma(p, s, 1.0 / 15.0);
  p = __builtin_fma(p, s, 1.0 / 13.0);
  p = __builtin_fma(p, s, 1.0 / 11.0);
  p = __builtin_fma(p, s, 1.0 / 9.0);
  p = __builtin_fma(p, s, 1.0 / 7.0);
  p = __builtin_fma(p, s, 1.0 / 5.0);
  p = __builtin_fma(p, s, 1.0 / 3.0);
  p = __builtin_fma(p * s, 2.0 * f, 2.0 * f);
  return __builtin_fma((double)e, LN2_HI, __builtin_fma((double)e, LN2_LO, p));
}

}  // namespace tfm
