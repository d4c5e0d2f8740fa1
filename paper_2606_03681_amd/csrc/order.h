// Logits as integers in the same order, and the smallest logit that min_p keeps; for the host too,
// so that the search can be checked there.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace tfm {

// Key of a logit: 0 for what is never drawn (-inf and NaN).
__host__ __device__ __forceinline__ uint32_t key_of(float x) {
  if (!(x > -__builtin_inff())) return 0;
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.f);  // -0 and 0 are equal
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__host__ __device__ __forceinline__ float of_key(uint32_t k) {
  return __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// The smallest key in [lo, hi] that reaches, where every key above one that reaches does too and hi
// does: between `guess` and keys at doubling distances from it, then by halving.  Two or three tests
// where the guess is right, 64 at most wherever it lies.
template <class F>
__host__ __device__ __forceinline__ uint32_t first_key(uint32_t lo, uint32_t hi, uint32_t guess,
                                                       F reaches) {
  uint32_t step = 1;
  if (reaches(guess)) {
    hi = guess;
    while (lo < hi) {
      const uint32_t k = hi - lo > step ? hi - step : lo;
      if (!reaches(k)) {
        lo = k + 1;
        break;
      }
      hi = k;
      step += step;
    }
  } else {
    lo = guess + 1;
    while (lo < hi) {
      const uint32_t k = hi - lo > step ? lo + (step - 1) : hi - 1;
      if (reaches(k)) {
        hi = k;
        break;
      }
      lo = k + 1;
      step += step;
    }
  }
  while (lo < hi) {
    const uint32_t k = lo + (hi - lo) / 2;
    if (reaches(k)) hi = k;
    else lo = k + 1;
  }
  return lo;
}

// Key of the smallest logit s with (s - top) / tau >= least: least = log(min_p) <= 0, tau > 0, and
// top, the row's largest logit, not -inf or NaN.  top + least tau is a few keys off, but where the
// two cancel the keys next to 0 are far denser than the values that s - top can take.
__host__ __device__ __forceinline__ uint32_t min_p_key(double least, float tau, float top) {
  const uint32_t kmax = key_of(top), lowest = 0x00800000u;  // (of -FLT_MAX)
  if (top == __builtin_inff()) return kmax;
  const double itau = 1.0 / (double)tau;
  auto reaches = [&](uint32_t k) { return ((double)of_key(k) - (double)top) * itau >= least; };
  const double guess = (double)top + least * (double)tau;
  uint32_t k = lowest;
  if (guess > -3.4028234663852886e38) {
    k = key_of((float)guess);
    k = k < lowest ? lowest : k > kmax ? kmax : k;
  }
  return first_key(lowest, kmax, k, reaches);
}

}  // namespace tfm
