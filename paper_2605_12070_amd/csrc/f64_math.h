// 64-bit base-2 exponential and logarithm for the vocabulary rows' exact paths.
#pragma once

#include <hip/hip_runtime.h>

namespace dppo {

constexpr double kLn2F64 = 0.69314718055994530942;
constexpr double kLog2eF64 = 1.44269504088896340736;

// 2^f for |f| <= 1/2: the polynomial of degree 9 through 2^f at the ten Chebyshev nodes of the
// interval, relative error 1.9e-14 (ten fused multiply-adds, which run at the 32-bit rate on this
// device).
__device__ __forceinline__ double exp2_poly(double f) {
  double p = 1.0205905413765595e-07;
  p = __builtin_fma(p, f, 1.325964524488711e-06);
  p = __builtin_fma(p, f, 1.5252672924850737e-05);
  p = __builtin_fma(p, f, 0.0001540343375125101);
  p = __builtin_fma(p, f, 0.0013333558200794592);
  p = __builtin_fma(p, f, 0.009618129193934313);
  p = __builtin_fma(p, f, 0.05550410866465167);
  p = __builtin_fma(p, f, 0.2402265069564034);
  p = __builtin_fma(p, f, 0.6931471805599462);
  return __builtin_fma(p, f, 1.0000000000000135);
}

// 2^x; 0 below 2^-1100 (-inf included), NaN for NaN and +inf.
__device__ __forceinline__ double exp2_f64(double x) {
  const double n = __builtin_rint(x);
  const double r = __builtin_ldexp(exp2_poly(x - n), (int)n);
  return x < -1100.0 ? 0.0 : r;
}

// log2 x for positive x in float's range: the 32-bit logarithm and one Newton step (its error of
// 1e-7 |y| squares to 1e-13 or less).
__device__ __forceinline__ double log2_f64(double x) {
  const double y = (double)log2f((float)x);
  const double e = __builtin_fma(x, exp2_f64(-y), -1.0);
  return y + e * (1.0 - 0.5 * e) * kLog2eF64;
}

}  // namespace dppo
