// 64-bit base-2 exponential and logarithm for the vocabulary rows' exact paths.
#pragma once

#include <hip/hip_runtime.h>

#include "dppo_device.h"

namespace dppo {

constexpr double kLn2F64 = 0.69314718055994530942;
constexpr double kLog2eF64 = 1.44269504088896340736;

// p * f + c with the constant in a scalar register: left to itself the compiler keeps the polynomial's
// constants in vector registers (18 of them) and copies each before it is accumulated upon.
__device__ __forceinline__ double fma_const(double p, double f, double c) {
  double r;
  asm("v_fma_f64 %0, %1, %2, %3" : "=v"(r) : "v"(p), "v"(f), "s"(c));
  return r;
}

// 2^f for |f| <= 1/2: the polynomial of degree 9 through 2^f at the ten Chebyshev nodes of the
// interval, relative error 1.9e-14 (fused multiply-adds: 5.2 cycles a wave, in 32 bits 2.9; most other
// 64-bit instructions take as long as those).
__device__ __forceinline__ double exp2_poly(double f) {
  double p = fma_const(f, 1.0205905413765595e-07, 1.325964524488711e-06);
  p = fma_const(p, f, 1.5252672924850737e-05);
  p = fma_const(p, f, 0.0001540343375125101);
  p = fma_const(p, f, 0.0013333558200794592);
  p = fma_const(p, f, 0.009618129193934313);
  p = fma_const(p, f, 0.05550410866465167);
  p = fma_const(p, f, 0.2402265069564034);
  p = fma_const(p, f, 0.6931471805599462);
  return fma_const(p, f, 1.0000000000000135);
}

// 2^(x / 64) for many x: a table of 2^(j / 64) in LDS (64 doubles: every bank once or twice) and a
// polynomial of degree 3 through the Chebyshev nodes of the rest, relative error 4.5e-12; about
// three quarters of exp2_f64's instructions. x = z K + S with an integer S: the integer nearest to x
// is read off the low bits of fma(z, K, S + 1.5 2^52), and the rest is one more fused multiply-add,
// exact for any z. |x| < 2^31, or NaN, which stays NaN.
constexpr int kExpTable = 64;
constexpr double kRoundMagic = 6755399441055744.0;   // 1.5 * 2^52
__device__ __forceinline__ double exp2_tab(double z, double K, double S_magic, const double* table) {
  const double t = __builtin_fma(z, K, S_magic);
  const int n = (int)(uint32_t)__builtin_bit_cast(uint64_t, t);
  const double r = __builtin_fma(z, K, S_magic - t);
  double p = fma_const(r, 2.1173168200092995e-07, 5.8649192871976494e-05);
  p = fma_const(p, r, 0.010830424696239445);
  p = fma_const(p, r, 0.9999999999955212);
  return __builtin_ldexp(p * table[n & (kExpTable - 1)], n >> 6);
}

// 2^x; 0 below 2^-1100 (-inf included), NaN for NaN and +inf.
__device__ __forceinline__ double exp2_f64(double x) {
  const double n = __builtin_rint(x);
  const double r = __builtin_ldexp(exp2_poly(x - n), (int)n);
  return x < -1100.0 ? 0.0 : r;
}

// By the workgroup's first 64 threads; a barrier follows before the table is read.
__device__ __forceinline__ void exp2_table_fill(double* table) {
  if (threadIdx.x < kExpTable) table[threadIdx.x] = exp2_f64((double)threadIdx.x / kExpTable);
}

// log2 x for positive x in float's range: the 32-bit logarithm and one Newton step (its error of
// 1e-7 |y| squares to 1e-13 or less).
__device__ __forceinline__ double log2_f64(double x) {
  const double y = (double)log2f((float)x);
  const double e = __builtin_fma(x, exp2_f64(-y), -1.0);
  return y + e * (1.0 - 0.5 * e) * kLog2eF64;
}

// Wave-wide sum and maximum in 64 bits; every lane returns the same bits (a fixed tree of DPP moves
// and permlane swaps, as the 32-bit ones).
__device__ __forceinline__ double f64_of(uint32_t lo, uint32_t hi) {
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int CTRL>
__device__ __forceinline__ double dpp_d(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  return f64_of(__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xF, 0xF, false),
                __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, 0xF, 0xF, false));
}
// across the four rows of 16 lanes
template <class F>
__device__ __forceinline__ double wave_fold_rows(double v, F&& f) {
  uint64_t u = __builtin_bit_cast(uint64_t, v);
  auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)u, (uint32_t)u, false, false);
  auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
  v = f(f64_of(lo[0], hi[0]), f64_of(lo[1], hi[1]));
  u = __builtin_bit_cast(uint64_t, v);
  lo = __builtin_amdgcn_permlane32_swap((uint32_t)u, (uint32_t)u, false, false);
  hi = __builtin_amdgcn_permlane32_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
  return f(f64_of(lo[0], hi[0]), f64_of(lo[1], hi[1]));
}
template <class F>
__device__ __forceinline__ double wave_fold_f64(double v, F&& f) {
  v = f(v, dpp_d<0xB1>(v));    // quad_perm [1,0,3,2]
  v = f(v, dpp_d<0x4E>(v));    // quad_perm [2,3,0,1]
  v = f(v, dpp_d<0x141>(v));   // row_half_mirror
  v = f(v, dpp_d<0x140>(v));   // row_mirror
  return wave_fold_rows(v, f);
}
__device__ __forceinline__ double wave_sum_f64(double v) {
  return wave_fold_f64(v, [](double a, double b) { return a + b; });
}
__device__ __forceinline__ double wave_max_f64(double v) {
  return wave_fold_f64(v, [](double a, double b) { return fmax(a, b); });
}
// Four wave-wide sums at less than half of four wave_sum_f64: in two steps each lane of a quad takes
// over one of them. Lane i returns v[i & 3]'s.
__device__ __forceinline__ double wave_sum4_f64(const double (&v)[4]) {
  const int lane = (int)(threadIdx.x & 63);
  const bool odd = lane & 1, upper = lane & 2;
  const double a = (odd ? v[1] : v[0]) + dpp_d<0xB1>(odd ? v[0] : v[1]);       // from lane ^ 1
  const double b = (odd ? v[3] : v[2]) + dpp_d<0xB1>(odd ? v[2] : v[3]);
  double s = (upper ? b : a) + dpp_d<0x4E>(upper ? a : b);                     // from lane ^ 2
  s += dpp_d<0x124>(s);        // row_ror:4
  s += dpp_d<0x128>(s);        // row_ror:8
  return wave_fold_rows(s, [](double x, double y) { return x + y; });
}
// A value that every lane of the wave holds, in scalar registers.
__device__ __forceinline__ double wave_uniform(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  return f64_of((uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)u),
                (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(u >> 32)));
}

}  // namespace dppo
