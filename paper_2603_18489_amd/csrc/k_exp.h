// The exponentials of the vocabulary reduction and of the sampler.  Nothing in here needs the GPU: a test builds this file for the CPU, with a
// rounded 2^t in the hardware instruction's place.
#pragma once
#include <math.h>

namespace ec {

// e^d for -200 <= d <= 0, to about an ulp where that is a normal number: 2^t for the rounded product t = d log2 e, times
// 1 + (d - t ln 2).  float32's ln 2 is 1.9e-9 too large: ln 2 = 0.693147182464600 - 1.9046543e-9.  On MI355X, against 64 bits
// over 2^20 arguments from -87 to -50 as from -9 to -5: 1.4e-7 at most, -3.4e-9 on average, the bias of the hardware's 2^t itself
// (expf: 8.2e-8, -2.4e-9).  Sums of these and of expf's are equally exact: confidences of 5120 rows each of six vocabularies are
// 5.0e-8 to 7.9e-8 off r.m.s. with either.
__device__ __forceinline__ float exp_of_negative(float d) {
  const float t = d * 1.44269502f;
  const float r = fmaf(t, 1.9046543e-9f, fmaf(t, -0.693147182f, d));
  const float e = __builtin_amdgcn_exp2f(t);
  return fmaf(e, r, e);
}

// 2^(t + 46) for t <= 0.  2^t = 2^n p(t - n) with n the nearest whole number and p = 1 + f q(f), q of degree 8 through (2^f - 1) / f at the Chebyshev
// nodes of [-1/2, 1/2]: off by 3.7e-14 at most, and exact at whole t.
__device__ __forceinline__ double exp2_times_2to46(double t) {
  t = t > -200.0 ? t : -200.0;   // (past the last whose whole number is not 0)
  // n stands in the low bits of t + 1.5 2^52, and goes to the exponent as a whole number
  const double s = t + 0x1.8p52, f = t - (s - 0x1.8p52);
  double p = 0x1.b63880c66ae27p-24;
  p = fma(p, f, 0x1.63d136367c2a9p-20);
  p = fma(p, f, 0x1.ffcb951593514p-17);
  p = fma(p, f, 0x1.4308ac85aa724p-13);
  p = fma(p, f, 0x1.5d87fe86fe886p-10);
  p = fma(p, f, 0x1.3b2ab7181b757p-7);
  p = fma(p, f, 0x1.c6b08d7047e52p-5);
  p = fma(p, f, 0x1.ebfbdff823cedp-3);
  p = fma(p, f, 0x1.62e42fefa39efp-1);
  p = fma(p, f, 1.0);
  unsigned long long u, e;
  __builtin_memcpy(&u, &p, sizeof u);
  __builtin_memcpy(&e, &s, sizeof e);
  u += (e + 46) << 52;
  __builtin_memcpy(&p, &u, sizeof u);
  return p;
}
// 2^t for t <= 0 as a whole number of 2^-46: adding 2^52 rounds to a whole number, which then stands in the low bits
__device__ __forceinline__ unsigned long long exp2_fixed46(double t) {
  const double w = exp2_times_2to46(t) + 0x1p52;
  unsigned long long u;
  __builtin_memcpy(&u, &w, sizeof u);
  return u & 0xfffffffffffffull;
}

}  // namespace ec
