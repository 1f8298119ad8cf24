// Maxima of scores that come out of matrix products, for the attention kernels.
#pragma once
#include "k_common.h"

namespace ec {

__device__ __forceinline__ bf16x8 u4_as_bf16x8(uint4 v) {
  union { uint4 u; bf16x8 b; } c;
  c.u = v;
  return c.b;
}

// The larger of two, a number before a NaN.  (fmaxf quiets what comes from a matrix product or a lane swap with an
// instruction of its own for each operand; the median with infinity takes them as they are.)
__device__ __forceinline__ float max_of(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, INFINITY); }
__device__ __forceinline__ float max_of_swap16(float x) {
  const unsigned u = __float_as_uint(x);
  auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return max_of(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_of_swap32(float x) {
  const unsigned u = __float_as_uint(x);
  auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return max_of(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// largest of a lane's 8 scores
__device__ __forceinline__ float max_of_8(const f32x4& a, const f32x4& b) {
  return max_of(max_of(max_of(a[0], a[1]), max_of(a[2], a[3])), max_of(max_of(b[0], b[1]), max_of(b[2], b[3])));
}

}  // namespace ec
