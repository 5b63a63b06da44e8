// The 4-bit cache: K and V as 4-bit floats (sign, 0 0.5 1 1.5 2 3 4 6) in blocks of 32 channels that share a power of
// two (mx_layout.h).
#pragma once
#include "common.h"
#include "mx_layout.h"

namespace hspec {
namespace {

// The key, of 16, that lane l of 16 takes into LDS: bits of l at places A, B, C, E.  A 16-byte write is done 8 lanes at a time
// over 128 bytes, so the keys of 8 lanes side by side differ in the bits that choose the place within those (with
// keys in order a quarter to a third of the LDS cycles are conflicts, so none, and prompts and 17 tokens take 2 % more on the
// same card).
template <int A, int B, int C, int E>
__device__ __forceinline__ int spread16(int l) {
  return (l & 1) << A | (l >> 1 & 1) << B | (l >> 2 & 1) << C | (l >> 3 & 1) << E;
}

// 8 channels of a word as bf16 and as fp32: exact (the conversions take 2^(s - 127) as the exponent of a float, 0 and 255
// too).
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ bf16x8 mx_widen(unsigned code, unsigned scale) {
  const float s = __uint_as_float(scale << 23);
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ void mx_widen(unsigned code, unsigned scale, f32x4& lo, f32x4& hi) {
  const float s = __uint_as_float(scale << 23);
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 1);
  const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 3);
  lo = f32x4{a[0], a[1], b[0], b[1]};
  hi = f32x4{c[0], c[1], d[0], d[1]};
}

// Scale byte of a block whose largest magnitude is `top` (finite): the smallest 2^e with top < 7 2^e, so that no value
// is cut by more than half a step of the next binade; from 2^-126 to 2^125, so that what is finite in 32 bits stays it.
// Only top's bits decide.
__device__ __forceinline__ unsigned mx_scale(float top) {
  const unsigned u = __float_as_uint(top);
  const int s = (int)(u >> 23) - 2 + ((u & 0x7fffff) >= 0x600000 ? 1 : 0);   // top = 1.m 2^(E - 127)
  return (unsigned)(s < 1 ? 1 : s > 252 ? 252 : s);
}
__device__ __forceinline__ unsigned mx_scale(double top) {
  const unsigned long long u = (unsigned long long)__double_as_longlong(top);
  const int s = (int)(u >> 52) - 1023 + 127 - 2 + ((u & 0xfffffffffffffULL) >= 0xc000000000000ULL ? 1 : 0);
  return (unsigned)(s < 1 ? 1 : s > 252 ? 252 : s);
}
// Code of y under the scale byte s: the nearest value, ties to the even code.  (Scaling by a power of two is exact, or
// the result is far below the first border.)
__device__ __forceinline__ unsigned mx_code(float y, unsigned s) {
  const float t = fabsf(y) * __uint_as_float((254u - s) << 23);
  const unsigned c = (t > 0.25f) + (t >= 0.75f) + (t > 1.25f) + (t >= 1.75f) + (t > 2.5f) + (t >= 3.5f) + (t > 5.f);
  return c | (__float_as_uint(y) >> 31 << 3);
}
__device__ __forceinline__ unsigned mx_code(double y, unsigned s) {
  const double t = fabs(y) * __longlong_as_double((long long)(1023 + 127 - (int)s) << 52);
  const unsigned c = (t > 0.25) + (t >= 0.75) + (t > 1.25) + (t >= 1.75) + (t > 2.5) + (t >= 3.5) + (t > 5.);
  return c | ((unsigned)(__double_as_longlong(y) >> 63) & 8u);
}

}  // namespace
}  // namespace hspec
