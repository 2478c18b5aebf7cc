// SwiGLU in float32 and conversions of its results, shared by the products that end in it.
#pragma once

#include "common.h"

namespace moepd {

// silu(g) * u.  With q = e^-|g|, silu is g / (1 + q), times q where g is negative: q never
// overflows, and 1 + q is between 1 and 2.  q as 2^(t + lo): the product's rounding error and
// log2 e's own, lo, would otherwise cost |g| ulp; with it, and the hardware's 2^x and
// reciprocal (1 ulp each), the result is within a few ulp.  Far below zero q and g q pass
// below the normal numbers (which the hardware's 2^x flushes), at -87 and -92, while u may
// bring the result back: there q carries a factor of 2^64 that 1 + q leaves out and u gives
// back, good down to gates of -131.  Past 256 q is 0 in any case.
// LIMIT: 0 also for a gate of minus infinity, where g q is NaN.
template <bool LIMIT = false>
__device__ __forceinline__ float swiglu_of(float g, float u) {
#pragma clang fp contract(off)  // t + 64 must start from the rounded t, whose error lo holds
  constexpr float kLog2e = 1.44269504f, kLog2eLow = 1.92596303e-8f, kLn2 = 0.693147181f;
  const float a = fminf(__builtin_fabsf(g), 256.f);
  const float t = -a * kLog2e;
  const float lo = __builtin_fmaf(-a, kLog2eLow, __builtin_fmaf(-a, kLog2e, -t));
  const bool deep = g < -44.f;
  const float k = deep ? 0x1p-64f : 1.f;
  const float e = __builtin_amdgcn_exp2f(t + (deep ? 64.f : 0.f));
  const float q = __builtin_fmaf(e, lo * kLn2, e);
  return (g < 0.f ? (LIMIT ? -a : g) * q : g) * __builtin_amdgcn_rcpf(__builtin_fmaf(q, k, 1.f)) * (u * k);
}

// From dh to the gradients in gate and up: dg = dh u s (1 + g (1 - s)), du = dh g s, with s =
// 1 / (1 + e^-g) and q as in swiglu_of (the compiler computes it once for both).  g q is 0 from where
// q is.  Of deep gates s, as q, carries a factor of 2^64, which u or dh gives
// back: good down to gates of -131.  The slope meets the larger of u and dh first, and the
// factor goes from the smaller one if that is above 1, else from the larger: nothing on the
// way to a normal dg passes below the normal numbers, or (factors above 5e36 aside) past the range.
__device__ __forceinline__ void swiglu_grad(float g, float u, float dh, float& dg, float& du) {
#pragma clang fp contract(off)
  constexpr float kLog2e = 1.44269504f, kLog2eLow = 1.92596303e-8f, kLn2 = 0.693147181f;
  const float a = fminf(__builtin_fabsf(g), 256.f);
  const float t = -a * kLog2e;
  const float lo = __builtin_fmaf(-a, kLog2eLow, __builtin_fmaf(-a, kLog2e, -t));
  const bool deep = g < -44.f;
  const float k = deep ? 0x1p-64f : 1.f;
  const float e = __builtin_amdgcn_exp2f(t + (deep ? 64.f : 0.f));
  const float q = __builtin_fmaf(e, lo * kLn2, e);
  const float near = __builtin_amdgcn_rcpf(__builtin_fmaf(q, k, 1.f)), far = q * near;  // s and 1 - s where g >= 0
  const float s = g < 0.f ? far : near;
  const float m = g < 0.f ? -a : g;
  const float slope = s * (1.f + (g > 256.f ? 0.f : m * (g < 0.f ? near : far)));  // far is 0 past 256; NaN stays
  const bool swap = __builtin_fabsf(dh) > __builtin_fabsf(u);
  const float large = swap ? dh : u, small = swap ? u : dh;
  const bool above = __builtin_fabsf(small) > 1.f;
  dg = large * (above ? 1.f : k) * slope * (small * (above ? k : 1.f));
  du = m * s * (dh * k);
}

// Two values to bf16, nearest even, packed.
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

}  // namespace moepd
