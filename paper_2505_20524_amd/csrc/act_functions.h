// The activations in binary32, for their producers and for their gradients.
#pragma once
#include "common.h"

namespace {

enum { ACT_XIELU = 0, ACT_GELU = 1, ACT_TANH = 2 };

// binary32 evaluation.  Both exponential-type functions are built on the hardware base-2 exponential (one unit
// in the last place) away from the origin and on a short polynomial whose leading term is exact near it, where
// the exponential form would cancel (tables generated by tanh_expm1_coeffs.py); the two forms are both
// evaluated and one is selected, so the code is branch-free.  The results are within 2^-21 relative of the
// exact values, a third of the instructions of the library routines.
#include "tanh_expm1_coeffs.inc"
// e^x - 1 for x <= 0
FOG_DEVICE float expm1_neg(float x) {
  float q = kExpm1Poly[4];
#pragma unroll
  for (int i = 3; i >= 0; --i) q = __builtin_fmaf(q, x, kExpm1Poly[i]);
  const float near = x * __builtin_fmaf(x, q, 1.0f);                                     // x + x^2 Q(x); keeps the sign of a zero
  const float far = __builtin_amdgcn_exp2f(x * 1.44269504088896340736f) - 1.0f;
  return x > kExpm1Switch ? near : far;
}
FOG_DEVICE float tanh_fast(float z) {
  const float w = z * z;
  float p = kTanhPoly[3];
#pragma unroll
  for (int i = 2; i >= 0; --i) p = __builtin_fmaf(p, w, kTanhPoly[i]);
  const float near = z * __builtin_fmaf(w, p, 1.0f);                                     // z + z^3 P(z^2); keeps the sign of a zero
  const float e = __builtin_amdgcn_exp2f(fabsf(z) * 2.88539008177792681472f);            // e^(2 |z|); overflows to +inf, whose reciprocal is 0
  const float far = __builtin_copysignf(__builtin_fmaf(-2.0f, __builtin_amdgcn_rcpf(e + 1.0f), 1.0f), z);
  return fabsf(z) < kTanhSwitch ? near : far;                                            // a NaN takes the second form and stays NaN
}

// The remaining operations of xIELU are single multiplies and adds, so the result is within a few units in the
// last place of the exact value wherever the two terms of the negative branch do not cancel.
FOG_DEVICE float xielu(float x, float ap, float an) {
  const float pos = __builtin_fmaf(ap * x, x, 0.5f * x);
  const float neg = __builtin_fmaf(an, expm1_neg(x), (0.5f - an) * x);   // for x > 0 an unused value (possibly inf or NaN)
  return x > 0.0f ? pos : neg;
}

// x Phi(x).  With t = |x|, Phi(-t) = exp(-t^2 / 2) R(t), R a scaled Mills ratio: (t + k) R(t) is a degree-10
// polynomial in u = (t - k) / (t + k) (table generated by gelu_coeffs.py, 5e-8 relative), so the tail costs
// one reciprocal, ten fused multiply-adds and one exponential, without branches.  x <= 0: -t Phi(-t), which
// keeps its relative accuracy far into the tail (error about t^2 2^-24 from the rounded exponent);
// x > 0: x - t Phi(-t), no cancellation since Phi(-t) <= 1/2.  Beyond |x| = 14 the tail is below the
// smallest normal binary32 number and is taken as 0.
#include "gelu_coeffs.inc"
FOG_DEVICE float gelu_tail(float t) {                                         // Phi(-t), 0 <= t <= 14
  const float rinv = __builtin_amdgcn_rcpf(t + kTailK);
  const float u = (t - kTailK) * rinv;
  float p = kTailPoly[10];
#pragma unroll
  for (int i = 9; i >= 0; --i) p = __builtin_fmaf(p, u, kTailPoly[i]);
  const float e = __builtin_amdgcn_exp2f(t * t * -0.72134752044448170368f);   // exp(-t^2 / 2)
  return e * (p * rinv);
}
FOG_DEVICE float gelu(float x) {
  const float t = fminf(fabsf(x), 14.0f);
  const float tt = t * gelu_tail(t);
  return x < 0.0f ? -tt : x - tt;   // a zero keeps its sign
}

template <int ACT>
FOG_DEVICE float act(float x, float p0, float p1) {
  if (ACT == ACT_XIELU) return xielu(x, p0, p1);
  if (ACT == ACT_GELU) return gelu(x);
  return tanh_fast(p0 * x);
}

}  // namespace
