// gelu.h -- GELU(z) = z Phi(z) and its derivative in single precision.
#pragma once
#include <hip/hip_runtime.h>

namespace afno {

// GELU(z) = z Phi(z).  The lower tail u = Phi(-|z|) = t Q(t) exp(-z^2 / 2), t = 1 / (1 + 0.3 |z|),
// with Q a degree-7 fit to erfcx(|z| / sqrt 2) / (2 t) on |z| <= 9 (least squares reweighted to a
// minimax relative error of 5e-8); then z - |z| u above zero and z u below.  Against float64 the
// result, in single precision, is within 7e-7 of its own size for z > -3 and 7e-6 from there to
// -12.9 (a model in float32 of every step: 4.4e-7 and 6.7e-6; the fit reaches past its 9), and within
// 2e-37 below, where the exponential leaves the normal numbers; 0.5 z (1 + erf) has 1e-7 to 2e-7
// for |z| < 1, and below loses all digits by z = -6 to the subtraction.  About 25 issue slots a
// value where erff takes over 60: the epilogue's values are the exposed part of the block's first
// product (64,800 x 3072 x 768: 426 us with erff, 387 with this, 320 without any).  |z| is bounded
// in the tail only (z = +inf gives +inf; -inf and NaN give NaN, as z Phi(z) does).
__device__ __forceinline__ float gelu(float z) {
  const float a = fminf(fabsf(z), 16.f);
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3f, a, 1.f));
  float q = 0.037535712f;
  q = __builtin_fmaf(q, t, -0.16501968f);
  q = __builtin_fmaf(q, t, 0.21997128f);
  q = __builtin_fmaf(q, t, -0.06640263f);
  q = __builtin_fmaf(q, t, 0.13542020f);
  q = __builtin_fmaf(q, t, 0.097783938f);
  q = __builtin_fmaf(q, t, 0.1211057f);
  q = __builtin_fmaf(q, t, 0.11960549f);
  const float e = __builtin_amdgcn_exp2f(a * a * -0.72134752f);  // exp(-a^2 / 2)
  const float u = t * q * e;
  return z > 0.f ? __builtin_fmaf(-a, u, z) : z * u;
}

// GELU(z) in two thirds of the issue slots, for results of few bits: the lower tail's logarithm to base 2 as a polynomial of
// degree 8 on |z| <= 9 (least squares reweighted to a minimax error of 6.0e-6 of the tail), which takes no reciprocal; then
// max(z, 0) - |z| u on both sides.  Against float64, by a float32 model, within 6.8e-6 of its own size for z > -3,
// 1.3e-5 from there to -9 and 1.2e-18 below.  +inf gives +inf, -inf gives -1e-18, NaN NaN.
__device__ __forceinline__ float gelu_short(float z) {
  const float a = fminf(fabsf(z), 9.f);
  float q = 7.463253e-08f;
  q = __builtin_fmaf(q, a, -3.6557733e-06f);
  q = __builtin_fmaf(q, a, 7.9437545e-05f);
  q = __builtin_fmaf(q, a, -0.0010200484f);
  q = __builtin_fmaf(q, a, 0.008750868f);
  q = __builtin_fmaf(q, a, -0.054304663f);
  q = __builtin_fmaf(q, a, -0.45824152f);
  q = __builtin_fmaf(q, a, -1.151295f);
  q = __builtin_fmaf(q, a, -0.9999966f);
  return __builtin_fmaf(-a, __builtin_amdgcn_exp2f(q), __builtin_elementwise_maximum(z, 0.f));
}

// GELU'(z) = Phi(z) + z phi(z) with the tail and the exponential of gelu(): Phi is u below zero and
// 1 - u above.  Against float64 within 2.1e-7 in a model in float32 of every step, 3.2e-7 with the
// reciprocal and the exponential a last place off (the two terms cancel near z = -0.75, so there is no
// bound relative to the value).  +inf gives 1, -inf 0, NaN NaN.
__device__ __forceinline__ float gelu_grad(float z) {
  const float a = __builtin_elementwise_minimum(fabsf(z), 16.f);  // NaN stays
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3f, a, 1.f));
  float q = 0.037535712f;
  q = __builtin_fmaf(q, t, -0.16501968f);
  q = __builtin_fmaf(q, t, 0.21997128f);
  q = __builtin_fmaf(q, t, -0.06640263f);
  q = __builtin_fmaf(q, t, 0.13542020f);
  q = __builtin_fmaf(q, t, 0.097783938f);
  q = __builtin_fmaf(q, t, 0.1211057f);
  q = __builtin_fmaf(q, t, 0.11960549f);
  const float e = __builtin_amdgcn_exp2f(a * a * -0.72134752f);  // exp(-a^2 / 2)
  // a phi(a) - u: below zero with its sign turned, above 1 and this
  const float d = e * __builtin_fmaf(-t, q, a * 0.39894228f);
  return z > 0.f ? 1.f + d : -d;
}

}  // namespace afno
