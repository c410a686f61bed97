// The normal distribution function, for the GELU gate.
#pragma once

namespace asd {
namespace {

// (Phi(g), exp(-g^2 / 2)).  With x = |g| / sqrt(2) and t = 1 / (1 + p x), erfc(x) exp(x^2) is smooth in t over 0 < t <= 1 and
// vanishes with it:  Phi(-|g|) = t (a0 + a1 t + .. + a7 t^7) exp(-x^2).  The coefficients are a weighted least-squares fit, with the
// weights moved to where the error is largest until it is level, of the RELATIVE error for x <= 10: 9.8e-8 at p = 0.43.  (The
// classical form with five coefficients keeps an absolute error of 7.5e-8, which is 5e-4 of Phi at g = -4 and 6e-3 at -7: too
// coarse for a row all of whose gates are there.)  What 32 bits add is mostly the rounding of the exponent: the whole is within
// (8 + g^2) 2^-23 of Phi, to g = -13, beyond which the exponential leaves the range and Phi is 0.  It has no branch, and its
// exponential is the one that the gate's derivative needs.
__device__ __forceinline__ float2 normal_cdf(float g) {
  float t, e;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(fmaf(fabsf(g), 0.43f * 0.7071067811865476f, 1.f)));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(g * g * -0.7213475204444817f));
  float p = fmaf(t, 0.03657291147f, -0.1540478234f);
  p = fmaf(t, p, 0.1899436529f);
  p = fmaf(t, p, -0.04115215831f);
  p = fmaf(t, p, 0.1225403397f);
  p = fmaf(t, p, 0.1027362494f);
  p = fmaf(t, p, 0.1221469137f);
  p = fmaf(t, p, 0.1212599082f);
  const float tail = p * t * e;
  return make_float2(g < 0.f ? tail : 1.f - tail, e);
}

}  // namespace
}  // namespace asd
