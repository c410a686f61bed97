// The normal distribution function, for the GELU gate.
#pragma once

namespace asd {
namespace {

// (Phi(g), exp(-g^2 / 2)) by the rational approximation of Hastings (Abramowitz and Stegun, Handbook of Mathematical Functions,
// 7.1.26):  erfc(x) = (a1 t + .. + a5 t^5) exp(-x^2),  t = 1 / (1 + p x),  x >= 0, off by at most 1.5e-7, so Phi by 7.5e-8 and
// the roundings of 32 bits.  It has no branch, and its exponential is the one that the gate's derivative needs.
__device__ __forceinline__ float2 normal_cdf(float g) {
  float t, e;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(fmaf(fabsf(g), 0.3275911f * 0.7071067811865476f, 1.f)));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(g * g * -0.7213475204444817f));
  float p = fmaf(t, 1.061405429f, -1.453152027f);
  p = fmaf(t, p, 1.421413741f);
  p = fmaf(t, p, -0.284496736f);
  p = fmaf(t, p, 0.254829592f);
  const float tail = 0.5f * p * t * e;
  return make_float2(g < 0.f ? tail : 1.f - tail, e);
}

}  // namespace
}  // namespace asd
