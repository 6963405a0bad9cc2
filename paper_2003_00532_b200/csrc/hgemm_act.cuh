// The activations of hgemm.h and their derivatives, in binary32. Device code only.
#pragma once

#include <cmath>

#include "../../include/hgemm.h"

namespace hgemm {

constexpr float INV_SQRT_2PI = 0.39894228040143268f;
constexpr float TANH_C = 0.79788456080286536f;   // sqrt(2 / pi)
constexpr float TANH_A = 0.044715f;
constexpr float LOG2E = 1.4426950408889634f;

// 1 / (1 + 2^x). The approximate exponential and reciprocal are off by a few units of 2^-22, far below
// the rounding of a 16-bit result; 1 + inf gives 0.
__device__ __forceinline__ float inv_1p_exp2(float x) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
  return r;
}
// ... and what it leaves of 1, without cancellation: 2^x / (1 + 2^x) where that is the smaller one.
__device__ __forceinline__ float inv_1p_exp2(float x, float& rest) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
  rest = e < 1.f ? e * r : 1.f - r;
  return r;
}
// The normal distribution function of z, and exp(-z^2 / 2). With y = |z|: Phi(-y) = exp(-y^2 / 2) q(1 / (1 + 0.4 y)), where q is
// the polynomial of degree 8 whose largest relative error over 0 <= y <= 13.3 is smallest (7e-8; fitted by exchange of the
// extrema), beyond which the exponential is 0. In binary32 the relative error is 3.3e-7 near 0 and grows with the exponent's rounding,
// y^2 2^-24, to 1e-5 at the far end: 1 + erf(z / sqrt 2) instead loses all digits of Phi by z = -5.5.
__device__ __forceinline__ float normal_cdf(float z, float& e) {
  float t;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(-0.5f * LOG2E * z * z));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(fmaf(0.4f, fabsf(z), 1.f)));
  float q = -0.04007509283295739f;
  q = fmaf(q, t, 0.2026474537159677f);
  q = fmaf(q, t, -0.3773960009590717f);
  q = fmaf(q, t, 0.25465877506026896f);
  q = fmaf(q, t, -0.01456649474708183f);
  q = fmaf(q, t, 0.15920147825351733f);
  q = fmaf(q, t, 0.1556192953768003f);
  q = fmaf(q, t, 0.15992345802992847f);
  q = fmaf(q, t, -1.2905281525769618e-05f);
  const float tail = e * q;
  return z > 0.f ? 1.f - tail : tail;
}
// act(z) for a result that is rounded to 16 bits.
template <int ACT>
__device__ __forceinline__ float act_fwd(float z) {
  if (ACT == HGEMM_ACT_RELU) return z <= 0.f ? 0.f : z;  // NaN stays NaN
  if (ACT == HGEMM_ACT_GELU) {
    float e;
    return z * normal_cdf(z, e);
  }
  // (1 + tanh(p)) / 2 = 1 / (1 + exp(-2 p))
  if (ACT == HGEMM_ACT_GELU_TANH) return z * inv_1p_exp2(z * (-2.f * LOG2E * TANH_C - 2.f * LOG2E * TANH_C * TANH_A * z * z));
  if (ACT == HGEMM_ACT_SILU) return z * inv_1p_exp2(-LOG2E * z);
  return z;
}

// act(z) and act'(z). The value is within 2^-14 of its size (a few units of 2^-22 for |z| < 3), the derivative within that of the
// sum of its two terms' magnitudes: the values are rounded to 16 bits, or summed over rows in binary32.
template <int ACT>
__device__ __forceinline__ void act_both(float z, float& f, float& df) {
  if (ACT == HGEMM_ACT_RELU) {
    f = z <= 0.f ? 0.f : z;
    df = z > 0.f ? 1.f : 0.f;
  } else if (ACT == HGEMM_ACT_GELU) {
    float e;
    const float cdf = normal_cdf(z, e);
    f = z * cdf;
    df = cdf + z * INV_SQRT_2PI * e;
  } else if (ACT == HGEMM_ACT_GELU_TANH) {
    float rest;
    const float q = inv_1p_exp2(z * (-2.f * LOG2E * TANH_C - 2.f * LOG2E * TANH_C * TANH_A * z * z), rest);
    f = z * q;
    const float t = f * rest;  // 0 far out, where z * z may be infinite
    df = t == 0.f ? q : q + t * (2.f * TANH_C) * (1.f + 3.f * TANH_A * z * z);
  } else if (ACT == HGEMM_ACT_SILU) {
    float rest;
    const float q = inv_1p_exp2(-LOG2E * z, rest);
    f = z * q;
    df = q + f * rest;
  } else {
    f = z;
    df = 1.f;
  }
}

}  // namespace hgemm
