// The activations of hgemm.h and their derivatives, in binary32. Device code only.
#pragma once

#include <cmath>

#include "../../include/hgemm.h"

namespace hgemm {

constexpr float SQRT_HALF = 0.70710678118654752f;
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
// act(z) for a result that is rounded to 16 bits.
template <int ACT>
__device__ __forceinline__ float act_fwd(float z) {
  if (ACT == HGEMM_ACT_RELU) return z <= 0.f ? 0.f : z;  // NaN stays NaN
  if (ACT == HGEMM_ACT_GELU) return 0.5f * z * (1.f + erff(z * SQRT_HALF));
  // (1 + tanh(p)) / 2 = 1 / (1 + exp(-2 p))
  if (ACT == HGEMM_ACT_GELU_TANH) return z * inv_1p_exp2(z * (-2.f * LOG2E * TANH_C - 2.f * LOG2E * TANH_C * TANH_A * z * z));
  if (ACT == HGEMM_ACT_SILU) return z * inv_1p_exp2(-LOG2E * z);
  return z;
}

// act(z) and act'(z), within a few units of 2^-22 of their size: the values are rounded to 16 bits, or summed over
// rows in binary32, where such errors average out below the rounding of the sum.
template <int ACT>
__device__ __forceinline__ void act_both(float z, float& f, float& df) {
  if (ACT == HGEMM_ACT_RELU) {
    f = z <= 0.f ? 0.f : z;
    df = z > 0.f ? 1.f : 0.f;
  } else if (ACT == HGEMM_ACT_GELU) {
    const float cdf = 0.5f * (1.f + erff(z * SQRT_HALF));
    f = z * cdf;
    df = cdf + z * INV_SQRT_2PI * expf(-0.5f * z * z);
  } else if (ACT == HGEMM_ACT_GELU_TANH) {
    const float q = inv_1p_exp2(z * (-2.f * LOG2E * TANH_C - 2.f * LOG2E * TANH_C * TANH_A * z * z));
    f = z * q;
    const float t = f * (1.f - q);  // 0 far out, where z * z may be infinite
    df = t == 0.f ? q : q + t * (2.f * TANH_C) * (1.f + 3.f * TANH_A * z * z);
  } else if (ACT == HGEMM_ACT_SILU) {
    const float q = inv_1p_exp2(-LOG2E * z);
    f = z * q;
    df = q + f * (1.f - q);
  } else {
    f = z;
    df = 1.f;
  }
}

}  // namespace hgemm
