// Activations of the stand-alone operators (nf_act): value and derivative at the pre-activation z.
#pragma once
#include <type_traits>

#include "nf_internal.h"

static inline bool nf_act_ok(int act) { return act >= NF_ACT_NONE && act <= NF_ACT_GELU; }

// 1 / (1 + e^-z).  With bf16 storage the approximate exponential and reciprocal are used: their error, about 2^-22 (1 + |z|) relative,
// is far below the 2^-9 of the stored result.  fp32 storage keeps the full-precision functions.
template <typename T>
__device__ __forceinline__ float nf_sigmoid(float z) {
  if constexpr (std::is_same<T, float>::value) return 1.f / (1.f + expf(-z));
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.4426950408889634f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));  // 0 where e is infinite
  return r;
}
// Standard normal distribution function by erfc, which keeps the small values of the left tail.  bf16 storage: erfc of a positive argument x as
// t exp(p(t) - x^2), t = 1 / (1 + x / 2), with the Chebyshev fit p of Press et al., Numerical Recipes (function erfcc; fractional error
// below 1.2e-7, to which fp32 adds about 2^-23 (1 + x^2)); a quarter of the instructions of the full-precision function.
template <typename T>
__device__ __forceinline__ float nf_normal_cdf(float z) {
  if constexpr (std::is_same<T, float>::value) return 0.5f * erfcf(z * -0.70710678118654752f);
  const float x = fabsf(z) * 0.70710678118654752f;
  float t, e;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(fmaf(0.5f, x, 1.f)));
  float p = 0.17087277f;
  p = fmaf(p, t, -0.82215223f);
  p = fmaf(p, t, 1.48851587f);
  p = fmaf(p, t, -1.13520398f);
  p = fmaf(p, t, 0.27886807f);
  p = fmaf(p, t, -0.18628806f);
  p = fmaf(p, t, 0.09678418f);
  p = fmaf(p, t, 0.37409196f);
  p = fmaf(p, t, 1.00002368f);
  p = fmaf(p, t, -1.26551223f);
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fmaf(-x, x, p) * 1.4426950408889634f));
  e *= 0.5f * t;
  return z < 0.f ? e : 1.f - e;
}
__device__ __forceinline__ float nf_relu(float z) {  // a NaN stays one
  float r;
  asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(z));
  return r;
}
template <typename T>
__device__ __forceinline__ float nf_act_value(float z, int act) {
  if (act == NF_ACT_RELU) return nf_relu(z);
  if (act == NF_ACT_SILU) return z * nf_sigmoid<T>(z);
  if (act == NF_ACT_GELU) return z * nf_normal_cdf<T>(z);
  return z;
}
template <typename T>
__device__ __forceinline__ float nf_act_grad(float z, int act) {
  if (act == NF_ACT_RELU) return z > 0.f ? 1.f : 0.f;
  if (act == NF_ACT_SILU) {
    const float s = nf_sigmoid<T>(z);
    return fmaf(z * s, 1.f - s, s);
  }
  if (act == NF_ACT_GELU) return fmaf(z * 0.39894228040143268f, std::is_same<T, float>::value ? expf(-0.5f * z * z) : __expf(-0.5f * z * z), nf_normal_cdf<T>(z));
  return 1.f;
}
// dy act'(z); behind a closed ReLU 0 whatever dy was
template <typename T>
__device__ __forceinline__ float nf_act_dz(float z, float dy, int act) {
  if (act == NF_ACT_NONE) return dy;
  if (act == NF_ACT_RELU) return z > 0.f ? dy : 0.f;
  return dy * nf_act_grad<T>(z, act);
}
