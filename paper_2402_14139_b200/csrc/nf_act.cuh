// Activations of the stand-alone operators (nf_act): value and derivative at the pre-activation z.
#pragma once
#include <type_traits>

#include "nf_internal.h"

static inline bool nf_act_ok(int act) { return act >= NF_ACT_NONE && act <= NF_ACT_GELU; }

// 1 / (1 + e^-z).  With bf16 storage the fast exponential and division are used: their error, about 2^-21 (1 + |z|), is far below
// the 2^-9 of the stored result.  fp32 storage keeps the full-precision functions.
template <typename T>
__device__ __forceinline__ float nf_sigmoid(float z) {
  if constexpr (std::is_same<T, float>::value) return 1.f / (1.f + expf(-z));
  return __fdividef(1.f, 1.f + __expf(fminf(-z, 80.f)));  // the fast division returns 0 for divisors above 2^126: e^80 stays below
}
// Standard normal distribution function by erfc, which keeps the small values of the left tail
__device__ __forceinline__ float nf_normal_cdf(float z) { return 0.5f * erfcf(z * -0.70710678118654752f); }

template <typename T>
__device__ __forceinline__ float nf_act_value(float z, int act) {
  if (act == NF_ACT_RELU) return z < 0.f ? 0.f : z;  // a NaN stays one
  if (act == NF_ACT_SILU) return z * nf_sigmoid<T>(z);
  if (act == NF_ACT_GELU) return z * nf_normal_cdf(z);
  return z;
}
template <typename T>
__device__ __forceinline__ float nf_act_grad(float z, int act) {
  if (act == NF_ACT_RELU) return z > 0.f ? 1.f : 0.f;
  if (act == NF_ACT_SILU) {
    const float s = nf_sigmoid<T>(z);
    return fmaf(z * s, 1.f - s, s);
  }
  if (act == NF_ACT_GELU) return fmaf(z * 0.39894228040143268f, expf(-0.5f * z * z), nf_normal_cdf(z));
  return 1.f;
}
