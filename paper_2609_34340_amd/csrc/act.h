// Activations of the dense products and their derivatives, in 32 bits.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "internal.h"

namespace vp {

// 1 / (1 + exp(-v)), to a few units of the last place for |v| in the tens (the product with log2 e is rounded).
__device__ inline float logistic(float v) {
#ifdef __HIP_DEVICE_COMPILE__
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -1.44269504089f));
#else
  return v;
#endif
}
// And 1 less it, as exact.  exp(-v) ends at 2^120 here (a NaN stays), so that its product with the reciprocal stays 1.
struct Logistic { float s, rest; };
__device__ inline Logistic logistic_pair(float v) {
#ifdef __HIP_DEVICE_COMPILE__
  float e = __builtin_amdgcn_exp2f(v * -1.44269504089f);
  e = e > 0x1p120f ? 0x1p120f : e;
  const float s = __builtin_amdgcn_rcpf(1.0f + e);
  return {s, e * s};
#else
  return {v, v};
#endif
}

// The normal distribution Phi(v) and exp(-v^2 / 2).  With t = 1 / (1 + 0.265 |v|), the tail Phi(-|v|) exp(v^2 / 2), which
// falls from 1/2 like 1 / |v|, is a polynomial in t without a constant: its coefficients are a fit of the relative error
// over |v| <= 14 (1.4e-8), and 32 bits evaluate it to 4e-7 of the tail where |v| < 1, 1e-6 below 4; the tail of large |v|
// keeps its relative size, which a difference of 1 and erf loses.
struct Normal { float cdf, bell; };
__device__ inline Normal normal(float v) {
#ifdef __HIP_DEVICE_COMPILE__
  const float a = __builtin_fabsf(v);
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.265f, a, 1.0f));
  float q = 0.030624598264694214f;
  q = __builtin_fmaf(q, t, -0.14330121874809265f);
  q = __builtin_fmaf(q, t, 0.21595148742198944f);
  q = __builtin_fmaf(q, t, -0.1142875924706459f);
  q = __builtin_fmaf(q, t, 0.13655565679073334f);
  q = __builtin_fmaf(q, t, 0.060894742608070374f);
  q = __builtin_fmaf(q, t, 0.10255515575408936f);
  q = __builtin_fmaf(q, t, 0.10526677221059799f);
  q = __builtin_fmaf(q, t, 0.10574039816856384f);
  const float bell = __builtin_amdgcn_exp2f(a * a * -0.72134752044f);
  const float tail = q * t * bell;
  return {v > 0.0f ? 1.0f - tail : tail, bell};
#else
  return {v, v};
#endif
}

// The argument of the tanh form's logistic, and its derivative.
constexpr float kTanhSlope = 1.59576912161f, kTanhCube = 0.044715f;   // 2 sqrt(2 / pi)

template <int ACT> __device__ inline float activation(float v) {
  if constexpr (ACT == VP_ACT_RELU) return v < 0.0f ? 0.0f : v;   // NaN stays
  if constexpr (ACT == VP_ACT_SILU) return v * logistic(v);
  if constexpr (ACT == VP_ACT_GELU) return v * normal(v).cdf;
  if constexpr (ACT == VP_ACT_GELU_TANH) return v * logistic(kTanhSlope * v * __builtin_fmaf(kTanhCube * v, v, 1.0f));
  return v;
}

// v, no further from 0 than `most` (one instruction, which loses a NaN).
__device__ inline float within(float v, float most) {
#ifdef __HIP_DEVICE_COMPILE__
  return __builtin_amdgcn_fmed3f(v, -most, most);
#else
  return v;
#endif
}

// gradient * activation'(v).  Past 100 and 20 the factors of the logistic and the bell are those there, and the derivatives
// 1, or less than 1e-32: below, the factor would outgrow what the logistic's end at 2^-120 leaves; above, it would be an
// infinity times 0, v^2 from 5e19 on and v itself where a kept 16-bit value rounded to infinity.  A NaN comes from the
// logistic or the distribution, which take v itself.
template <int ACT> __device__ inline float through(float gradient, float v) {
  if constexpr (ACT == VP_ACT_RELU) return v <= 0.0f ? 0.0f : gradient;
  if constexpr (ACT == VP_ACT_SILU) {
    const Logistic q = logistic_pair(v);
    return gradient * q.s * __builtin_fmaf(within(v, 100.0f), q.rest, 1.0f);
  }
  if constexpr (ACT == VP_ACT_GELU) {
    const Normal n = normal(v);
    return gradient * __builtin_fmaf(within(v, 20.0f) * 0.398942280401f, n.bell, n.cdf);
  }
  if constexpr (ACT == VP_ACT_GELU_TANH) {
    const Logistic q = logistic_pair(kTanhSlope * v * __builtin_fmaf(kTanhCube * v, v, 1.0f));
    v = within(v, 20.0f);
    return gradient * q.s * __builtin_fmaf(v * q.rest, kTanhSlope * __builtin_fmaf(3.0f * kTanhCube * v, v, 1.0f), 1.0f);
  }
  return gradient;
}

// Calls f with the activation as a type.
template <typename F> __host__ __device__ inline void with_act(int act, F f) {
  switch (act) {
    case VP_ACT_RELU: f(std::integral_constant<int, VP_ACT_RELU>{}); break;
    case VP_ACT_SILU: f(std::integral_constant<int, VP_ACT_SILU>{}); break;
    case VP_ACT_GELU: f(std::integral_constant<int, VP_ACT_GELU>{}); break;
    case VP_ACT_GELU_TANH: f(std::integral_constant<int, VP_ACT_GELU_TANH>{}); break;
    default: f(std::integral_constant<int, VP_ACT_NONE>{});
  }
}

}  // namespace vp
