// The gated layer's activations: value and derivative in float32.
#pragma once

#include "train_kernels.h"

namespace fqt {

// s(z) = 1 / (1 + exp(-z)).  exp2 and the reciprocal are the hardware's, one
// unit in the last place each; the exponent's rounding makes it |z| 2^-24
// relative where s is small.
__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504088896341f));
}

template <fqt_act ACT>
__device__ __forceinline__ void activate(float a, float& value, float& slope) {
  if constexpr (ACT == FQT_RELU) {
    value = a < 0.0f ? 0.0f : a;
    slope = a > 0.0f ? 1.0f : 0.0f;
  } else if constexpr (ACT == FQT_SILU) {
    const float s = sigmoid(a);
    value = a * s;
    slope = fmaf(value, 1.0f - s, s);
  } else {
    // a s(z) with z = 2 u; beyond |a| = 16 s(z) is 0 or 1 in float32, and z stays finite
    const float t = __builtin_amdgcn_fmed3f(a, -16.0f, 16.0f), t2 = t * t;
    constexpr float C1 = 1.59576912160573071f, C3 = 0.0713548162726009f;  // 2 sqrt(2 / pi), times 0.044715
    const float s = sigmoid(t * fmaf(C3, t2, C1));
    value = a * s;
    slope = fmaf(value * (1.0f - s), fmaf(3.0f * C3, t2, C1), s);
  }
}

// Calls f with the activation as a constant.
template <class F>
__device__ __forceinline__ void with_act(fqt_act act, const F& f) {
  if (act == FQT_SILU)
    f(std::integral_constant<fqt_act, FQT_SILU>{});
  else if (act == FQT_GELU_TANH)
    f(std::integral_constant<fqt_act, FQT_GELU_TANH>{});
  else
    f(std::integral_constant<fqt_act, FQT_RELU>{});
}

}  // namespace fqt
