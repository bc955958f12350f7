// activation.h -- the gated block's activations and their derivatives.
#pragma once

#include <type_traits>

#include "abcd_internal.h"

namespace abcd {

// By the hardware's base-2 exponential and reciprocal.
__device__ __forceinline__ float sigmoid(float g) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896341f * g));
}

// a(g) and a'(g). The activation is a template argument of the kernels: with a
// branch at every element no two elements' exponentials overlap.
// kShort: for what is rounded to 16 bits, the error function by Abramowitz and Stegun's
// 7.1.26, within 1.5e-7 of it: a polynomial of 1 / (1 + p |x|) times the exponential
// that the derivative needs too.
template <int kAct, bool kShort>
__device__ __forceinline__ float activate(float g, float& slope) {
  if (kAct == ABCD_ACT_SILU) {
    const float s = sigmoid(g), v = g * s;
    slope = fmaf(v, 1.0f - s, s);
    return v;
  }
  if (kAct == ABCD_ACT_GELU) {
    const float e = __builtin_amdgcn_exp2f(-0.72134752044448170f * g * g);  // e^(-g^2 / 2)
    float c;  // the normal distribution
    if (kShort) {
      const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f * 0.70710678118654752f, fabsf(g), 1.0f));
      float s = fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f);
      s = fmaf(t, s, 0.5f * 1.421413741f);
      s = fmaf(t, s, 0.5f * -0.284496736f);
      s = fmaf(t, s, 0.5f * 0.254829592f) * t * e;
      c = g < 0.0f ? s : 1.0f - s;
    } else {
      c = 0.5f + 0.5f * erff(0.70710678118654752f * g);
    }
    slope = fmaf(g * 0.39894228040143268f, e, c);
    return g * c;
  }
  slope = g > 0.0f ? 1.0f : 0.0f;
  return fmaxf(g, 0.0f);
}

// Calls f with act as a constant.
template <typename F>
int32_t with_act(int act, F f) {
  if (act == ABCD_ACT_SILU) return f(std::integral_constant<int, ABCD_ACT_SILU>{});
  if (act == ABCD_ACT_GELU) return f(std::integral_constant<int, ABCD_ACT_GELU>{});
  return f(std::integral_constant<int, ABCD_ACT_RELU>{});
}

}  // namespace abcd
