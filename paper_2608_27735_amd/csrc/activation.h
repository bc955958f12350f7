// activation.h -- the gated block's activations and their derivatives.
#pragma once

#include "abcd_internal.h"

namespace abcd {

// By the hardware's base-2 exponential and reciprocal.
__device__ __forceinline__ float sigmoid(float g) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896341f * g));
}

// a(g) and a'(g). The activation is the same for every lane.
__device__ __forceinline__ float activate(float g, int act, float& slope) {
  if (act == ABCD_ACT_SILU) {
    const float s = sigmoid(g);
    slope = s * (1.0f + g * (1.0f - s));
    return g * s;
  }
  if (act == ABCD_ACT_GELU) {
    const float c = 0.5f + 0.5f * erff(0.70710678118654752f * g);
    slope = c + g * 0.39894228040143268f * __builtin_amdgcn_exp2f(-0.72134752044448170f * g * g);
    return g * c;
  }
  slope = g > 0.0f ? 1.0f : 0.0f;
  return fmaxf(g, 0.0f);
}

}  // namespace abcd
