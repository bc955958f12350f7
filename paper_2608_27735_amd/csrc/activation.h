// activation.h -- the gated block's activations and their derivatives.
#pragma once

#include <type_traits>

#include "abcd_internal.h"

namespace abcd {

// By the hardware's base-2 exponential and reciprocal. Far below 0 its relative error is
// that of the exponent's rounding, 2^-24 |g|.
__device__ __forceinline__ float sigmoid(float g) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896341f * g));
}

// e^(-g^2 / 2). The exponent has no more digits after its point than its size leaves (at
// g = -12 three fewer than the result's), so what the rounding of g^2 and of its
// factor cuts off goes in as a factor of its own.
__device__ __forceinline__ float bell(float g) {
  constexpr double kHalf = 0.72134752044448170368;  // of a base-2 logarithm's unit
  constexpr float kC = (float)kHalf, kLow = (float)(kHalf - (double)kC);
  const float a = fminf(fabsf(g), 16.0f);  // 0 from 13.3 on
  const float sq = a * a, t = kC * sq;
  const float off = fmaf(kC, sq, -t) + fmaf(kC, fmaf(a, a, -sq), kLow * sq);
  const float e = __builtin_amdgcn_exp2f(-t);
  return fmaf(e, -0.69314718055994531f * off, e);
}

// a(g) and a'(g). The activation is a template argument of the kernels: with a
// branch at every element no two elements' exponentials overlap.
// The normal distribution below 0 is e^(-g^2 / 2) times a smooth function of |g|, and
// the derivative needs the exponential anyway; the other factor is t Q(t), with t =
// 1 / (1 + p |g|) in (0, 1], fitted to the scaled complementary error function with the
// least relative error, so that the tail keeps its digits: Q of degree 5, 4.8e-6, for
// what is rounded to 16 bits (kShort); else of degree 9, 3.3e-8 (with the
// roundings of fp32 3.2e-7, measured from g = -12 on). 65,536 rows of 96 x 256 x 59
// in fp32, forward: 92 us, with erff 97; a step of 1M rows of 64 x 128 x 64 in bfloat16
// 386, with erff 456.
template <int kAct, bool kShort>
__device__ __forceinline__ float activate(float g, float& slope) {
  if (kAct == ABCD_ACT_SILU) {
    const float s = sigmoid(g), v = g * s;
    slope = fmaf(v, 1.0f - s, s);
    return v;
  }
  if (kAct == ABCD_ACT_GELU) {
    const float e = kShort ? __builtin_amdgcn_exp2f(-0.72134752044448170f * g * g) : bell(g);
    float s;
    if (kShort) {
      const float t = __builtin_amdgcn_rcpf(fmaf(0.31f, fabsf(g), 1.0f));
      s = fmaf(t, -0.07391444f, 0.18040521f);
      s = fmaf(t, s, 0.01579695f);
      s = fmaf(t, s, 0.1334017f);
      s = fmaf(t, s, 0.12044814f);
      s = fmaf(t, s, 0.123860106f) * t * e;
    } else {
      const float t = __builtin_amdgcn_rcpf(fmaf(0.31819805f, fabsf(g), 1.0f));
      s = fmaf(t, -0.02069551f, 0.095343746f);
      s = fmaf(t, s, -0.15029088f);
      s = fmaf(t, s, 0.07120013f);
      s = fmaf(t, s, -0.011178771f);
      s = fmaf(t, s, 0.05997515f);
      s = fmaf(t, s, 0.08762608f);
      s = fmaf(t, s, 0.11413582f);
      s = fmaf(t, s, 0.12694158f);
      s = fmaf(t, s, 0.12694266f) * t * e;
    }
    const float c = g < 0.0f ? s : 1.0f - s;  // the normal distribution
    slope = fmaf(g * 0.39894228040143268f, e, c);
    return g * c;
  }
  const float v = g < 0.0f ? 0.0f : g;  // a NaN stays one, and so does its slope
  slope = g > 0.0f ? 1.0f : v;
  return v;
}

// Calls f with act as a constant.
template <typename F>
int32_t with_act(int act, F f) {
  if (act == ABCD_ACT_SILU) return f(std::integral_constant<int, ABCD_ACT_SILU>{});
  if (act == ABCD_ACT_GELU) return f(std::integral_constant<int, ABCD_ACT_GELU>{});
  return f(std::integral_constant<int, ABCD_ACT_RELU>{});
}

}  // namespace abcd
