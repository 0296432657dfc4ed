// The activations of the gated layers, with their derivatives.
#pragma once
#include <type_traits>

#include "float_types.h"

namespace bnn {

// The normal distribution's function, and exp(-z^2 / 2).  Of a = |z| the tail is exp(-a^2 / 2) t P(t), t = 1 / (1 + 0.345 a): P is fitted
// to exp(a^2 / 2) (1 - erf(a / sqrt 2)) / 2 on 0 .. 14, least squares with weights moved to where the relative error is largest, 2e-8 at
// the end.  With what the squares and the exponent lose put back, a value below zero is off by 6 * 2^-24 of itself, as far as fp32's
// normal numbers reach (1 + erf there loses all of its digits).  Beyond 16 it is 0.  (fp16, 1000 x 1024 to 2321: 19.2 us, 18.7 with a
// formula good to 1.5e-7 of 1 and not of the value, 22.5 with erfcf.)
__device__ __forceinline__ float normal_function(float z, float &density) {
  constexpr float C = -0.72134752044448170f, C_REST = (float)(-0.72134752044448170368 - (double)C), LN2 = 0.69314718055994531f;
  const float a = fminf(fabsf(z), 16.0f);
  const float square = a * a, power = square * C;
  const float rest = fmaf(fmaf(a, a, -square), C, fmaf(square, C_REST, fmaf(square, C, -power)));
  const float t = __builtin_amdgcn_rcpf(fmaf(0.345f, a, 1.0f));
  density = __builtin_amdgcn_exp2f(power);
  density = fmaf(density, rest * LN2, density);
  float p = -0.028381976f;
  p = fmaf(p, t, 0.145282045f);
  p = fmaf(p, t, -0.271173209f);
  p = fmaf(p, t, 0.187196776f);
  p = fmaf(p, t, -0.0376017168f);
  p = fmaf(p, t, 0.111799605f);
  p = fmaf(p, t, 0.117238283f);
  p = fmaf(p, t, 0.138020888f);
  p = fmaf(p, t, 0.137619287f);
  const float tail = density * (t * p);
  return z < 0.0f ? tail : 1.0f - tail;
}

// The activation, or with SLOPE also its derivative.  exp and the quotient are the hardware's (relative error of a few
// 2^-24; what exp loses for large arguments belongs to values next to zero).
template <bool SLOPE>
__device__ __forceinline__ float activation(int act, float z, float &slope) {
  constexpr float LOG2E = 1.44269504088896341f;
  float a;
  if (act == BNN_ACT_SILU) {
    const float t = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -LOG2E));
    a = z * t;
    if (SLOPE) slope = t * (1.0f + z * (1.0f - t));
  } else if (act == BNN_ACT_GELU) {
    float density;
    const float t = normal_function(z, density);
    a = z * t;
    if (SLOPE) slope = t + z * 0.39894228040143268f * density;
  } else if (act == BNN_ACT_GELU_TANH) {
    const float k = 0.79788456080286536f, c = 0.044715f;
    const float t = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-2.0f * LOG2E * k * (z + c * z * z * z)));  // (1 + tanh) / 2
    a = z * t;
    if (SLOPE) slope = t + 2.0f * z * t * (1.0f - t) * k * (1.0f + 3.0f * c * fminf(z * z, 1e30f));
  } else {
    a = z > 0.0f || z != z ? z : 0.0f;
    if (SLOPE) slope = z > 0.0f ? 1.0f : 0.0f;
  }
  return a;
}

// f with the activation as a tag.
template <class F>
bnn_status with_act(int act, const F &f) {
  switch (act) {
    case BNN_ACT_SILU: return f(std::integral_constant<int, BNN_ACT_SILU>());
    case BNN_ACT_GELU: return f(std::integral_constant<int, BNN_ACT_GELU>());
    case BNN_ACT_GELU_TANH: return f(std::integral_constant<int, BNN_ACT_GELU_TANH>());
    default: return f(std::integral_constant<int, BNN_ACT_RELU>());
  }
}

}  // namespace bnn
