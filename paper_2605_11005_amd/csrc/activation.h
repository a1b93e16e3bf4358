// The activations of the linear layer (MOE_ACT_*), their slopes, and which function of them a kernel takes.
//
// FAST is for results that are rounded to bf16: the hardware's exp2 and reciprocal (about 1 ulp each), and erfc(u) = (c1 t + .. + c6 t^6) exp(-u^2)
// with t = 1 / (1 + 0.415 u) for u >= 0, the form of Abramowitz and Stegun's formula 7.1.26.  Its coefficients are the least largest error of
// erfc that a linear program finds over u = 0 .. 9.6, where 1.5e-7 or 6e-5 of the value, whichever is less, counts as one: found 0.95.  So what is left
// of gelu far below zero is off by 6e-5 of itself, a sixtieth of bf16's rounding (7.1.26 itself, one term shorter, is good to 1.5e-7 and no
// fraction of the value: 0.9 % at z = -7, 3.5 % at -13).  For fp32 the mathematical library's functions are called.  With S(v) = 1 / (1 + exp(-v)):
//   silu        z S(z)                    gelu (erf)   z erfc(-z / sqrt 2) / 2
//   gelu (tanh) z (1 + tanh u) / 2 = z S(2 u),  u = sqrt(2 / pi) (z + 0.044715 z^3)
// A NaN stays one in all of them.
#pragma once
#include "common.h"
#include "../../include/moe.h"

namespace {

template <bool FAST>
__device__ __forceinline__ float logistic(float v) {
  if constexpr (FAST) return sigmoid_fast(v);
  else return 1.0f / (1.0f + expf(-v));
}
// erfc(|z| / sqrt 2) / 2, the normal distribution's tail; *density: exp(-z^2 / 2)
template <bool FAST>
__device__ __forceinline__ float normal_tail(float z, float* density) {
  if constexpr (FAST) {
    const float t = __builtin_amdgcn_rcpf(1.0f + (0.415f * 0.70710678118654752f) * fabsf(z));
    *density = __builtin_amdgcn_exp2f((-0.5f * 1.44269504088896f) * z * z);
    const float poly =
        (((((-0.169389807f * t + 0.517603468f) * t - 0.123529036f) * t + 0.326369515f) * t + 0.213340989f) * t + 0.235604727f) * t;
    return 0.5f * poly * *density;
  } else {
    *density = expf(-0.5f * z * z);
    return 0.5f * erfcf(0.70710678118654752f * fabsf(z));
  }
}
constexpr float GELU_A = 1.5957691216057308f, GELU_B = GELU_A * 0.044715f;      // 2 sqrt(2 / pi); 2 u = z (A + B z^2)

template <int ACT, bool FAST>
__device__ __forceinline__ float act_value(float z) {
  if constexpr (ACT == MOE_ACT_RELU) return z < 0.f ? 0.f : z;
  else if constexpr (ACT == MOE_ACT_SILU) return z * logistic<FAST>(z);
  else if constexpr (ACT == MOE_ACT_GELU_TANH) return z * logistic<FAST>(z * (GELU_A + GELU_B * z * z));
  else if constexpr (ACT == MOE_ACT_GELU) {
    float density;
    const float tail = normal_tail<FAST>(z, &density);
    return z * (z > 0.f ? 1.f - tail : tail);
  } else return z;
}
// g times the slope at z
template <int ACT, bool FAST>
__device__ __forceinline__ float act_slope(float z, float g) {
  if constexpr (ACT == MOE_ACT_RELU) return z <= 0.f ? 0.f : g;
  else if constexpr (ACT == MOE_ACT_SILU) {
    const float s = logistic<FAST>(z);
    return g * (s * (1.f + z * (1.f - s)));
  } else if constexpr (ACT == MOE_ACT_GELU_TANH) {
    z = z > 100.f ? 100.f : z < -100.f ? -100.f : z;      // (0 or 1 long before; z^3 would pass fp32, and 0 times infinity is NaN)
    const float s = logistic<FAST>(z * (GELU_A + GELU_B * z * z));
    return g * (s * (1.f + z * (1.f - s) * (GELU_A + 3.f * GELU_B * z * z)));
  } else if constexpr (ACT == MOE_ACT_GELU) {
    float density;
    const float tail = normal_tail<FAST>(z, &density);
    return g * ((z > 0.f ? 1.f - tail : tail) + z * density * 0.39894228040143268f);
  } else return g;
}

// f(Int<ACT>{}) for the activation of a call
template <typename F>
__host__ __device__ __forceinline__ auto with_activation(int act, F f) {
  switch (act) {
    case MOE_ACT_RELU: return f(Int<MOE_ACT_RELU>{});
    case MOE_ACT_GELU: return f(Int<MOE_ACT_GELU>{});
    case MOE_ACT_GELU_TANH: return f(Int<MOE_ACT_GELU_TANH>{});
    case MOE_ACT_SILU: return f(Int<MOE_ACT_SILU>{});
    default: return f(Int<MOE_ACT_NONE>{});
  }
}
// eight values in bf16's precision
__device__ __forceinline__ void activate(int act, float* x) {
  with_activation(act, [&](auto a) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = act_value<decltype(a)::value, true>(x[i]);
  });
}

}  // namespace
