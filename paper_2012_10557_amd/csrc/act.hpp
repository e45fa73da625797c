// Activations of the epilogues and of group norm, and their derivatives, in
// fp32 for values stored as T.  Nothing here is contracted with what surrounds
// it, so that every path of a kernel (16-byte accesses or not) gives the same
// bits.
#pragma once

#include <type_traits>

#include "common.hpp"

namespace ekya {

enum Act { ACT_NONE = 0, ACT_RELU = 1, ACT_SILU = 2, ACT_GELU = 3 };

// 1 / (1 + exp(-u)); exp(-u) may overflow, the quotient is then 0.  bf16: the
// hardware's exp2 and reciprocal, off by about (|u| + 2) 2^-24, far below the
// 2^-9 of the result's rounding.  fp32: the same two, the exponent in two parts
// (what u log2 e loses is added to first order) and a Newton step on the
// reciprocal, off by 3 halves of a step; library exponential and division took
// 25 us where this takes 20 (group norm backward, 19 x 1147 x 120).  From
// |u| = 87.3 on neither the second part nor the step is taken: exp(-u) is then
// below 2^-126 and the quotient 1, or the quotient below 2^-126 and 0, and parts
// of an infinite exponent would make it NaN.
template <typename T> __device__ __forceinline__ float sigmoid_of(float u) {
#pragma clang fp contract(off)
  if constexpr (sizeof(T) == 4) {
    const float t = u * -1.44269502f;
    const float lo = fmaf(u, -1.44269502f, -t) + u * -1.92596299e-8f;
    const bool in = fabsf(t) < 126.f;
    float e = __builtin_amdgcn_exp2f(t);
    e = in ? fmaf(e, 0.693147181f * lo, e) : e;
    const float d = 1.f + e, r = __builtin_amdgcn_rcpf(d);
    return in ? fmaf(fmaf(-d, r, 1.f), r, r) : r;
  }
  return __builtin_amdgcn_rcpf(1.f + __expf(-u));
}

// (1 + erf(u / sqrt 2)) / 2.  fp32: by erfc, which keeps its digits where the
// sum cancels (u far below 0).  bf16: below 0, exp(-u^2 / 2) t (c0 + .. + c5 t^5)
// with t = 1 / (1 + p |u|); above it 1 less that.  p and c are fitted to
// erfc(x) exp(x^2) / 2, x = |u| / sqrt 2, by reweighted least squares until the
// largest error is least, an error counting by the larger of 1e-7 and 2e-4 of the
// value: it is off by 5e-8 at most, and below 0 by 1.03e-4 of itself, a 38th of
// the result's rounding (a fit of the absolute error alone lost half a step
// at -6 and two and a half at -10).  `e` receives exp(-u^2 / 2).
template <typename T> __device__ __forceinline__ float normal_cdf(float u, float& e) {
#pragma clang fp contract(off)
  if constexpr (sizeof(T) == 4) {
    e = expf(-0.5f * u * u);
    return 0.5f * erfcf(-0.70710678f * u);
  }
  e = __builtin_amdgcn_exp2f(u * u * -0.721347520f);
  const float t = __builtin_amdgcn_rcpf(fmaf(0.290620893f, fabsf(u), 1.f));
  float p = fmaf(t, -0.0886891708f, 0.28227067f);
  p = fmaf(t, p, -0.0903111845f);
  p = fmaf(t, p, 0.178372741f);
  p = fmaf(t, p, 0.101264767f);
  const float h = t * fmaf(t, p, 0.117092133f) * e;
  return u < 0.f ? h : 1.f - h;
}

template <int ACT, typename T> __device__ __forceinline__ float act_fwd(float u) {
#pragma clang fp contract(off)
  if constexpr (ACT == ACT_RELU) return relu_nan(u);
  if constexpr (ACT == ACT_SILU) return u * sigmoid_of<T>(u);
  float e;
  if constexpr (ACT == ACT_GELU) return u * normal_cdf<T>(u, e);
  return u;
}

// dy * act'(u).  A masked-out ReLU gradient is 0 even where dy is not finite.
template <int ACT, typename T> __device__ __forceinline__ float act_bwd(float dy, float u) {
#pragma clang fp contract(off)
  if constexpr (ACT == ACT_RELU) return u > 0.f ? dy : 0.f;
  if constexpr (ACT == ACT_SILU) {
    const float p = sigmoid_of<T>(u);
    return dy * (p * (1.f + u * (1.f - p)));
  }
  if constexpr (ACT == ACT_GELU) {
    float e;
    const float p = normal_cdf<T>(u, e);
    return dy * (p + u * (0.39894228f * e));
  }
  return dy;
}

// Calls f(std::integral_constant<int, ACT>) for a checked activation.
template <typename F> auto act_dispatch(int act, F&& f) {
  switch (act) {
    case ACT_RELU: return f(std::integral_constant<int, ACT_RELU>{});
    case ACT_SILU: return f(std::integral_constant<int, ACT_SILU>{});
    case ACT_GELU: return f(std::integral_constant<int, ACT_GELU>{});
    default: return f(std::integral_constant<int, ACT_NONE>{});
  }
}

}  // namespace ekya
