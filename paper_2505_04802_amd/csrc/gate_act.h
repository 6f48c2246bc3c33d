// The gate of a feed-forward layer, act = SiLU or GELU, and its derivative (gated_gemm.hip, gated_f32.hip).
#pragma once

#include "common.h"

namespace reslim {

// Phi(-u), the normal distribution's tail, for u >= 0: 2^P(u) with the degree-6 fit of gelu.h up to 5, whose error is 1.5e-5 of Phi, and beyond it P(5) and a
// cubic in u - 5 fitted to the logarithm down to where Phi leaves fp32 (u = 13), 1.6e-3 of Phi: less than half a step of bf16.  It falls to zero, and NaN stays NaN.
__device__ __forceinline__ float gate_normal_tail(float u) {
  const float w = __builtin_amdgcn_fmed3f(u, 0.0f, 5.0f), d = u - w;
  float p = fmaf(2.975744064e-05f, w, -7.135751075e-04f);
  p = fmaf(p, w, 7.775241509e-03f);
  p = fmaf(p, w, -5.269032717e-02f);
  p = fmaf(p, w, -4.595123231e-01f);
  p = fmaf(p, w, -1.150926590e+00f);
  p = fmaf(p, w, -1.000011683e+00f);
  const float q = fmaf(fmaf(-6.91575691e-04f, d, -7.03860663e-01f), d, -7.47598466f);
  return __builtin_amdgcn_exp2f(fmaf(q, d, p));
}

// act(v) and its derivative for results that are rounded to bf16.  SiLU: v p, p = 1 / (1 + e^-v); slope p + v p (1 - p), to a few half steps of fp32 times
// |v|.  GELU: v Phi(v), to 1.5e-5 of it from -5 on and 1.6e-3 below; slope Phi(v) + v phi(v), Phi(v) as exact.  At the infinities both give what the definition gives in
// fp32: act(+inf) = +inf, act(-inf) and the slopes NaN.
template <bool GELU>
__device__ __forceinline__ float gate_act(float v) {
  if constexpr (GELU) {
    const float tail = gate_normal_tail(fabsf(v));
    return v * (v < 0.f ? tail : 1.0f - tail);
  } else {
    return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -1.44269504088896341f));
  }
}
template <bool GELU>
__device__ __forceinline__ void gate_act_slope(float v, float &a, float &slope) {
  if constexpr (GELU) {
    const float tail = gate_normal_tail(fabsf(v)), cdf = v < 0.f ? tail : 1.0f - tail;
    a = v * cdf;
    slope = fmaf(v * 0.3989422804014327f, __builtin_amdgcn_exp2f(v * v * -0.72134752044448170f), cdf);
  } else {
    const float p = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -1.44269504088896341f));
    a = v * p;
    slope = fmaf(a, 1.0f - p, p);
  }
}
// The same with the library's functions, for fp32 results.
template <bool GELU>
__device__ __forceinline__ void gate_act_slope_f32(float v, float &a, float &slope) {
  if constexpr (GELU) {
    const float p = 0.5f * (1.0f + erff(v * 0.70710678118654752f));
    a = v * p;
    slope = fmaf(v * 0.3989422804014327f, expf(-0.5f * v * v), p);
  } else {
    const float p = 1.0f / (1.0f + expf(-v));
    a = v * p;
    slope = fmaf(a, 1.0f - p, p);
  }
}
template <bool GELU>
__device__ __forceinline__ float gate_act_f32(float v) {
  if constexpr (GELU) return 0.5f * v * (1.0f + erff(v * 0.70710678118654752f));
  else return v / (1.0f + expf(-v));
}

}  // namespace reslim
