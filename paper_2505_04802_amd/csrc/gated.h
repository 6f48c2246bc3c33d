// Internal declarations of the gated feed-forward layer: y = (act(x Wg^T + bg) o (x Wu^T + bu)) Wo^T + bo.
// gated.hip holds the entry points, gated_gemm.hip the bf16 and e4m3 products, gated_f32.hip the fp32 path.
#pragma once

#include "gated_plan.h"
#include "gelu.h"
#include "rows_common.h"

namespace reslim {

// act(v) and its derivative to about 2e-6 of the larger of the two, for results that are rounded to bf16; NaN stays NaN.
// SiLU: v p, p = 1 / (1 + e^-v); slope p + v p (1 - p).  GELU: v Phi(v), slope Phi(v) + v phi(v), Phi(-|v|) = 2^P(|v|) as in gelu.h.
template <bool GELU>
__device__ __forceinline__ float gate_act(float v) {
  if constexpr (GELU) return gelu_erf_fast(v) + (v != v ? v : 0.f);      // that function's bounds drop a NaN
  else return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -1.44269504088896341f));
}
template <bool GELU>
__device__ __forceinline__ void gate_act_slope(float v, float &a, float &slope) {
  if constexpr (GELU) {
    const float u = __builtin_amdgcn_fmed3f(fabsf(v), 0.0f, 5.0f);
    float p = fmaf(2.975744064e-05f, u, -7.135751075e-04f);
    p = fmaf(p, u, 7.775241509e-03f);
    p = fmaf(p, u, -5.269032717e-02f);
    p = fmaf(p, u, -4.595123231e-01f);
    p = fmaf(p, u, -1.150926590e+00f);
    p = fmaf(p, u, -1.000011683e+00f);
    const float tail = __builtin_amdgcn_exp2f(p);
    a = fmaf(-u, tail, v < 0.f ? 0.f : v);
    slope = fmaf(v * 0.3989422804014327f, __builtin_amdgcn_exp2f(v * v * -0.72134752044448170f), v < 0.f ? tail : 1.0f - tail);
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

struct GatedIn {                       // x W_in^T and what follows up to the hidden layer
  const void *x, *w_in;                // [M, D], [2R, D]: bf16 or e4m3
  const float *x_scale, *in_scale;     // e4m3: [M], [2R]
  const float *b_in;                   // [2R] or null
  void *gu, *h;                        // [M, 2R] or null, [M, R]
  int M, D, R;
};
hipError_t gated_gemm_init();
hipError_t launch_gated_in(const GatedIn &g, bool gelu, hipStream_t st);
// out [M, N] bf16 = a [M, K] times w [N, K] transposed, or w [K, N] (across), + bias (may be null); how: gated_choose_out(); part: how.slices M N floats
// where how.slices > 1.  other: microseconds that kernels beside the ring cost on top (the ring alone reads w across).
GatedChoice gated_choose_out(int M, int N, int K, double other);
hipError_t launch_gated_out(const GatedChoice &how, const void *a, const void *w, bool across, const float *bias, const float *zeros, void *out, int M, int N, int K, float *part,
                            hipStream_t st);
// d_gu [M, 2R] from dy [M, D], the output map [D, R] (across) or its transpose [R, D], and the forward's gu
GatedChoice gated_choose_dgate(int M, int D, int R, double other);
hipError_t launch_gated_dgate(const GatedChoice &how, const void *dy, const void *w, bool across, const void *gu, void *d_gu, int M, int D, int R, bool gelu, hipStream_t st);
// wt_in [D, 2R] = w_in^T, wt_out [R, D] = w_out^T in one launch; a destination that is null is left out
hipError_t launch_gated_transpose(const void *w_in, void *wt_in, const void *w_out, void *wt_out, int D, int R, hipStream_t st);

// fp32, any sizes; see gated_f32.hip.  part: partial sums of the slices of a product [M, N] over K, gated_f32_product_bytes()
size_t gated_f32_product_bytes(int M, int N, int K);
hipError_t launch_gated_f32_in(const GatedIn &g, bool gelu, hipStream_t st);
hipError_t launch_gated_f32_out(const float *h, const float *w_out, const float *b_out, float *y, int M, int D, int R, float *part, hipStream_t st);
hipError_t launch_gated_f32_dgate(const float *dy, const float *w_out, const float *gu, float *d_gu, int M, int D, int R, bool gelu, hipStream_t st);
hipError_t launch_gated_f32_dx(const float *d_gu, const float *w_in, float *dx, int M, int D, int R, float *part, hipStream_t st);
// dw [N, K] = dy[M, N]^T x[M, K], db (or null) = column sums of dy
size_t gated_f32_wgrad_bytes(int M, int N, int K);
hipError_t launch_gated_f32_wgrad(const float *dy, const float *x, float *dw, float *db, int M, int N, int K, void *ws, hipStream_t st);

}  // namespace reslim
