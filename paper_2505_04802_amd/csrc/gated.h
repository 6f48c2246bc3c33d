// Internal declarations of the gated feed-forward layer: y = (act(x Wg^T + bg) o (x Wu^T + bu)) Wo^T + bo.
// gated.hip holds the entry points, gated_gemm.hip the bf16 and e4m3 products, gated_f32.hip the fp32 path.
#pragma once

#include "gate_act.h"
#include "gated_plan.h"
#include "gelu.h"
#include "rows_common.h"

namespace reslim {

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
