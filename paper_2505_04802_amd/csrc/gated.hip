// Entry points of the gated feed-forward layer: checks, workspace, and the order of the launches.
//
// Forward: one launch for both projections, activation and product, one for the output map (two where its sum is sliced).  Gradient
// (bf16): transposed copies of the matrices whose product does not run on 64 x 64 tiles (the input gradients contract over
// the weights' rows, which those tiles alone read as they lie), the hidden layer's gradient with the gradients of gate and up in its
// epilogue, dx, and one launch for both weight gradients with their biases.
//   bf16 and e4m3: the hidden layer is rounded to bf16 between the products, [dg | du] between theirs.  The second product's matrix instructions take bf16 operands
// (fp32 ones run at a tenth of the rate and twice the bytes), and the hidden layer is an output of the training forward.  The roundings take the 2-norm error of a bf16
// result from 1.7e-3, what rounding it once leaves, to 2.4e-3.
#include <algorithm>
#include <mutex>

#include "gated.h"

namespace reslim {

constexpr int kGatedMaxD = 16384, kGatedMaxR = 65536;
static __device__ __align__(256) float gated_no_bias[kGatedMaxD];      // zeros, never written

constexpr int kGatedDevices = 64;
static std::mutex g_gated_mutex;
static bool g_gated_ready[kGatedDevices];
static const float *g_gated_zeros[kGatedDevices];

// Kernel attributes and the address of the zeros on the current device; once for every device.
static hipError_t gated_ready(const float **zeros) {
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= kGatedDevices) return hipErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(g_gated_mutex);
  if (!g_gated_ready[dev]) {
    void *p = nullptr;
    e = hipGetSymbolAddress(&p, HIP_SYMBOL(gated_no_bias));
    if (e == hipSuccess) e = gemm_init();
    if (e == hipSuccess) e = wgrad_init();
    if (e == hipSuccess) e = gated_gemm_init();
    if (e != hipSuccess) return e;
    g_gated_zeros[dev] = static_cast<const float *>(p);
    g_gated_ready[dev] = true;
  }
  *zeros = g_gated_zeros[dev];
  return hipSuccess;
}

// Workspaces of the bf16 and e4m3 forms go by the device's compute units; without a device they are sized for the 256 of a whole MI355X.
static int gated_units(const char *fn, int x_dtype) {
  const float *zeros = nullptr;
  const hipError_t e = x_dtype == RESLIM_F32 ? hipSuccess : gated_ready(&zeros);
  return e == hipSuccess || e == hipErrorNoDevice ? RESLIM_OK : refuse_hip(fn, e);
}

// ------------------------------------------------------------------ no rows: parameter gradients of zero
struct ZeroArgs { uint16_t *p[4]; int64_t n[4]; };
__global__ __launch_bounds__(256) void gated_zero_kernel(ZeroArgs a) {
  uint16_t *p = a.p[blockIdx.y];
  if (!p) return;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < a.n[blockIdx.y]; i += static_cast<int64_t>(gridDim.x) * 256) p[i] = 0;
}

// ------------------------------------------------------------------ workspaces
static size_t gated_hidden_bytes(int M, int R, int x_dtype) { return align256(static_cast<size_t>(M) * R * (x_dtype == RESLIM_F32 ? 4 : 2)); }
// partial sums of a product's slices: out [M, N] over K
static size_t gated_part_bytes(int slices, int M, int N) { return slices > 1 ? align256(static_cast<size_t>(slices) * M * N * sizeof(float)) : 0; }
// How the output map is computed, and the forward's workspace: partial sums, behind them the hidden layer.  Both go by the device's compute units: one
// plan for the size that is checked and the launches, made after gated_ready.
struct GatedFwdPlan {
  GatedChoice out;
  size_t hidden_at, total;
};
static GatedFwdPlan gated_fwd_plan(int M, int D, int R, int x_dtype) {
  GatedFwdPlan p = {};
  if (M < 1) return p;
  if (x_dtype != RESLIM_F32) p.out = gated_choose_out(M, D, R, 0.0);
  p.hidden_at = x_dtype == RESLIM_F32 ? gated_f32_product_bytes(M, D, R) : gated_part_bytes(p.out.slices, M, D);
  p.total = p.hidden_at + gated_hidden_bytes(M, R, x_dtype);
  return p;
}

// How the two input gradients of the bf16 path are computed.  The 64 x 64 tiles read the weights as they lie; for the other kernels they are copied
// transposed first, read and written once at about 4.5 TB/s, after the launch.
struct GatedBwdPlan { GatedChoice dgate, dx; };
static GatedBwdPlan gated_bwd_plan(int M, int D, int R) {
  const double copy = 4e-6 / 4.5 * D * static_cast<double>(R);
  return {gated_choose_dgate(M, D, R, 2.0 + copy), gated_choose_out(M, D, 2 * R, 2.0 + 2 * copy)};
}
struct GatedBwdWs {
  GatedBwdPlan plan;           // bf16
  void *d_gu;                  // act [M, 2R]
  void *wt_in, *wt_out;        // bf16 [D, 2R], [R, D], or null
  void *part;                  // partial sums of dx
  void *wgrad;                 // partial sums of the parameter gradients
  void *sink_in, *sink_out;    // 2R and D floats: bias gradients that nobody asked for
  size_t total;
};
static void gated_ops(WgradOp (&op)[2], const void *d_gu, const void *x, const void *dy, const void *h, int D, int R) {
  op[0] = {d_gu, x, nullptr, nullptr, 2 * R, D};
  op[1] = {dy, h, nullptr, nullptr, D, R};
}
static GatedBwdWs plan_gated_bwd(int M, int D, int R, int dtype, void *base) {
  unsigned char *p = static_cast<unsigned char *>(base);
  size_t off = 0;
  auto take = [&](size_t bytes) { unsigned char *q = p + off; off += align256(bytes); return q; };
  const size_t es = type_bytes(dtype), m = M, d = D, r = R;
  GatedBwdWs w = {};
  if (M < 1) return w;
  w.d_gu = take(m * 2 * r * es);
  if (dtype == RESLIM_BF16) {
    w.plan = gated_bwd_plan(M, D, R);
    w.part = take(gated_part_bytes(w.plan.dx.slices, M, D));
    if (w.plan.dx.kernel != kGatedRing) w.wt_in = take(2 * r * d * 2);
    if (w.plan.dgate.kernel != kGatedRing) w.wt_out = take(r * d * 2);
    w.sink_in = take(2 * r * sizeof(float));
    w.sink_out = take(d * sizeof(float));
    WgradOp op[2];
    gated_ops(op, nullptr, nullptr, nullptr, nullptr, D, R);
    w.wgrad = take(wgrad_ws_bytes(RESLIM_BF16, op, 2, M));
  } else {
    w.part = take(gated_f32_product_bytes(M, D, 2 * R));
    w.wgrad = take(std::max(gated_f32_wgrad_bytes(M, 2 * R, D), gated_f32_wgrad_bytes(M, D, R)));
  }
  w.total = off;
  return w;
}

// ------------------------------------------------------------------ checks
static int gated_shape(const char *fn, int rows, int D, int R, int x_dtype) {
  if (x_dtype != RESLIM_F32 && x_dtype != RESLIM_BF16 && x_dtype != RESLIM_E4M3) return refuse(RESLIM_EINVAL, fn, "x_dtype must be RESLIM_F32, RESLIM_BF16 or RESLIM_E4M3");
  if (rows < 0 || rows > 2000000000 || D < 1 || D > kGatedMaxD || R < 1 || R > kGatedMaxR) return refuse(RESLIM_ESHAPE, fn, "need 0 <= rows <= 2,000,000,000, 1 <= D <= 16384 and 1 <= R <= 65536");
  if (x_dtype == RESLIM_F32 && rows > 4000000) return refuse(RESLIM_ESHAPE, fn, "the fp32 path takes up to 4,000,000 rows");
  // ... and as many tiles of its widest layer and of its result as one launch has work-groups
  const int64_t strips = (static_cast<int64_t>(rows) + 63) / 64;
  if (x_dtype == RESLIM_F32 && strips * std::max((R + 31) / 32, (D + 63) / 64) > most_groups(256))
    return refuse(RESLIM_ESHAPE, fn, "the fp32 path takes up to 2^23 tiles of 64 rows by 32 hidden or 64 output features");
  if (x_dtype == RESLIM_BF16 && (D % 64 || R % 64)) return refuse(RESLIM_ESHAPE, fn, "bf16 needs D and R to be multiples of 64");
  if (x_dtype == RESLIM_E4M3 && (D % 128 || R % 64)) return refuse(RESLIM_ESHAPE, fn, "e4m3 needs D to be a multiple of 128 and R of 64");
  return RESLIM_OK;
}
static int gated_check(const char *fn, const reslim_gated_mlp_weights *w, int gate, int rows, int D, int R, int x_dtype, std::initializer_list<const void *> buffers,
                       std::initializer_list<const void *> optional) {
  const int rc = gated_shape(fn, rows, D, R, x_dtype);
  if (rc != RESLIM_OK) return rc;
  if (gate != RESLIM_GATE_SILU && gate != RESLIM_GATE_GELU) return refuse(RESLIM_EINVAL, fn, "unknown gate");
  if (!w || !w->w_in || !w->w_out) return refuse(RESLIM_EINVAL, fn, "null weights");
  if ((x_dtype == RESLIM_E4M3) != (w->in_scale != nullptr)) return refuse(RESLIM_EINVAL, fn, "in_scale goes with RESLIM_E4M3, and only with it");
  const size_t al = x_dtype == RESLIM_F32 ? 4 : 16;
  bool start = aligned(w->w_in, al) && aligned(w->w_out, al) && aligned(w->in_scale, al) && aligned(w->b_in, al) && aligned(w->b_out, al);
  for (const void *b : buffers) {
    if (!b && rows > 0) return refuse(RESLIM_EINVAL, fn, "null buffer");
    start = start && aligned(b, al);
  }
  for (const void *b : optional) start = start && aligned(b, al);
  return start ? RESLIM_OK : refuse(RESLIM_EINVAL, fn, "a buffer does not start on 16 bytes (fp32: 4)");
}
static int gated_room(const char *fn, const void *ws, size_t ws_bytes, size_t need) {
  if (need == 0 || (ws && aligned(ws, 256) && ws_bytes >= need)) return RESLIM_OK;
  return refuse(RESLIM_EWORKSPACE, fn, "workspace null, not 256-byte aligned or smaller than the workspace query says");
}

static hipError_t gated_forward(const GatedFwdPlan &plan, const GatedIn &in, const reslim_gated_mlp_weights *w, int x_dtype, bool gelu, void *y, void *part, const float *zeros, hipStream_t st) {
  const bool f32 = x_dtype == RESLIM_F32;
  const hipError_t e = f32 ? launch_gated_f32_in(in, gelu, st) : launch_gated_in(in, gelu, st);
  if (e != hipSuccess) return e;
  if (f32) return launch_gated_f32_out(static_cast<const float *>(in.h), static_cast<const float *>(w->w_out), w->b_out, static_cast<float *>(y), in.M, in.D, in.R, static_cast<float *>(part), st);
  return launch_gated_out(plan.out, in.h, w->w_out, false, w->b_out, zeros, y, in.M, in.D, in.R, static_cast<float *>(part), st);
}

}  // namespace reslim

using namespace reslim;

extern "C" int reslim_gated_mlp_workspace_bytes(int32_t rows, int32_t D, int32_t R, int32_t x_dtype, size_t *out) {
  const char *fn = "reslim_gated_mlp_workspace_bytes";
  if (!out) return refuse(RESLIM_EINVAL, fn, "null argument");
  int rc = gated_shape(fn, rows, D, R, x_dtype);
  if (rc != RESLIM_OK) return rc;
  if ((rc = gated_units(fn, x_dtype)) != RESLIM_OK) return rc;
  *out = gated_fwd_plan(rows, D, R, x_dtype).total;
  return RESLIM_OK;
}

extern "C" int reslim_gated_mlp_fwd(const void *x, const float *x_scale, const reslim_gated_mlp_weights *w, int32_t gate, int32_t rows, int32_t D, int32_t R,
                                    int32_t x_dtype, void *y, void *workspace, size_t ws_bytes, void *hip_stream) {
  const char *fn = "reslim_gated_mlp_fwd";
  int rc = gated_check(fn, w, gate, rows, D, R, x_dtype, {x, y}, {});
  if (rc != RESLIM_OK) return rc;
  if (rows > 0 && (x_dtype == RESLIM_E4M3) != (x_scale != nullptr)) return refuse(RESLIM_EINVAL, fn, "x_scale goes with RESLIM_E4M3, and only with it");
  if (!aligned(x_scale, 4)) return refuse(RESLIM_EINVAL, fn, "a buffer is not aligned to its elements");
  if (rows == 0) return RESLIM_OK;
  const float *zeros = nullptr;
  hipError_t e = gated_ready(&zeros);
  const GatedFwdPlan plan = gated_fwd_plan(rows, D, R, x_dtype);
  if ((rc = gated_room(fn, workspace, ws_bytes, plan.total)) != RESLIM_OK) return rc;
  unsigned char *h = static_cast<unsigned char *>(workspace) + plan.hidden_at;
  const GatedIn in = {x, w->w_in, x_scale, w->in_scale, w->b_in, nullptr, h, rows, D, R};
  if (e == hipSuccess) e = gated_forward(plan, in, w, x_dtype, gate == RESLIM_GATE_GELU, y, workspace, zeros, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? RESLIM_OK : refuse_hip(fn, e);
}

extern "C" int reslim_gated_mlp_fwd_train(const void *x, const reslim_gated_mlp_weights *w, int32_t gate, int32_t rows, int32_t D, int32_t R, int32_t x_dtype,
                                          void *gu, void *h, void *y, void *workspace, size_t ws_bytes, void *hip_stream) {
  const char *fn = "reslim_gated_mlp_fwd_train";
  int rc = gated_check(fn, w, gate, rows, D, R, x_dtype, {x, gu, h, y}, {});
  if (rc != RESLIM_OK) return rc;
  if (x_dtype == RESLIM_E4M3) return refuse(RESLIM_EINVAL, fn, "training takes RESLIM_F32 or RESLIM_BF16");
  if (rows == 0) return RESLIM_OK;
  const float *zeros = nullptr;
  hipError_t e = gated_ready(&zeros);
  const GatedFwdPlan plan = gated_fwd_plan(rows, D, R, x_dtype);
  if ((rc = gated_room(fn, workspace, ws_bytes, plan.total)) != RESLIM_OK) return rc;
  const GatedIn in = {x, w->w_in, nullptr, nullptr, w->b_in, gu, h, rows, D, R};
  if (e == hipSuccess) e = gated_forward(plan, in, w, x_dtype, gate == RESLIM_GATE_GELU, y, workspace, zeros, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? RESLIM_OK : refuse_hip(fn, e);
}

static int gated_grad_type(const char *fn, int x_dtype, int grad_dtype) {
  if (x_dtype == RESLIM_E4M3) return refuse(RESLIM_EINVAL, fn, "training takes RESLIM_F32 or RESLIM_BF16");
  if (grad_dtype != RESLIM_F32 && (grad_dtype != RESLIM_BF16 || x_dtype != RESLIM_BF16)) return refuse(RESLIM_EINVAL, fn, "grad_dtype must be RESLIM_F32, or RESLIM_BF16 with x_dtype RESLIM_BF16");
  return RESLIM_OK;
}

extern "C" int reslim_gated_mlp_bwd_workspace_bytes(int32_t rows, int32_t D, int32_t R, int32_t x_dtype, int32_t grad_dtype, size_t *out) {
  const char *fn = "reslim_gated_mlp_bwd_workspace_bytes";
  if (!out) return refuse(RESLIM_EINVAL, fn, "null argument");
  int rc = gated_shape(fn, rows, D, R, x_dtype);
  if (rc == RESLIM_OK) rc = gated_grad_type(fn, x_dtype, grad_dtype);
  if (rc == RESLIM_OK) rc = gated_units(fn, x_dtype);
  if (rc != RESLIM_OK) return rc;
  *out = plan_gated_bwd(rows, D, R, x_dtype, nullptr).total;
  return RESLIM_OK;
}

extern "C" int reslim_gated_mlp_bwd(const void *x, const void *gu, const void *h, const void *dy, const reslim_gated_mlp_weights *w, int32_t gate, int32_t rows,
                                    int32_t D, int32_t R, int32_t x_dtype, int32_t grad_dtype, void *dx, const reslim_gated_mlp_grads *grads, void *workspace,
                                    size_t ws_bytes, void *hip_stream) {
  const char *fn = "reslim_gated_mlp_bwd";
  if (!grads || !grads->w_in || !grads->w_out) return refuse(RESLIM_EINVAL, fn, "null gradients");
  int rc = gated_check(fn, w, gate, rows, D, R, x_dtype, {x, gu, h, dy}, {dx, grads->w_in, grads->w_out, grads->b_in, grads->b_out});
  if (rc == RESLIM_OK) rc = gated_grad_type(fn, x_dtype, grad_dtype);
  if (rc != RESLIM_OK) return rc;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const float *zeros = nullptr;
  hipError_t e = gated_ready(&zeros);
  if (e != hipSuccess) return refuse_hip(fn, e);
  if (rows == 0) {
    const int64_t es = grad_dtype == RESLIM_BF16 ? 1 : 2, n = static_cast<int64_t>(D) * R;      // in 16-bit words
    ZeroArgs z = {{static_cast<uint16_t *>(grads->w_in), static_cast<uint16_t *>(grads->b_in), static_cast<uint16_t *>(grads->w_out), static_cast<uint16_t *>(grads->b_out)},
                  {2 * n * es, 2 * R * es, n * es, D * es}};
    gated_zero_kernel<<<dim3(1024, 4), dim3(256), 0, st>>>(z);
    e = hipGetLastError();
    return e == hipSuccess ? RESLIM_OK : refuse_hip(fn, e);
  }
  const GatedBwdWs ws = plan_gated_bwd(rows, D, R, x_dtype, workspace);
  if ((rc = gated_room(fn, workspace, ws_bytes, ws.total)) != RESLIM_OK) return rc;
  const bool gelu = gate == RESLIM_GATE_GELU;
  if (x_dtype == RESLIM_F32) {
    auto f = [](const void *p) { return static_cast<const float *>(p); };
    auto o = [](void *p) { return static_cast<float *>(p); };
    e = launch_gated_f32_dgate(f(dy), f(w->w_out), f(gu), o(ws.d_gu), rows, D, R, gelu, st);
    if (e == hipSuccess && dx) e = launch_gated_f32_dx(f(ws.d_gu), f(w->w_in), o(dx), rows, D, R, o(ws.part), st);
    if (e == hipSuccess) e = launch_gated_f32_wgrad(f(ws.d_gu), f(x), o(grads->w_in), o(grads->b_in), rows, 2 * R, D, ws.wgrad, st);
    if (e == hipSuccess) e = launch_gated_f32_wgrad(f(dy), f(h), o(grads->w_out), o(grads->b_out), rows, D, R, ws.wgrad, st);
    return e == hipSuccess ? RESLIM_OK : refuse_hip(fn, e);
  }
  e = launch_gated_transpose(w->w_in, dx ? ws.wt_in : nullptr, w->w_out, ws.wt_out, D, R, st);
  if (e == hipSuccess) e = launch_gated_dgate(ws.plan.dgate, dy, ws.wt_out ? ws.wt_out : w->w_out, !ws.wt_out, gu, ws.d_gu, rows, D, R, gelu, st);
  if (e == hipSuccess && dx)
    e = launch_gated_out(ws.plan.dx, ws.d_gu, ws.wt_in ? ws.wt_in : w->w_in, !ws.wt_in, nullptr, zeros, dx, rows, D, 2 * R, static_cast<float *>(ws.part), st);
  if (e == hipSuccess) {
    WgradOp op[2];
    gated_ops(op, ws.d_gu, x, dy, h, D, R);
    op[0].dw = static_cast<float *>(grads->w_in);
    op[0].db = static_cast<float *>(grads->b_in ? grads->b_in : ws.sink_in);
    op[1].dw = static_cast<float *>(grads->w_out);
    op[1].db = static_cast<float *>(grads->b_out ? grads->b_out : ws.sink_out);
    e = launch_wgrad(RESLIM_BF16, op, 2, rows, ws.wgrad, st, grad_dtype == RESLIM_BF16);
  }
  return e == hipSuccess ? RESLIM_OK : refuse_hip(fn, e);
}
