// Root-mean-square norm of token rows with the residual's addition in front, and its gradient.
//
//   s = x + delta,  r = 1 / sqrt(mean(s^2) + eps),  y = s r gamma                      (forward)
//   g = gamma dy,   ds = d_sum + r (g - s r mean(g s r)),  dgamma = sum_rows dy s r     (gradient)
//
// Both move every element once and compute next to nothing, so memory bounds them: a row stays in the registers of the
// threads that share it (a wave up to 1024 features, a work-group beyond) between the sums and the result, every load
// of a row is issued before the first is used, and 16 bytes of the stream is what a thread takes at a time, wherever they start.  Sums are
// fp32 in an order that depends on the row's width alone, so a row's result does not depend on the
// others.  s is normalised before it is rounded to the stream's type.  161,408 x 1024 (fp32 stream, bf16 addend and result) take 356 us, 5.6 TB/s,
// 37,520 x 4096 (bf16, e4m3 result) 187 us, 5.75 TB/s; a large copy reaches 4.9.
#include <algorithm>
#include <type_traits>

#include "rows_common.h"

namespace reslim {

struct NormArgs {
  const void *x, *delta;
  const float *gamma;
  void *sum, *y;
  float *y_scale;
  float eps;
  int64_t rows;
  int D;
};

// TAIL: a row ends inside a piece.  Its loads reach into the next row, as far as there is one, so that they go out with the others; what
// they bring from there is not used, and the piece is stored element by element.  At 29,304 x 4095 5.2 TB/s (fp32 stream, bf16 result) where
// 4096 features run at 5.6; element by element throughout, 2.3.
template <class S, class A, class Y, int V, int NT, int NC, bool TAIL>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void rmsnorm_kernel(NormArgs a) {
  constexpr int RPB = NT < 256 ? 256 / NT : 1;
  __shared__ float box[2][NT / 64];
  const int t = threadIdx.x % NT;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * RPB + threadIdx.x / NT;
  if (row >= a.rows) return;                 // whole waves, and only where no barrier follows (NT == 64)
  const int64_t at = row * a.D;
  const S *x = static_cast<const S *>(a.x) + at;
  const A *d = static_cast<const A *>(a.delta) + at;
  const int64_t most = TAIL ? a.rows * a.D - at : 0;       // elements from this row on
  auto store = [&](auto *p, int k, const float (&from)[V]) {
    typedef typename std::remove_reference<decltype(*p)>::type T;
    if (!TAIL || k + V <= a.D) Piece<T, V>::store(p + k, from);
    else store_some<T, V>(p + k, a.D - k, from);
  };
  float v[NC][V], w[NC][V];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int k = (i * NT + t) * V;
    if (k < a.D) {
      if (!TAIL || k + V <= most) {
        Piece<S, V>::load(x + k, v[i]);
        if (a.delta) Piece<A, V>::load(d + k, w[i]);
      } else {
        load_some<S, V>(x + k, a.D - k, v[i]);
        if (a.delta) load_some<A, V>(d + k, a.D - k, w[i]);
      }
    }
  }
  float sq = 0.f;
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int k = (i * NT + t) * V;
    if (k < a.D) {
      if (a.delta) {
#pragma unroll
        for (int j = 0; j < V; ++j) v[i][j] += w[i][j];
      }
      if (a.sum) store(static_cast<S *>(a.sum) + at, k, v[i]);
      if constexpr (TAIL) {
#pragma unroll
        for (int j = 0; j < V; ++j) v[i][j] = k + j < a.D ? v[i][j] : 0.f;
      }
#pragma unroll
      for (int j = 0; j < V; ++j) sq = fmaf(v[i][j], v[i][j], sq);
    }
  }
  const float r = rsqrtf(row_all<NT, false>(sq, box[0]) / static_cast<float>(a.D) + a.eps);
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int k = (i * NT + t) * V;
    if (k < a.D) {
      float g[V];
      if (!TAIL || k + V <= a.D) Piece<float, V>::load(a.gamma + k, g);
      else load_some<float, V>(a.gamma + k, a.D - k, g);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        v[i][j] = v[i][j] * r * g[j];
        top = fmaxf(top, fabsf(v[i][j]));
      }
      if constexpr (!std::is_same<Y, e4m3_t>::value) store(static_cast<Y *>(a.y) + at, k, v[i]);
    }
  }
  if constexpr (std::is_same<Y, e4m3_t>::value) {
    // the largest magnitude of the row becomes 448; a row of zeros keeps scale 0 and zeros
    top = row_all<NT, true>(top, box[1]);
    if (t == 0) a.y_scale[row] = top / kE4m3Max;
    const float lift = top < 0x1p-96f ? 0x1p64f : 1.0f;      // 448 / top leaves fp32 below 2^-119
    const float up = top > 0.f ? kE4m3Max / (top * lift) : 0.f;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int k = (i * NT + t) * V;
      if (k < a.D) {
#pragma unroll
        for (int j = 0; j < V; ++j) v[i][j] = v[i][j] * lift * up;
        store(static_cast<e4m3_t *>(a.y) + at, k, v[i]);
      }
    }
  }
}

struct NormBwdArgs {
  const void *s, *dy, *d_sum;
  const float *gamma;
  void *dx, *d_delta;
  float *partial;        // [work-groups, D]
  float eps;
  int64_t rows;
  int D;
};

// A work-group takes every gridDim-th row (four of them at widths of a wave), so that the chip works on neighbouring rows, and keeps its part of
// dgamma in registers.  The next row's loads are in flight while a row is summed and written: 37,520 x 4096 (fp32 stream, bf16 gradient, skip
// gradient) 467 us, 5.27 TB/s; without them 592, 4.15 TB/s.
template <class S, class A, int V, int NT, int NC, bool TAIL>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void rmsnorm_bwd_kernel(NormBwdArgs a) {
  constexpr int RPB = NT < 256 ? 256 / NT : 1;
  __shared__ float box[2][2 * (NT / 64)];
  __shared__ float sm[RPB > 1 ? RPB : 1][RPB > 1 ? NT * NC * V : 1];
  const int t = threadIdx.x % NT, part = threadIdx.x / NT;
  const int64_t r0 = static_cast<int64_t>(blockIdx.x) * RPB + part, stride = static_cast<int64_t>(gridDim.x) * RPB;
  float gam[NC][V], acc[NC][V];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int k = (i * NT + t) * V;
#pragma unroll
    for (int j = 0; j < V; ++j) gam[i][j] = acc[i][j] = 0.f;
    if (k < a.D) {
      if (!TAIL || k + V <= a.D) Piece<float, V>::load(a.gamma + k, gam[i]);
      else load_some<float, V>(a.gamma + k, a.D - k, gam[i]);
    }
  }
  const float inv_d = 1.0f / static_cast<float>(a.D);
  // Sixteen elements to a thread in work-groups of sixteen waves leave no registers for a second row, nor for a tail that has to be told
  // from the next row's elements: it is loaded element by element there, and the skip gradient with its tail where it is added.
  constexpr bool kAhead = NT < 1024 || NC * V <= 8, kReach = TAIL && kAhead;
  Held<S, V> s[NC], z[NC], sn[kAhead ? NC : 1], zn[kAhead ? NC : 1];
  Held<A, V> e[NC], en[kAhead ? NC : 1];
  auto store = [&](auto *p, int k, const float (&from)[V]) {
    typedef typename std::remove_reference<decltype(*p)>::type T;
    if (!TAIL || k + V <= a.D) Piece<T, V>::store(p + k, from);
    else store_some<T, V>(p + k, a.D - k, from);
  };
  auto load = [&](int64_t row, auto &ds, auto &de, auto &dz) {
    const int64_t at = row * a.D;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int k = (i * NT + t) * V;
      if (k < a.D) {
        if (!TAIL || (kReach ? at + k + V <= a.rows * a.D : k + V <= a.D)) {
          ds[i].load(static_cast<const S *>(a.s) + at + k);
          de[i].load(static_cast<const A *>(a.dy) + at + k);
          if ((!TAIL || kReach) && a.d_sum) dz[i].load(static_cast<const S *>(a.d_sum) + at + k);
        } else {
          ds[i].load_some(static_cast<const S *>(a.s) + at + k, a.D - k);
          de[i].load_some(static_cast<const A *>(a.dy) + at + k, a.D - k);
          if (kReach && a.d_sum) dz[i].load_some(static_cast<const S *>(a.d_sum) + at + k, a.D - k);
        }
      }
    }
  };
  int turn = 0;
  if (kAhead && r0 < a.rows) load(r0, sn, en, zn);
  for (int64_t row = r0; row < a.rows; row += stride, turn ^= 1) {
    const int64_t at = row * a.D;
    if constexpr (kAhead) {
#pragma unroll
      for (int i = 0; i < NC; ++i) { s[i] = sn[i]; e[i] = en[i]; z[i] = zn[i]; }
      if (row + stride < a.rows) load(row + stride, sn, en, zn);
    } else {
      load(row, s, e, z);
    }
    float sq = 0.f, gs = 0.f;
#pragma unroll
    for (int i = 0; i < NC; ++i)
      if ((i * NT + t) * V < a.D) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const bool in = !kReach || (i * NT + t) * V + j < a.D;
          const float f = in ? s[i][j] : 0.f;
          sq = fmaf(f, f, sq);
          gs = fmaf(gam[i][j] * (in ? e[i][j] : 0.f), f, gs);
        }
      }
    row_sum2<NT>(sq, gs, box[turn]);
    const float r = rsqrtf(sq / static_cast<float>(a.D) + a.eps);
    const float c = gs * r * inv_d;          // mean(g s r)
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int k = (i * NT + t) * V;
      if (k < a.D) {
        if constexpr (TAIL && !kReach) {
          const S *from = static_cast<const S *>(a.d_sum) + at + k;
          if (a.d_sum && k + V <= a.D) z[i].load(from);
          else if (a.d_sum) z[i].load_some(from, a.D - k);
        }
        float o[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float h = s[i][j] * r;
          acc[i][j] = fmaf(e[i][j], h, acc[i][j]);
          o[j] = r * (gam[i][j] * e[i][j] - h * c);
          if (a.d_sum) o[j] += z[i][j];
        }
        store(static_cast<S *>(a.dx) + at, k, o);
        if (a.d_delta) store(static_cast<A *>(a.d_delta) + at, k, o);
      }
    }
  }
  float *out = a.partial + static_cast<int64_t>(blockIdx.x) * a.D;
  if constexpr (RPB > 1) {                   // the row groups' sums, added in their order
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) sm[part][(i * NT + t) * V + j] = acc[i][j];
    __syncthreads();
    for (int k = threadIdx.x; k < a.D; k += 256) {
      float v = sm[0][k];
#pragma unroll
      for (int p = 1; p < RPB; ++p) v += sm[p][k];
      out[k] = v;
    }
  } else {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int k = (i * NT + t) * V;
      if (k < a.D) store(out, k, acc[i]);
    }
  }
}

constexpr int kNormMaxD = 16384;
constexpr int kNormBwdGroups = 768;       // three work-groups for every compute unit (512 to 2048 are within 5 %)

static int64_t norm_bwd_groups(int64_t rows) { return rows < kNormBwdGroups ? rows : kNormBwdGroups; }

// Threads that share a row of D features and pieces of V that each holds: a wave, four or sixteen, with up to 16 features a thread
// (the gradient keeps five values for each).
template <int V, class F>
static void norm_shape(int D, F &&f) {
  using std::integral_constant;
  auto fits = [&](auto nt, auto nc) {
    if (D > decltype(nt)::value * decltype(nc)::value * V) return false;
    f(nt, nc);
    return true;
  };
  typedef integral_constant<int, 64> Wave;
  typedef integral_constant<int, 256> Four;
  typedef integral_constant<int, 1024> Sixteen;
  typedef integral_constant<int, 16 / V> Full;
  typedef integral_constant<int, 8 / V> Part;
  (void)(fits(Wave{}, integral_constant<int, 1>{}) || fits(Wave{}, Part{}) || fits(Wave{}, Full{}) || fits(Four{}, Part{}) || fits(Four{}, Full{}) ||
         fits(Sixteen{}, Part{}) || fits(Sixteen{}, Full{}));
}

template <class S, class A, class Y, int V, bool TAIL>
static hipError_t launch_norm_v(NormArgs a, hipStream_t st) {
  auto past = [](auto *p, int64_t bytes) { return p ? reinterpret_cast<decltype(p)>(reinterpret_cast<uintptr_t>(p) + bytes) : p; };
  hipError_t e = hipSuccess;
  norm_shape<V>(a.D, [&](auto nt, auto nc) {
    constexpr int NT = decltype(nt)::value, NC = decltype(nc)::value, RPB = NT < 256 ? 256 / NT : 1, THREADS = NT < 256 ? 256 : NT;
    for (int64_t left = a.rows; left > 0 && e == hipSuccess;) {
      const int64_t n = std::min(left, most_groups(THREADS) * RPB), at = n * a.D;
      a.rows = n;
      rmsnorm_kernel<S, A, Y, V, NT, NC, TAIL><<<dim3(static_cast<unsigned>((n + RPB - 1) / RPB)), dim3(THREADS), 0, st>>>(a);
      e = hipGetLastError();
      a.x = past(a.x, at * sizeof(S)); a.sum = past(a.sum, at * sizeof(S)); a.delta = past(a.delta, at * sizeof(A));
      a.y = past(a.y, at * sizeof(Y)); a.y_scale = past(a.y_scale, n * sizeof(float));
      left -= n;
    }
  });
  return e;
}
// pieces of 16 bytes of the stream, from any address on
template <class S, class A, class Y>
static hipError_t launch_norm(const NormArgs &a, hipStream_t st) {
  constexpr int V = 16 / sizeof(S);
  return a.D % V ? launch_norm_v<S, A, Y, V, true>(a, st) : launch_norm_v<S, A, Y, V, false>(a, st);
}

template <class S, class A, int V, bool TAIL>
static hipError_t launch_norm_bwd_v(NormBwdArgs a, float *dgamma, hipStream_t st) {
  int64_t groups = 0;
  if (a.rows > 0) {
    norm_shape<V>(a.D, [&](auto nt, auto nc) {
      constexpr int NT = decltype(nt)::value, NC = decltype(nc)::value, RPB = NT < 256 ? 256 / NT : 1;
      groups = norm_bwd_groups((a.rows + RPB - 1) / RPB);
      if (groups == 1) a.partial = dgamma;
      rmsnorm_bwd_kernel<S, A, V, NT, NC, TAIL><<<dim3(static_cast<unsigned>(groups)), dim3(NT < 256 ? 256 : NT), 0, st>>>(a);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || groups == 1) return e;
  }
  return launch_partial_reduce(a.partial, dgamma, static_cast<int>(groups), a.D, a.D, st);      // no rows: zeros
}
template <class S, class A>
static hipError_t launch_norm_bwd(const NormBwdArgs &a, float *dgamma, hipStream_t st) {
  constexpr int V = 16 / sizeof(S);
  return a.D % V ? launch_norm_bwd_v<S, A, V, true>(a, dgamma, st) : launch_norm_bwd_v<S, A, V, false>(a, dgamma, st);
}

static int norm_check(const char *fn, int64_t rows, int D, float eps, int stream_dtype, int act_dtype) {
  if (rows < 0 || rows > INT32_MAX || D < 1 || D > kNormMaxD) return refuse(RESLIM_ESHAPE, fn, "need 0 <= rows < 2^31 and 1 <= D <= 16384");
  if (!(eps >= 0.f) || eps > 3.402823466e+38f) return refuse(RESLIM_EINVAL, fn, "eps must be finite and not negative");
  const bool types = (stream_dtype == RESLIM_F32 && (act_dtype == RESLIM_F32 || act_dtype == RESLIM_BF16)) || (stream_dtype == RESLIM_BF16 && act_dtype == RESLIM_BF16);
  return types ? RESLIM_OK : refuse(RESLIM_EINVAL, fn, "types must be (stream, act) = (F32, F32), (F32, BF16) or (BF16, BF16)");
}

}  // namespace reslim

using namespace reslim;

extern "C" int reslim_rmsnorm_fwd(const void *x, const void *delta, const float *gamma, float eps, int64_t rows, int32_t D, int32_t stream_dtype,
                                  int32_t act_dtype, int32_t y_dtype, void *sum, void *y, float *y_scale, void *hip_stream) {
  const char *fn = "reslim_rmsnorm_fwd";
  const int rc = norm_check(fn, rows, D, eps, stream_dtype, act_dtype);
  if (rc != RESLIM_OK) return rc;
  if (y_dtype != act_dtype && y_dtype != RESLIM_E4M3) return refuse(RESLIM_EINVAL, fn, "y must have the activation type or be E4M3");
  if ((y_dtype == RESLIM_E4M3) != (y_scale != nullptr)) return refuse(RESLIM_EINVAL, fn, "y_scale goes with E4M3 output, and only with it");
  if (!gamma || (rows > 0 && (!x || !y))) return refuse(RESLIM_EINVAL, fn, "null buffer");
  const size_t es = type_bytes(stream_dtype), ea = type_bytes(act_dtype);
  if (!aligned(x, es) || !aligned(sum, es) || !aligned(delta, ea) || !aligned(y, type_bytes(y_dtype)) || !aligned(gamma, 4) || !aligned(y_scale, 4))
    return refuse(RESLIM_EINVAL, fn, "a buffer is not aligned to its elements");
  if (rows == 0) return RESLIM_OK;
  const NormArgs a = {x, delta, gamma, sum, y, y_scale, eps, rows, D};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  hipError_t e;
  const bool q = y_dtype == RESLIM_E4M3;
  if (stream_dtype == RESLIM_BF16) e = q ? launch_norm<bf16_t, bf16_t, e4m3_t>(a, st) : launch_norm<bf16_t, bf16_t, bf16_t>(a, st);
  else if (act_dtype == RESLIM_BF16) e = q ? launch_norm<float, bf16_t, e4m3_t>(a, st) : launch_norm<float, bf16_t, bf16_t>(a, st);
  else e = q ? launch_norm<float, float, e4m3_t>(a, st) : launch_norm<float, float, float>(a, st);
  return e == hipSuccess ? RESLIM_OK : refuse_hip(fn, e);
}

extern "C" int reslim_rmsnorm_bwd_workspace_bytes(int64_t rows, int32_t D, size_t *out) {
  const char *fn = "reslim_rmsnorm_bwd_workspace_bytes";
  if (!out) return refuse(RESLIM_EINVAL, fn, "null argument");
  const int rc = norm_check(fn, rows, D, 0.f, RESLIM_F32, RESLIM_F32);
  if (rc != RESLIM_OK) return rc;
  *out = align256(static_cast<size_t>(norm_bwd_groups(rows)) * D * sizeof(float));
  return RESLIM_OK;
}

extern "C" int reslim_rmsnorm_bwd(const void *sum, const void *dy, const float *gamma, float eps, const void *d_sum, int64_t rows, int32_t D,
                                  int32_t stream_dtype, int32_t act_dtype, void *dx, void *d_delta, float *dgamma, void *workspace,
                                  size_t ws_bytes, void *hip_stream) {
  const char *fn = "reslim_rmsnorm_bwd";
  const int rc = norm_check(fn, rows, D, eps, stream_dtype, act_dtype);
  if (rc != RESLIM_OK) return rc;
  if (!gamma || !dgamma || (rows > 0 && (!sum || !dy || !dx))) return refuse(RESLIM_EINVAL, fn, "null buffer");
  const size_t es = type_bytes(stream_dtype), ea = type_bytes(act_dtype);
  if (!aligned(sum, es) || !aligned(d_sum, es) || !aligned(dx, es) || !aligned(dy, ea) || !aligned(d_delta, ea) || !aligned(gamma, 4) || !aligned(dgamma, 4))
    return refuse(RESLIM_EINVAL, fn, "a buffer is not aligned to its elements");
  if (rows > 1 && (!workspace || !aligned(workspace, 256) || ws_bytes < align256(static_cast<size_t>(norm_bwd_groups(rows)) * D * sizeof(float))))
    return refuse(RESLIM_EWORKSPACE, fn, "workspace null, not 256-byte aligned or smaller than reslim_rmsnorm_bwd_workspace_bytes()");
  const NormBwdArgs a = {sum, dy, d_sum, gamma, dx, d_delta, static_cast<float *>(workspace), eps, rows, D};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  hipError_t e;
  if (stream_dtype == RESLIM_BF16) e = launch_norm_bwd<bf16_t, bf16_t>(a, dgamma, st);
  else if (act_dtype == RESLIM_BF16) e = launch_norm_bwd<float, bf16_t>(a, dgamma, st);
  else e = launch_norm_bwd<float, float>(a, dgamma, st);
  return e == hipSuccess ? RESLIM_OK : refuse_hip(fn, e);
}
