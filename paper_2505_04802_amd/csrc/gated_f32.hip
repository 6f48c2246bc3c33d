// The gated feed-forward layer's products on the fp32 path, for small problems and parity: any sizes, any operand order.
//
//   C[m, n] = sum_k A(m, k) B(n, k), fp32 matrix instructions (v_mfma_f32_32x32x2), tiles of 128 x 64, slabs of 16 k staged through
// LDS as [row][k] whichever way the operands lie in memory, so that one kernel serves the forward products, the gradients of
// their inputs (B read across its rows) and of the weights (both read across, the sum over the tokens cut into slices that are
// added in order where there are few tiles).  A gated tile is 32 gate and 32 up rows of the same features.
#include <algorithm>
#include <type_traits>

#include "gated.h"

namespace reslim {
namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16;

enum F32Kind { kPlain, kGate, kDGate };
struct F32Args {
  const float *a, *b, *bias, *gu;      // gu: kDGate, what the forward kept
  float *out, *keep;                   // keep: kGate, [gate | up] or null
  int M, N, K;                         // kGate, kDGate: N features, with 2 N columns of gu
  int64_t a_step, b_step;              // elements from row to row (k contiguous) or from k to k (rows contiguous)
  int k_per;                           // k of a slice, a multiple of 16
  int64_t slice;                       // floats between the slices' results
};

constexpr int kBM = 128, kBN = 64, kBK = 16, kPitch = 20;      // rows of 20 floats: the 16-byte reads of 8 rows fall into different banks

// one operand's slab: ROWS x 16 values, `row0` its first row of `rows`, `k0` .. `k_end`; a thread holds ROWS / 16 of them
template <int ROWS, bool ALONG_K>
struct Slab {
  static constexpr int kEach = ROWS / 16;
  float v[kEach];
  template <class RowOf>
  __device__ __forceinline__ void load(const float *p, int64_t step, bool vec, int k0, int k_end, RowOf &&row_of) {
    const int t = threadIdx.x;
    if constexpr (ALONG_K) {                 // 16 / kEach threads to a row, each kEach consecutive k
      constexpr int PER = kBK / kEach;
      const int row = row_of(t / PER), k = k0 + t % PER * kEach;
      const float *q = p + static_cast<int64_t>(row) * step + k;
      if (vec && row >= 0 && k + kEach <= k_end) {
#pragma unroll
        for (int i = 0; i < kEach; i += 4) {
          const float4 f = *reinterpret_cast<const float4 *>(q + i);
          v[i] = f.x; v[i + 1] = f.y; v[i + 2] = f.z; v[i + 3] = f.w;
        }
      } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i) v[i] = row >= 0 && k + i < k_end ? q[i] : 0.f;
      }
    } else {                                 // sixteen threads to a k, each kEach consecutive rows
      const int k = k0 + t / 16, first = t % 16 * kEach;
      const bool in = k < k_end;
      const int r0 = row_of(first), r1 = row_of(first + kEach - 1);
      const float *q = p + static_cast<int64_t>(in ? k : 0) * step;
      if (vec && in && r0 >= 0 && r1 == r0 + kEach - 1) {
#pragma unroll
        for (int i = 0; i < kEach; i += 4) {
          const float4 f = *reinterpret_cast<const float4 *>(q + r0 + i);
          v[i] = f.x; v[i + 1] = f.y; v[i + 2] = f.z; v[i + 3] = f.w;
        }
      } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          const int r = row_of(first + i);
          v[i] = in && r >= 0 ? q[r] : 0.f;
        }
      }
    }
  }
  __device__ __forceinline__ void store(float *lds) const {
    const int t = threadIdx.x;
    if constexpr (ALONG_K) {
      constexpr int PER = kBK / kEach;
      float *q = lds + t / PER * kPitch + t % PER * kEach;
#pragma unroll
      for (int i = 0; i < kEach; i += 4) *reinterpret_cast<float4 *>(q + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    } else {
#pragma unroll
      for (int i = 0; i < kEach; ++i) lds[(t % 16 * kEach + i) * kPitch + t / 16] = v[i];
    }
  }
};

template <F32Kind KIND, bool GELU, bool A_ALONG, bool B_ALONG>
__global__ __launch_bounds__(256) void gated_f32_kernel(F32Args g) {
  __shared__ __align__(16) float As[kBM * kPitch], Bs[kBN * kPitch];
  constexpr int BNO = KIND == kGate ? kBN / 2 : kBN;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l32 = lane & 31, hi = lane >> 5;
  const int n0 = blockIdx.x * BNO, m0 = blockIdx.y * kBM;
  const int k_begin = blockIdx.z * g.k_per, k_end = min(g.K, k_begin + g.k_per);
  auto a_row = [&](int r) { return m0 + r < g.M ? m0 + r : -1; };
  auto b_row = [&](int r) {
    if constexpr (KIND == kGate) return n0 + (r & 31) < g.N ? n0 + (r & 31) + (r & 32 ? g.N : 0) : -1;
    else return n0 + r < g.N ? n0 + r : -1;
  };
  const bool a_vec = g.a_step % 4 == 0 && (reinterpret_cast<uintptr_t>(g.a) & 15) == 0;
  // rows of a gated tile's halves start anywhere when N is no multiple of four
  const bool b_vec = g.b_step % 4 == 0 && (reinterpret_cast<uintptr_t>(g.b) & 15) == 0 && (B_ALONG || KIND != kGate || g.N % 4 == 0);
  Slab<kBM, A_ALONG> sa;
  Slab<kBN, B_ALONG> sb;
  f32x16 acc[2] = {};
  sa.load(g.a, g.a_step, a_vec, k_begin, k_end, a_row);
  sb.load(g.b, g.b_step, b_vec, k_begin, k_end, b_row);
  for (int k0 = k_begin; k0 < k_end; k0 += kBK) {
    __syncthreads();
    sa.store(As);
    sb.store(Bs);
    __syncthreads();
    if (k0 + kBK < k_end) {
      sa.load(g.a, g.a_step, a_vec, k0 + kBK, k_end, a_row);
      sb.load(g.b, g.b_step, b_vec, k0 + kBK, k_end, b_row);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const float4 x = *reinterpret_cast<const float4 *>(&As[(wave * 32 + l32) * kPitch + 8 * s + 4 * hi]);
      float4 w[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) w[j] = *reinterpret_cast<const float4 *>(&Bs[(j * 32 + l32) * kPitch + 8 * s + 4 * hi]);
#pragma unroll
      for (int j = 0; j < 2; ++j) {          // operands swapped: the block is C^T
        acc[j] = __builtin_amdgcn_mfma_f32_32x32x2f32(w[j].x, x.x, acc[j], 0, 0, 0);
        acc[j] = __builtin_amdgcn_mfma_f32_32x32x2f32(w[j].y, x.y, acc[j], 0, 0, 0);
        acc[j] = __builtin_amdgcn_mfma_f32_32x32x2f32(w[j].z, x.z, acc[j], 0, 0, 0);
        acc[j] = __builtin_amdgcn_mfma_f32_32x32x2f32(w[j].w, x.w, acc[j], 0, 0, 0);
      }
    }
  }
  // register r of a block: row l32, column 8 (r / 4) + 4 hi + r % 4
  const int m = m0 + wave * 32 + l32;
  if (m >= g.M) return;
  if constexpr (KIND == kGate) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int n = n0 + 8 * (r / 4) + 4 * hi + r % 4;
      if (n >= g.N) continue;
      const float gate = acc[0][r] + (g.bias ? g.bias[n] : 0.f), up = acc[1][r] + (g.bias ? g.bias[g.N + n] : 0.f);
      if (g.keep) {
        g.keep[static_cast<int64_t>(m) * 2 * g.N + n] = gate;
        g.keep[static_cast<int64_t>(m) * 2 * g.N + g.N + n] = up;
      }
      g.out[static_cast<int64_t>(m) * g.N + n] = gate_act_f32<GELU>(gate) * up;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int n = n0 + j * 32 + 8 * (r / 4) + 4 * hi + r % 4;
        if (n >= g.N) continue;
        if constexpr (KIND == kDGate) {
          const int64_t at = static_cast<int64_t>(m) * 2 * g.N + n;
          float act, slope;
          gate_act_slope_f32<GELU>(g.gu[at], act, slope);
          g.out[at] = acc[j][r] * g.gu[at + g.N] * slope;
          g.out[at + g.N] = acc[j][r] * act;
        } else {
          g.out[blockIdx.z * g.slice + static_cast<int64_t>(m) * g.N + n] = acc[j][r] + (g.bias ? g.bias[n] : 0.f);
        }
      }
  }
}

// column sums of a [rows, N] matrix, a slab of rows for each work-group of 64 columns: partial [slabs, N]
constexpr int kSumRows = 256;
__global__ __launch_bounds__(256) void gated_colsum_kernel(const float *__restrict__ a, float *__restrict__ partial, int64_t rows, int N) {
  __shared__ float sm[4][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), grp = threadIdx.x >> 6;
  const int64_t r0 = static_cast<int64_t>(blockIdx.y) * kSumRows, r1 = min(rows, r0 + kSumRows);
  float s = 0.f;
  if (c < N)
    for (int64_t r = r0 + grp; r < r1; r += 4) s += a[r * N + c];
  sm[grp][threadIdx.x & 63] = s;
  __syncthreads();
  if (grp == 0 && c < N) partial[static_cast<int64_t>(blockIdx.y) * N + c] = (sm[0][threadIdx.x] + sm[1][threadIdx.x]) + (sm[2][threadIdx.x] + sm[3][threadIdx.x]);
}

template <F32Kind KIND, bool GELU, bool A_ALONG, bool B_ALONG>
hipError_t launch(F32Args g, int splits, hipStream_t st) {
  constexpr int BNO = KIND == kGate ? kBN / 2 : kBN;
  const int64_t gm = (static_cast<int64_t>(g.M) + kBM - 1) / kBM;
  if (gm > 65535 || splits > 65535) return hipErrorInvalidValue;
  gated_f32_kernel<KIND, GELU, A_ALONG, B_ALONG><<<dim3((g.N + BNO - 1) / BNO, static_cast<unsigned>(gm), splits), dim3(256), 0, st>>>(g);
  return hipGetLastError();
}
F32Args whole(const float *a, int64_t a_step, const float *b, int64_t b_step, float *out, int M, int N, int K) {
  F32Args g = {};
  g.a = a; g.b = b; g.out = out; g.M = M; g.N = N; g.K = K; g.a_step = a_step; g.b_step = b_step;
  g.k_per = (K + kBK - 1) / kBK * kBK;
  return g;
}

// Slices of the tokens: as many as give every compute unit two tiles, of at least 256 tokens each.
int wgrad_slices(int M, int N, int K) {
  const int64_t tiles = (static_cast<int64_t>(N) + kBM - 1) / kBM * ((static_cast<int64_t>(K) + kBN - 1) / kBN);
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(512 / tiles, M / 256)));
}
int sum_slabs(int M) { return (M + kSumRows - 1) / kSumRows; }

}  // namespace

hipError_t launch_gated_f32_in(const GatedIn &in, bool gelu, hipStream_t st) {
  F32Args g = whole(static_cast<const float *>(in.x), in.D, static_cast<const float *>(in.w_in), in.D, static_cast<float *>(in.h), in.M, in.R, in.D);
  g.bias = in.b_in;
  g.keep = static_cast<float *>(in.gu);
  return gelu ? launch<kGate, true, true, true>(g, 1, st) : launch<kGate, false, true, true>(g, 1, st);
}
hipError_t launch_gated_f32_out(const float *h, const float *w_out, const float *b_out, float *y, int M, int D, int R, hipStream_t st) {
  F32Args g = whole(h, R, w_out, R, y, M, D, R);
  g.bias = b_out;
  return launch<kPlain, false, true, true>(g, 1, st);
}
hipError_t launch_gated_f32_dgate(const float *dy, const float *w_out, const float *gu, float *d_gu, int M, int D, int R, bool gelu, hipStream_t st) {
  F32Args g = whole(dy, D, w_out, R, d_gu, M, R, D);
  g.gu = gu;
  return gelu ? launch<kDGate, true, true, false>(g, 1, st) : launch<kDGate, false, true, false>(g, 1, st);
}
hipError_t launch_gated_f32_dx(const float *d_gu, const float *w_in, float *dx, int M, int D, int R, hipStream_t st) {
  return launch<kPlain, false, true, false>(whole(d_gu, 2 * static_cast<int64_t>(R), w_in, D, dx, M, D, 2 * R), 1, st);
}
size_t gated_f32_wgrad_bytes(int M, int N, int K) {
  const int s = wgrad_slices(M, N, K);
  const size_t dw = s > 1 ? static_cast<size_t>(s) * N * K : 0, db = static_cast<size_t>(sum_slabs(M)) * N;
  return align256(std::max(dw, db) * sizeof(float));
}
hipError_t launch_gated_f32_wgrad(const float *dy, const float *x, float *dw, float *db, int M, int N, int K, void *ws, hipStream_t st) {
  int s = wgrad_slices(M, N, K);
  F32Args g = whole(dy, N, x, K, dw, N, K, M);
  g.k_per = ((M + s - 1) / s + kBK - 1) / kBK * kBK;
  s = (M + g.k_per - 1) / g.k_per;
  float *part = static_cast<float *>(ws);
  if (s > 1) {
    g.out = part;
    g.slice = static_cast<int64_t>(N) * K;
  }
  hipError_t e = launch<kPlain, false, false, false>(g, s, st);
  if (e == hipSuccess && s > 1) e = launch_partial_reduce(part, dw, s, g.slice, g.slice, st);
  if (e != hipSuccess || !db) return e;
  const int slabs = sum_slabs(M);
  if (slabs > 65535) return hipErrorInvalidValue;
  gated_colsum_kernel<<<dim3((N + 63) / 64, slabs), dim3(256), 0, st>>>(dy, part, M, N);
  e = hipGetLastError();
  return e == hipSuccess ? launch_partial_reduce(part, db, slabs, N, N, st) : e;
}

}  // namespace reslim
