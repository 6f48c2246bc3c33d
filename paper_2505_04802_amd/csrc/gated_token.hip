// The gated feed-forward layer for few rows (single tokens of a batch of sequences): the weights are read once and bound it.
//
// A work-group owns 16 features of the output (with gate and up rows 32 rows of W) and all of K, its waves a run of K each, so
// that every wave streams its part of the rows from memory straight into matrix instructions of 16 x 16: A operand 16 rows of W, B
// operand up to 16 token rows, 16 bytes a lane and row, 64 bytes of a row a step.  Several steps' loads are in flight while the ones
// before are multiplied.  The waves' sums meet in LDS, are added in wave order, and the epilogue (scales, biases, activation, product) runs
// there.  The token rows come out of the caches.  One code for bf16, e4m3 and fp32: only the multiplication differs.
#include <algorithm>
#include <type_traits>

#include "gated.h"

namespace reslim {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) long i64x2;

struct TokenArgs {
  const unsigned char *x, *w;
  const float *x_scale, *w_scale, *bias;
  void *out, *keep;            // keep: gated, [gate | up] or null
  int M, N, row_bytes;         // N: rows of one weight matrix
};

// 16 bytes of a row of W and of a token row, the same k: 32 bf16, 64 e4m3 or 16 fp32 of them over the four lane groups
template <class T>
__device__ __forceinline__ f32x4 multiply(const u32x4 &w, const u32x4 &x, f32x4 acc) {
  if constexpr (std::is_same<T, bf16_t>::value) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), acc, 0, 0, 0);
  } else if constexpr (std::is_same<T, e4m3_t>::value) {
    const i64x2 a = __builtin_bit_cast(i64x2, w), b = __builtin_bit_cast(i64x2, x);
    acc = __builtin_amdgcn_mfma_f32_16x16x32_fp8_fp8(a[0], b[0], acc, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_fp8_fp8(a[1], b[1], acc, 0, 0, 0);
  } else {
    const f32x4 a = __builtin_bit_cast(f32x4, w), b = __builtin_bit_cast(f32x4, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], acc, 0, 0, 0);
    return acc;
  }
}

// P = 2: gate and up rows; P = 1: the output map.  MT: tiles of 16 token rows.  NW: waves.  O: type of the results.
template <class T, class O, int P, bool GELU, int MT, int NW>
__global__ __launch_bounds__(NW * 64) void gated_token_kernel(TokenArgs a) {
  constexpr int U = MT == 4 ? 2 : 4;           // steps whose loads are in flight together
  __shared__ float part[NW][P * MT * 4][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r16 = lane & 15, kg = lane >> 4;
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * MT;
  const int steps = a.row_bytes / 64, per = (steps + NW - 1) / NW;
  const int s0 = wave * per, s1 = min(steps, s0 + per);
  const unsigned char *w[P], *x[MT];
#pragma unroll
  for (int p = 0; p < P; ++p) w[p] = a.w + (static_cast<size_t>(p) * a.N + min(n0 + r16, a.N - 1)) * a.row_bytes + kg * 16;
#pragma unroll
  for (int i = 0; i < MT; ++i) x[i] = a.x + static_cast<size_t>(min(m0 + 16 * i + r16, a.M - 1)) * a.row_bytes + kg * 16;
  f32x4 acc[P][MT] = {};
  u32x4 wr[2][U][P], xr[2][U][MT];
  auto fetch = [&](auto to, int s) {           // steps past the wave's last read it again and are not multiplied
    constexpr int B = decltype(to)::value;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const size_t at = static_cast<size_t>(min(s + u, s1 - 1)) * 64;
#pragma unroll
      for (int p = 0; p < P; ++p) wr[B][u][p] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(w[p] + at));
#pragma unroll
      for (int i = 0; i < MT; ++i) xr[B][u][i] = *reinterpret_cast<const u32x4 *>(x[i] + at);
    }
  };
  auto use = [&](auto from, int s) {
    constexpr int B = decltype(from)::value;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (s + u < s1) {                        // uniform
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int p = 0; p < P; ++p) acc[p][i] = multiply<T>(wr[B][u][p], xr[B][u][i], acc[p][i]);
      }
  };
  typedef std::integral_constant<int, 0> I0;
  typedef std::integral_constant<int, 1> I1;
  if (s0 < s1) {                               // uniform; K may have fewer steps than waves
    fetch(I0{}, s0);
    for (int s = s0; s < s1; s += 2 * U) {
      fetch(I1{}, s + U);
      use(I0{}, s);
      fetch(I0{}, s + 2 * U);
      use(I1{}, s + U);
    }
  }
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) part[wave][(p * MT + i) * 4 + r][lane] = acc[p][i][r];
  __syncthreads();
  // value (m, n) of the block: register n % 4 of lane 16 (n / 4) + m % 16 of tile m / 16
  for (int e = threadIdx.x; e < MT * 256; e += NW * 64) {
    const int ml = e >> 4, nl = e & 15, m = m0 + ml, n = n0 + nl;
    if (m >= a.M || n >= a.N) continue;
    float v[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int q = (p * MT + (ml >> 4)) * 4 + (nl & 3), l = ((nl >> 2) << 4) | (ml & 15);
      v[p] = part[0][q][l];
#pragma unroll
      for (int k = 1; k < NW; ++k) v[p] += part[k][q][l];
      if constexpr (std::is_same<T, e4m3_t>::value) v[p] *= a.x_scale[m] * a.w_scale[p * a.N + n];
      if (a.bias) v[p] += a.bias[p * a.N + n];
    }
    O *out = static_cast<O *>(a.out);
    if constexpr (P == 2) {
      if (a.keep) {
        O *gu = static_cast<O *>(a.keep) + static_cast<size_t>(m) * 2 * a.N + n;
        Act<O>::store(gu, v[0]);
        Act<O>::store(gu + a.N, v[1]);
      }
      const float act = std::is_same<O, float>::value ? gate_act_f32<GELU>(v[0]) : gate_act<GELU>(v[0]);
      Act<O>::store(out + static_cast<size_t>(m) * a.N + n, act * v[1]);
    } else {
      Act<O>::store(out + static_cast<size_t>(m) * a.N + n, v[0]);
    }
  }
}

template <class T, class O, int P, bool GELU, int NW>
hipError_t launch_rows(const TokenArgs &a, hipStream_t st) {
  const int mt = a.M <= 16 ? 1 : a.M <= 32 ? 2 : 4;
  const int64_t gy = (static_cast<int64_t>(a.M) + 16 * mt - 1) / (16 * mt);
  if (gy > 65535) return hipErrorInvalidValue;
  const dim3 grid((a.N + 15) / 16, static_cast<unsigned>(gy)), blk(NW * 64);
  if (mt == 1) gated_token_kernel<T, O, P, GELU, 1, NW><<<grid, blk, 0, st>>>(a);
  else if (mt == 2) gated_token_kernel<T, O, P, GELU, 2, NW><<<grid, blk, 0, st>>>(a);
  else gated_token_kernel<T, O, P, GELU, 4, NW><<<grid, blk, 0, st>>>(a);
  return hipGetLastError();
}
template <class T, class O>
hipError_t launch_in(const TokenArgs &a, bool gelu, hipStream_t st) {
  return gelu ? launch_rows<T, O, 2, true, 8>(a, st) : launch_rows<T, O, 2, false, 8>(a, st);
}

}  // namespace

hipError_t launch_gated_token_in(int x_dtype, const GatedIn &g, bool gelu, hipStream_t st) {
  const size_t row = static_cast<size_t>(g.D) * type_bytes(x_dtype);
  if (g.M < 1 || row % 64 || row > INT32_MAX) return hipErrorInvalidValue;
  const TokenArgs a = {static_cast<const unsigned char *>(g.x), static_cast<const unsigned char *>(g.w_in), g.x_scale, g.in_scale, g.b_in, g.h, g.gu, g.M, g.R, static_cast<int>(row)};
  if (x_dtype == RESLIM_BF16) return launch_in<bf16_t, bf16_t>(a, gelu, st);
  if (x_dtype == RESLIM_E4M3) return launch_in<e4m3_t, bf16_t>(a, gelu, st);
  return launch_in<float, float>(a, gelu, st);
}

hipError_t launch_gated_token_out(int dtype, const void *h, const void *w_out, const float *b_out, void *y, int M, int D, int R, hipStream_t st) {
  const size_t row = static_cast<size_t>(R) * type_bytes(dtype);
  if (M < 1 || row % 64 || row > INT32_MAX) return hipErrorInvalidValue;
  const TokenArgs a = {static_cast<const unsigned char *>(h), static_cast<const unsigned char *>(w_out), nullptr, nullptr, b_out, y, nullptr, M, D, static_cast<int>(row)};
  return dtype == RESLIM_BF16 ? launch_rows<bf16_t, bf16_t, 1, false, 16>(a, st) : launch_rows<float, float, 1, false, 16>(a, st);
}

}  // namespace reslim
