// The gated feed-forward layer's products on the fp32 path, for small problems and parity: any sizes, any operand order.
//
//   C[m, n] = sum_k A(m, k) B(n, k), fp32 matrix instructions (v_mfma_f32_32x32x2), tiles of 64 x 64 with a 32 x 32 block for each of
// four waves, slabs of 32 k in two LDS buffers, the slab after the next in flight in registers.  An operand whose k is contiguous is staged as
// [row][k], one whose rows are as [k][row], so that one kernel serves the forward products, the gradients of their inputs (B
// read across its rows) and of the weights (both read across, the bias gradient with them).  Where there are few tiles, k is cut into slices that
// are added in order.  A gated block is 16 gate and 16 up rows of the same features; lanes 16 apart exchange them.
//   The matrix instructions bound it: 16,384 x 2048 x 11,008 runs at 118 TFLOP/s, the library's 8192^3 at 153.  At 2048 x 512 x 1368 (one to four
// work-groups a compute unit) the forward takes 102 us and the gradient 225: 48 us for the hidden layer's (60 TFLOP/s, its epilogue
// moves 34 MB), 65 for the input's (88), 73 and 40 for the weights' (79, 72), 15 for the sums.
#include <algorithm>
#include <type_traits>

#include "gated.h"

namespace reslim {
namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4_any;      // four floats from any float on, one load all the same

enum F32Kind { kPlain, kGate, kDGate };
struct F32Args {
  const float *a, *b, *bias, *gu;      // gu: kDGate, what the forward kept
  float *out, *keep;                   // keep: kGate, [gate | up] or null
  int M, N, K;                         // kGate, kDGate: N features, with 2 N columns of gu
  int64_t a_step, b_step;              // elements from row to row (k contiguous) or from k to k (rows contiguous)
  int k_per;                           // k of a slice, a multiple of kBK
  int64_t slice;                       // floats between the slices' results
  float *sums;                         // kPlain with A read across: sums over k of A's rows [slices, M], or null
};

constexpr int kTile = 64, kBK = 32;
constexpr int kPitchK = 36, kPitchRow = 68;      // floats of a [row][k] row and of a [k][row] one: 16-byte accesses of neighbouring rows fall into different banks

// One operand's slabs of 64 x 32 values, eight of them a thread.  row_of: the operand's row for a row of the tile, or -1; step: elements from
// row to row (ALONG_K) or from k to k.  Rows that do not exist are read as others that do: they reach only results that are not stored.  No
// lane of a whole slab's loads takes a path of its own, so that they stay in flight over a slab's products: with a condition
// on every piece the compiler waited for one operand before it asked for the other.
template <bool ALONG_K>
struct Slab {
  static constexpr int kFloats = ALONG_K ? kTile * kPitchK : kBK * kPitchRow;
  f32x4 v[2];
  const float *at[2];          // this thread's first values of slab 0: ALONG_K four k of two rows, else four rows at two k
  int64_t step;
  int live;                    // k of the slab in v that exist, where not all do
  int k, last;                 // its first k in a slab; not ALONG_K: the last of its four rows that exists
  bool fours;                  // not ALONG_K: all or none of any thread's four rows exist
  template <class RowOf>
  __device__ __forceinline__ void start(const float *p, int64_t step_, int rows, RowOf &&row_of) {
    const int t = threadIdx.x;
    step = step_;
    if constexpr (ALONG_K) {                 // eight threads to a row
      k = t % 8 * 4;
#pragma unroll
      for (int j = 0; j < 2; ++j) at[j] = p + static_cast<int64_t>(max(row_of(t / 8 + 32 * j), 0)) * step + k;
    } else {                                 // sixteen threads to a k
      const int first = t % 16 * 4;
      k = t / 16;
      last = 0;
      fours = rows % 4 == 0 || row_of(kTile - 1) >= 0;
#pragma unroll
      for (int i = 1; i < 4; ++i) last += row_of(first + i) >= 0;
#pragma unroll
      for (int j = 0; j < 2; ++j) at[j] = p + static_cast<int64_t>(k + 16 * j) * step + max(row_of(first), 0);
    }
  }
  __device__ __forceinline__ void load(int k0, int k_end) {
    const float *q[2];
    live = k_end - k0;
    if (live >= kBK) {                       // uniform
#pragma unroll
      for (int j = 0; j < 2; ++j) q[j] = ALONG_K ? at[j] + k0 : at[j] + k0 * step;
      if (ALONG_K || fours) {                // uniform
#pragma unroll
        for (int j = 0; j < 2; ++j) v[j] = *reinterpret_cast<const f32x4_any *>(q[j]);
      } else {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) v[j][i] = q[j][min(i, last)];
      }
    } else {                                 // k past the end: the last one, zero in LDS
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        q[j] = ALONG_K ? at[j] + k0 - k : at[j] + (k0 + min(0, live - 1 - k - 16 * j)) * step;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[j][i] = q[j][ALONG_K ? min(k + i, live - 1) : min(i, last)];
      }
    }
  }
  __device__ __forceinline__ void store(float *lds) {
    const int t = threadIdx.x;
    if (live < kBK) {                        // uniform
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[j][i] = k + (ALONG_K ? i : 16 * j) < live ? v[j][i] : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
      *reinterpret_cast<f32x4 *>(lds + (ALONG_K ? (t / 8 + 32 * j) * kPitchK + t % 8 * 4 : (t / 16 + 16 * j) * kPitchRow + t % 16 * 4)) = v[j];
  }
  // four consecutive k of a row of the tile
  static __device__ __forceinline__ void read(const float *lds, int row, int k, float (&f)[4]) {
    if constexpr (ALONG_K) {
      const float4 x = *reinterpret_cast<const float4 *>(lds + row * kPitchK + k);
      f[0] = x.x; f[1] = x.y; f[2] = x.z; f[3] = x.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = lds[(k + i) * kPitchRow + row];
    }
  }
};

template <F32Kind KIND, bool GELU, bool A_ALONG, bool B_ALONG>
__global__ __launch_bounds__(256) void gated_f32_kernel(F32Args g) {
  __shared__ __align__(16) float As[2][Slab<A_ALONG>::kFloats], Bs[2][Slab<B_ALONG>::kFloats];
  constexpr int BNO = KIND == kGate ? kTile / 2 : kTile;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l32 = lane & 31, hi = lane >> 5, wm = wave >> 1, wn = wave & 1;
  const int n0 = blockIdx.x * BNO, m0 = blockIdx.y * kTile;
  const int k_begin = blockIdx.z * g.k_per, k_end = min(g.K, k_begin + g.k_per);
  auto a_row = [&](int r) { return m0 + r < g.M ? m0 + r : -1; };
  auto b_row = [&](int r) {
    if constexpr (KIND == kGate) {
      const int n = n0 + (r >> 5) * 16 + (r & 15);
      return n < g.N ? n + (r & 16 ? g.N : 0) : -1;
    } else {
      return n0 + r < g.N ? n0 + r : -1;
    }
  };
  static_assert(KIND != kGate || B_ALONG, "a gated tile's rows are not in a run");
  Slab<A_ALONG> sa;
  Slab<B_ALONG> sb;
  f32x16 acc = {};
  // sums over k of A's rows, in the work-groups of the first column tile, from the registers that the slabs pass through
  constexpr bool kSums = KIND == kPlain && !A_ALONG;
  const bool sums = kSums && g.sums && blockIdx.x == 0;
  float rs[kSums ? 4 : 1] = {};
  auto add = [&]() {
    if constexpr (kSums) {
      if (sums) {                            // uniform
#pragma unroll
        for (int i = 0; i < 4; ++i) rs[i] += sa.v[0][i] + sa.v[1][i];
      }
    }
  };
  sa.start(g.a, g.a_step, g.M, a_row);
  sb.start(g.b, g.b_step, g.N, b_row);
  sa.load(k_begin, k_end);
  sb.load(k_begin, k_end);
  sa.store(As[0]);
  sb.store(Bs[0]);
  add();
  if (k_begin + kBK < k_end) {
    sa.load(k_begin + kBK, k_end);
    sb.load(k_begin + kBK, k_end);
  }
  __syncthreads();
  // A slab's turn begins with its first reads and with the next slab's way from registers to the other buffer (last read before the barrier
  // that ended the slab before), so that nothing but the barrier stands between the products of two slabs.
  int buf = 0;
  for (int k0 = k_begin; k0 < k_end; k0 += kBK, buf ^= 1) {
    float x[kBK / 8][4], w[kBK / 8][4];
    auto read = [&](int s) {
      Slab<A_ALONG>::read(As[buf], wm * 32 + l32, 8 * s + 4 * hi, x[s]);
      Slab<B_ALONG>::read(Bs[buf], wn * 32 + l32, 8 * s + 4 * hi, w[s]);
    };
    auto multiply = [&](int s) {
#pragma unroll
      for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[s][i], w[s][i], acc, 0, 0, 0);
    };
    read(0);
    read(1);
    if (k0 + kBK < k_end) {
      sa.store(As[buf ^ 1]);
      sb.store(Bs[buf ^ 1]);
      add();
      if (k0 + 2 * kBK < k_end) {
        sa.load(k0 + 2 * kBK, k_end);
        sb.load(k0 + 2 * kBK, k_end);
      }
    }
    multiply(0);
    read(2);
    read(3);
    multiply(1);
    multiply(2);
    multiply(3);
    __syncthreads();
  }
  if constexpr (kSums) {
    if (sums) {                              // the 16 threads that share four rows, in their order
      float *part = As[0];                   // [16][64]
#pragma unroll
      for (int i = 0; i < 4; ++i) part[threadIdx.x / 16 * kTile + threadIdx.x % 16 * 4 + i] = rs[i];
      __syncthreads();
      const int r = m0 + static_cast<int>(threadIdx.x);
      if (threadIdx.x < kTile && r < g.M) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += part[i * kTile + threadIdx.x];
        g.sums[static_cast<int64_t>(blockIdx.z) * g.M + r] = s;
      }
    }
  }
  // register r of the block: row 8 (r / 4) + 4 hi + r % 4, column l32: a store writes runs of 32 columns of two rows
  const int row0 = m0 + wm * 32 + 4 * hi;
  auto row_of = [&](int r) { return row0 + 8 * (r / 4) + r % 4; };
  if constexpr (KIND == kGate) {
    // columns 0 .. 15 of the block are gates, 16 .. 31 the same features' up projections: the lanes of either half get the other value of eight rows
    const bool up_lane = l32 & 16;
    const int n = n0 + wn * 16 + (l32 & 15);
    const float bg = g.bias && n < g.N ? g.bias[n] : 0.f, bu = g.bias && n < g.N ? g.bias[g.N + n] : 0.f;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const float mine = up_lane ? acc[r + 8] : acc[r], other = __shfl_xor(up_lane ? acc[r] : acc[r + 8], 16);
      const float gate = (up_lane ? other : mine) + bg, up = (up_lane ? mine : other) + bu;
      const int m = row_of(up_lane ? r + 8 : r);
      if (m >= g.M || n >= g.N) continue;
      if (g.keep) {
        g.keep[static_cast<int64_t>(m) * 2 * g.N + n] = gate;
        g.keep[static_cast<int64_t>(m) * 2 * g.N + g.N + n] = up;
      }
      g.out[static_cast<int64_t>(m) * g.N + n] = gate_act_f32<GELU>(gate) * up;
    }
  } else {
    const int n = n0 + wn * 32 + l32;
    if (n >= g.N) return;
    const float bias = g.bias && blockIdx.z == 0 ? g.bias[n] : 0.f;      // the first slice brings the bias
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int m = row_of(r);
      if (m >= g.M) continue;
      if constexpr (KIND == kDGate) {
        const int64_t at = static_cast<int64_t>(m) * 2 * g.N + n;
        float act, slope;
        gate_act_slope_f32<GELU>(g.gu[at], act, slope);
        g.out[at] = acc[r] * g.gu[at + g.N] * slope;
        g.out[at + g.N] = acc[r] * act;
      } else {
        g.out[blockIdx.z * g.slice + static_cast<int64_t>(m) * g.N + n] = acc[r] + bias;
      }
    }
  }
}

template <F32Kind KIND, bool GELU, bool A_ALONG, bool B_ALONG>
hipError_t launch(const F32Args &g, int slices, hipStream_t st) {
  constexpr int BNO = KIND == kGate ? kTile / 2 : kTile;
  const int64_t gm = (static_cast<int64_t>(g.M) + kTile - 1) / kTile;
  if (gm > 65535 || slices > 65535) return hipErrorInvalidValue;
  gated_f32_kernel<KIND, GELU, A_ALONG, B_ALONG><<<dim3((g.N + BNO - 1) / BNO, static_cast<unsigned>(gm), slices), dim3(256), 0, st>>>(g);
  return hipGetLastError();
}
F32Args whole(const float *a, int64_t a_step, const float *b, int64_t b_step, float *out, int M, int N, int K) {
  F32Args g = {};
  g.a = a; g.b = b; g.out = out; g.M = M; g.N = N; g.K = K; g.a_step = a_step; g.b_step = b_step;
  g.k_per = (K + kBK - 1) / kBK * kBK;
  return g;
}

// out [n] and sums [m] (or null): the slices' values added in their order, four floats a thread
__global__ __launch_bounds__(256) void gated_f32_sum_kernel(const float *__restrict__ part, float *__restrict__ out, int64_t n, float *__restrict__ sums, int64_t m, int slices) {
  int64_t at = 4 * (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x);
  if (at >= n) {                             // whole work-groups take the product, the ones behind them the sums
    at -= (n + 1023) / 1024 * 1024;
    if (at < 0 || at >= m) return;
    part += slices * n;
    out = sums;
    n = m;
  }
  if (at + 4 <= n) {
    f32x4 s = *reinterpret_cast<const f32x4_any *>(part + at);
#pragma unroll 4
    for (int k = 1; k < slices; ++k) s += *reinterpret_cast<const f32x4_any *>(part + k * n + at);
    *reinterpret_cast<f32x4_any *>(out + at) = s;
  } else {
    for (; at < n; ++at) {
      float s = part[at];
      for (int k = 1; k < slices; ++k) s += part[k * n + at];
      out[at] = s;
    }
  }
}

// Slices of k: as many as fill the four work-groups that a compute unit holds, of at least three slabs each: a slab takes an empty chip about
// 1 us, the launch that adds the slices 2 to 5 (gradient of 673 x 83 x 363 46 us; with eight slabs 68, with two 45, but 69 for 65 at 3700 x 100 x 300).
int f32_slices(int M, int N, int K) {
  const int64_t tiles = (static_cast<int64_t>(M) + kTile - 1) / kTile * ((static_cast<int64_t>(N) + kTile - 1) / kTile);
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(1024 / tiles, K / (3 * kBK))));
}
size_t slice_bytes(int M, int N, int K, int more) {      // more: floats of a slice beside the product
  const int s = f32_slices(M, N, K);
  return s > 1 ? align256(static_cast<size_t>(s) * (static_cast<size_t>(M) * N + more) * sizeof(float)) : 0;
}
// C = A B^T (+ bias; with g.sums set also the sums of A's rows), in slices where that pays
template <bool A_ALONG, bool B_ALONG>
hipError_t product(F32Args g, float *part, hipStream_t st) {
  int s = f32_slices(g.M, g.N, g.K);
  g.k_per = ((g.K + s - 1) / s + kBK - 1) / kBK * kBK;
  s = (g.K + g.k_per - 1) / g.k_per;
  float *out = g.out, *sums = g.sums;
  const int64_t n = static_cast<int64_t>(g.M) * g.N;
  if (s > 1) {
    g.out = part;
    g.sums = sums ? part + s * n : nullptr;
    g.slice = n;
  }
  const hipError_t e = launch<kPlain, false, A_ALONG, B_ALONG>(g, s, st);
  if (e != hipSuccess || s == 1) return e;
  const int64_t groups = (n + 1023) / 1024 + (sums ? (g.M + 1023) / 1024 : 0);
  gated_f32_sum_kernel<<<dim3(static_cast<unsigned>(groups)), dim3(256), 0, st>>>(part, out, n, sums, sums ? g.M : 0, s);
  return hipGetLastError();
}

// ------------------------------------------------------------------ few rows
// A work-group owns 16 features of the result (with gate and up rows 32 rows of W) and all of K, its eight waves a run of K each, so that every
// wave streams its part of the rows from memory straight into matrix instructions of 16 x 16: A operand 16 rows of W, B operand the token
// rows, four k a lane and row.  The waves' sums meet in LDS and are added in wave order.
struct FewArgs {
  const float *x, *w, *bias;
  float *out, *keep;           // keep: gated, [gate | up] or null
  int M, N, K;                 // N: rows of one weight matrix
};

template <int P, bool GELU>
__global__ __launch_bounds__(512) void gated_f32_few_kernel(FewArgs a) {
  constexpr int U = 4, NW = 8;                 // steps whose loads are in flight together; waves
  __shared__ float part[NW][P * 4][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r16 = lane & 15, kg = lane >> 4, n0 = blockIdx.x * 16;
  const int steps = a.K / 16, per = (steps + NW - 1) / NW, s0 = wave * per, s1 = min(steps, s0 + per);
  const float *w[P], *x = a.x + static_cast<size_t>(min(r16, a.M - 1)) * a.K + kg * 4;
#pragma unroll
  for (int p = 0; p < P; ++p) w[p] = a.w + (static_cast<size_t>(p) * a.N + min(n0 + r16, a.N - 1)) * a.K + kg * 4;
  f32x4 acc[P] = {}, wr[2][U][P], xr[2][U];
  auto fetch = [&](auto to, int s) {           // steps past the wave's last read it again and are not multiplied
    constexpr int B = decltype(to)::value;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = min(s + u, s1 - 1) * 16;
#pragma unroll
      for (int p = 0; p < P; ++p) wr[B][u][p] = *reinterpret_cast<const f32x4 *>(w[p] + at);
      xr[B][u] = *reinterpret_cast<const f32x4 *>(x + at);
    }
  };
  auto use = [&](auto from, int s) {
    constexpr int B = decltype(from)::value;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (s + u < s1) {                        // uniform
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[p] = __builtin_amdgcn_mfma_f32_16x16x4f32(wr[B][u][p][i], xr[B][u][i], acc[p], 0, 0, 0);
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
    for (int r = 0; r < 4; ++r) part[wave][p * 4 + r][lane] = acc[p][r];
  __syncthreads();
  // value (m, n): register n % 4 of lane 16 (n / 4) + m
  const int m = threadIdx.x >> 4, nl = threadIdx.x & 15, n = n0 + nl;
  if (threadIdx.x >= 256 || m >= a.M || n >= a.N) return;
  float v[P];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int q = p * 4 + (nl & 3), l = ((nl >> 2) << 4) | m;
    v[p] = part[0][q][l];
#pragma unroll
    for (int k = 1; k < NW; ++k) v[p] += part[k][q][l];
    if (a.bias) v[p] += a.bias[p * a.N + n];
  }
  if constexpr (P == 2) {
    if (a.keep) {
      float *gu = a.keep + static_cast<size_t>(m) * 2 * a.N + n;
      gu[0] = v[0];
      gu[a.N] = v[1];
    }
    v[0] = gate_act_f32<GELU>(v[0]) * v[1];
  }
  a.out[static_cast<size_t>(m) * a.N + n] = v[0];
}

// Up to 16 rows whose contractions are whole steps of 16 from 16 bytes on: 1 x 1024 x 2752 18 us against 37 with tiles, 16 rows 25 against 39, 16 x
// 2048 x 8192 76 against 82; 32 rows would take two passes over the weights.
bool few_rows(const void *x, const void *w, int M, int K) { return M <= 16 && K % 16 == 0 && aligned(x, 16) && aligned(w, 16); }

}  // namespace

hipError_t launch_gated_f32_in(const GatedIn &in, bool gelu, hipStream_t st) {
  if (few_rows(in.x, in.w_in, in.M, in.D)) {
    const FewArgs a = {static_cast<const float *>(in.x), static_cast<const float *>(in.w_in), in.b_in, static_cast<float *>(in.h), static_cast<float *>(in.gu), in.M, in.R, in.D};
    if (gelu) gated_f32_few_kernel<2, true><<<dim3((in.R + 15) / 16), dim3(512), 0, st>>>(a);
    else gated_f32_few_kernel<2, false><<<dim3((in.R + 15) / 16), dim3(512), 0, st>>>(a);
    return hipGetLastError();
  }
  F32Args g = whole(static_cast<const float *>(in.x), in.D, static_cast<const float *>(in.w_in), in.D, static_cast<float *>(in.h), in.M, in.R, in.D);
  g.bias = in.b_in;
  g.keep = static_cast<float *>(in.gu);
  return gelu ? launch<kGate, true, true, true>(g, 1, st) : launch<kGate, false, true, true>(g, 1, st);
}
size_t gated_f32_product_bytes(int M, int N, int K) { return slice_bytes(M, N, K, 0); }
hipError_t launch_gated_f32_out(const float *h, const float *w_out, const float *b_out, float *y, int M, int D, int R, float *part, hipStream_t st) {
  if (few_rows(h, w_out, M, R)) {
    const FewArgs a = {h, w_out, b_out, y, nullptr, M, D, R};
    gated_f32_few_kernel<1, false><<<dim3((D + 15) / 16), dim3(512), 0, st>>>(a);
    return hipGetLastError();
  }
  F32Args g = whole(h, R, w_out, R, y, M, D, R);
  g.bias = b_out;
  return product<true, true>(g, part, st);
}
hipError_t launch_gated_f32_dgate(const float *dy, const float *w_out, const float *gu, float *d_gu, int M, int D, int R, bool gelu, hipStream_t st) {
  F32Args g = whole(dy, D, w_out, R, d_gu, M, R, D);
  g.gu = gu;
  return gelu ? launch<kDGate, true, true, false>(g, 1, st) : launch<kDGate, false, true, false>(g, 1, st);
}
hipError_t launch_gated_f32_dx(const float *d_gu, const float *w_in, float *dx, int M, int D, int R, float *part, hipStream_t st) {
  return product<true, false>(whole(d_gu, 2 * static_cast<int64_t>(R), w_in, D, dx, M, D, 2 * R), part, st);
}
size_t gated_f32_wgrad_bytes(int M, int N, int K) { return slice_bytes(N, K, M, N); }
hipError_t launch_gated_f32_wgrad(const float *dy, const float *x, float *dw, float *db, int M, int N, int K, void *ws, hipStream_t st) {
  F32Args g = whole(dy, N, x, K, dw, N, K, M);
  g.sums = db;
  return product<false, false>(g, static_cast<float *>(ws), st);
}

}  // namespace reslim
