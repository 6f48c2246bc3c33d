// The gated feed-forward layer's products on matrix tiles, bf16 and e4m3 operands (gfx950).
//
// Both projections, the activation and the product are one launch: the main loops of gemm_pp.inc and gemm_small.inc load
// half of a tile's weight rows from the gate matrix and half from the up matrix, interleaved so that every wave ends with
// the gate projection of 32 features in its column half 0 and the up projection of the same features in column half 1.  The
// hidden layer is then formed in the accumulators and written once, M R values instead of 2 M R written and read again.
#include <algorithm>
#include <type_traits>

#include "gated.h"
#include "gemm_kernel.h"
#include "gemm_plan.h"

namespace reslim {
namespace gated {

// Four values of a lane's accumulators to bf16, staged through the wave's 4 KB of LDS, 64 rows x 32 columns at a time: row r
// at 64 r bytes, its 16-byte chunk c at c ^ ((r >> 2) & 3), the two halves of a chunk exchanged in every second run of 16 rows,
// so that the 8-byte writes of 32 lanes (32 rows, one column quad) and the 16-byte reads of 16 lanes (four rows) each touch every
// bank once.  A store instruction then writes 16 row segments of 64 bytes.
template <bool GUARD, class F>
__device__ __forceinline__ void stage_rows(const GemmArgs &g, bf16_t *out, int ldo, int m_first, int n_first, int lane, unsigned char *stg, F &&value) {
  const int l32 = lane & 31, hi = lane >> 5;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int r = b * 32 + l32;
    unsigned char *row = stg + r * 64 + ((hi ^ ((r >> 4) & 1)) << 3);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float v[4];
      value(b, q, v);
      *reinterpret_cast<u32x2 *>(row + ((q ^ ((r >> 2) & 3)) << 4)) = u32x2{pack2(v[0], v[1]), pack2(v[2], v[3])};
    }
  }
  const int c = lane & 3, n = n_first + c * 8;
#pragma unroll
  for (int it = 0; it < 4; ++it) {
    const int r = it * 16 + (lane >> 2), m = m_first + r;
    u32x4 v = *reinterpret_cast<const u32x4 *>(stg + r * 64 + ((c ^ ((r >> 2) & 3)) << 4));
    if (it & 1) v = u32x4{v[2], v[3], v[0], v[1]};
    if (!GUARD || (m < g.M && n < g.N)) *reinterpret_cast<u32x4 *>(out + static_cast<size_t>(m) * ldo + n) = v;
  }
  __builtin_amdgcn_sched_barrier(0);
}

// Hidden layer (and [gate | up]) of rows m_base .. m_base + 32 MI - 1 and features n_base .. n_base + 31.  acc[i][0] is the gate, acc[i][1]
// the up projection, a lane holding row l32 of block i and features 8 q + 4 hi + 0..3 in register quad q.
template <int EPI, bool GUARD, int MI>
__device__ __forceinline__ void epilogue_gated(const GemmArgs &g, const f32x16 (&acc)[MI][2], int m_base, int n_base, int lane, unsigned char *stg) {
  constexpr bool kGelu = EPI & kEpiGelu1, kKeep = EPI & kEpiKeep;
  const int l32 = lane & 31, hi = lane >> 5;
  auto column = [&](int p, int q) {
    const int n = n_base + 8 * q + 4 * hi;
    return p * g.N + (GUARD ? min(n, g.N - 4) : n);
  };
  // bf16: biases; e4m3: the columns' factors, whose biases are read where they are added (both do not fit beside the accumulators)
  float4 col[2][4];
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float *from = epi_e4m3(EPI) ? g.w_scale : g.bias;
      col[p][q] = from ? *reinterpret_cast<const float4 *>(from + column(p, q)) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  // the next output adds the bias again: without this the compiler keeps the biased values and spills
  auto again = [&]() {
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int q = 0; q < 4; ++q) asm volatile("" : "+v"(col[p][q].x), "+v"(col[p][q].y), "+v"(col[p][q].z), "+v"(col[p][q].w));
  };
#pragma unroll
  for (int i = 0; i < MI; i += 2) {
    float rows[2] = {1.f, 1.f};
    if constexpr (epi_e4m3(EPI)) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int m = m_base + (i + b) * 32 + l32;
        rows[b] = g.x_scale[GUARD ? min(m, g.M - 1) : m];
      }
    }
    auto projected = [&](int p, int b, int q, float (&v)[4]) {
      const float c[4] = {col[p][q].x, col[p][q].y, col[p][q].z, col[p][q].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = epi_e4m3(EPI) ? acc[i + b][p][4 * q + e] * (rows[b] * c[e]) : acc[i + b][p][4 * q + e] + c[e];
      if constexpr (epi_e4m3(EPI)) {
        if (g.bias) {                        // uniform
          const float4 o = *reinterpret_cast<const float4 *>(g.bias + column(p, q));
          v[0] += o.x; v[1] += o.y; v[2] += o.z; v[3] += o.w;
        }
      }
    };
    const int m = m_base + i * 32;
    if constexpr (kKeep) {
      bf16_t *gu = static_cast<bf16_t *>(g.out2);
      stage_rows<GUARD>(g, gu, 2 * g.N, m, n_base, lane, stg, [&](int b, int q, float (&v)[4]) { projected(0, b, q, v); });
      again();
      stage_rows<GUARD>(g, gu + g.N, 2 * g.N, m, n_base, lane, stg, [&](int b, int q, float (&v)[4]) { projected(1, b, q, v); });
      again();
    }
    stage_rows<GUARD>(g, static_cast<bf16_t *>(g.out), g.N, m, n_base, lane, stg, [&](int b, int q, float (&v)[4]) {
      float up[4];
      projected(0, b, q, v);
      projected(1, b, q, up);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = gate_act<kGelu>(v[e]) * up[e];
    });
  }
}

// Gradients of gate and up projection from the hidden layer's (acc) and what the forward kept: 32 x 32 blocks in fp32 through the wave's
// LDS (row r at 128 r bytes, its 16-byte chunk c at c ^ ((r >> 1) & 7)), so that eight lanes hold 32 neighbouring columns of a row
// and read and write 64-byte segments.  The kept values of the next block are requested ahead of the block at hand.
template <int EPI, bool GUARD, int MI, int NI>
__device__ __forceinline__ void epilogue_dgate(const GemmArgs &g, const f32x16 (&acc)[MI][NI], int m_base, int n_base, int lane, unsigned char *stg) {
  constexpr bool kGelu = EPI & kEpiGelu1;
  constexpr int DEPTH = kGelu ? 1 : 2;       // GELU's slope takes the registers of the second block
  const int l32 = lane & 31, hi = lane >> 5, lr = lane >> 3, lc = lane & 7;
  const bf16_t *gu = static_cast<const bf16_t *>(g.gu);
  u32x2 kept[DEPTH][4][2];
  auto fetch = [&](int b) {
    const int i = b / NI, j = b % NI;
    const int n = GUARD ? min(n_base + j * 32 + lc * 4, g.N - 4) : n_base + j * 32 + lc * 4;
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      const int mu = m_base + i * 32 + it * 8, m = GUARD ? min(mu + lr, g.M - 1) : mu + lr;
      const bf16_t *p = gu + static_cast<size_t>(m) * (2 * g.N) + n;
      kept[b % DEPTH][it][0] = *reinterpret_cast<const u32x2 *>(p);
      kept[b % DEPTH][it][1] = *reinterpret_cast<const u32x2 *>(p + g.N);
    }
  };
#pragma unroll
  for (int b = 0; b < DEPTH; ++b) fetch(b);
  unsigned char *wrow = stg + l32 * 128;
  const int wsw = (l32 >> 1) & 7;
  bf16_t *out = static_cast<bf16_t *>(g.out);
#pragma unroll
  for (int b = 0; b < MI * NI; ++b) {
    const int i = b / NI, j = b % NI;
    const f32x16 &a = acc[i][j];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<float4 *>(wrow + (((2 * q + hi) ^ wsw) << 4)) = make_float4(a[4 * q], a[4 * q + 1], a[4 * q + 2], a[4 * q + 3]);
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      const int r = it * 8 + lr, m = m_base + i * 32 + r, n = n_base + j * 32 + lc * 4;
      const float4 dh4 = *reinterpret_cast<const float4 *>(stg + r * 128 + ((lc ^ ((r >> 1) & 7)) << 4));
      const float dh[4] = {dh4.x, dh4.y, dh4.z, dh4.w};
      float dg[4], du[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t wg = kept[b % DEPTH][it][0][e / 2], wu = kept[b % DEPTH][it][1][e / 2];
        const float vg = __uint_as_float(e % 2 ? wg & 0xffff0000u : wg << 16), vu = __uint_as_float(e % 2 ? wu & 0xffff0000u : wu << 16);
        float act, slope;
        gate_act_slope<kGelu>(vg, act, slope);
        dg[e] = dh[e] * vu * slope;
        du[e] = dh[e] * act;
      }
      if (!GUARD || (m < g.M && n < g.N)) {
        bf16_t *o = out + static_cast<size_t>(m) * (2 * g.N) + n;
        *reinterpret_cast<u32x2 *>(o) = u32x2{pack2(dg[0], dg[1]), pack2(dg[2], dg[3])};
        *reinterpret_cast<u32x2 *>(o + g.N) = u32x2{pack2(du[0], du[1]), pack2(du[2], du[3])};
      }
      __builtin_amdgcn_sched_barrier(0);     // four rows' arithmetic at once does not fit beside the accumulators
    }
    __builtin_amdgcn_sched_barrier(0);
    if (b + DEPTH < MI * NI) fetch(b + DEPTH);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// A slice's sums, fp32, 32 x 32 blocks through the wave's LDS as above: eight whole 128-byte lines a store.
template <bool GUARD, int MI, int NI>
__device__ __forceinline__ void epilogue_slice(const GemmArgs &g, const f32x16 (&acc)[MI][NI], int m_base, int n_base, int lane, unsigned char *stg) {
  const int l32 = lane & 31, hi = lane >> 5, lr = lane >> 3, lc = lane & 7;
  float *out = static_cast<float *>(g.out) + static_cast<size_t>(blockIdx.y) * g.M * g.N;
  unsigned char *wrow = stg + l32 * 128;
  const int wsw = (l32 >> 1) & 7;
#pragma unroll
  for (int b = 0; b < MI * NI; ++b) {
    const f32x16 &a = acc[b / NI][b % NI];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<float4 *>(wrow + (((2 * q + hi) ^ wsw) << 4)) = make_float4(a[4 * q], a[4 * q + 1], a[4 * q + 2], a[4 * q + 3]);
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      const int r = it * 8 + lr, m = m_base + b / NI * 32 + r, n = n_base + b % NI * 32 + lc * 4;
      const float4 v = *reinterpret_cast<const float4 *>(stg + r * 128 + ((lc ^ ((r >> 1) & 7)) << 4));
      if (!GUARD || (m < g.M && n < g.N)) *reinterpret_cast<float4 *>(out + static_cast<size_t>(m) * g.N + n) = v;
    }
  }
}

// stg: this wave's kEpiStageBytes of LDS.  GUARD = false: the wave's part of the tile lies inside the output.
template <int EPI, bool GUARD, int MI, int NI>
__device__ __forceinline__ void epilogue_wave(const GemmArgs &g, const f32x16 (&acc)[MI][NI], int m_base, int n_base, int lane, unsigned char *stg) {
  static_assert(MI % 2 == 0 && NI == 2, "pairs of row blocks; gate beside up");
  if constexpr (epi_gated(EPI)) epilogue_gated<EPI, GUARD, MI>(g, acc, m_base, n_base, lane, stg);
  else if constexpr (EPI == EPI_SLICE) epilogue_slice<GUARD, MI, NI>(g, acc, m_base, n_base, lane, stg);
  else epilogue_dgate<EPI, GUARD, MI, NI>(g, acc, m_base, n_base, lane, stg);
}

#include "gemm_small.inc"
#include "gemm_pp.inc"

typedef TileCfg<128, 128, 64, 2, 2, 1, 3> TileSmall;

// N: rows of one weight matrix (both for gated products).  The estimates of gemm_choose hold for a product of as many weight rows.
template <int EPI>
static hipError_t launch(GemmArgs g, hipStream_t st) {
  constexpr bool kGated = epi_gated(EPI);
  const GemmEpi cost = epi_dgate(EPI) ? kEpiStream : EPI & kEpiKeep ? kEpiTwo : kEpiGelu;
  const GemmKernel pick = gemm_choose(g.M, kGated ? 2 * g.N : g.N, epi_e4m3(EPI) ? g.K / 2 : g.K, cost, g_num_cus);
  if (pick == kGemm256x256) return launch_bf16_pp<2, EPI>(g, st);
  if constexpr (!epi_e4m3(EPI)) {
    if (pick == kGemm128) return launch_bf16_tc<TileSmall, EPI>(g, st);
  }
  return launch_bf16_pp<1, EPI>(g, st);
}

template <int EPI>
static hipError_t init_one() {
  hipError_t e = set_attr_pp<2, EPI>();
  if (e == hipSuccess) e = set_attr_pp<1, EPI>();
  if constexpr (!epi_e4m3(EPI)) {
    if (e == hipSuccess) e = set_attr<TileSmall, EPI>();
  }
  return e;
}

// out[i] = sum of the slices' values in their order, and the column's bias; four values a thread
__global__ __launch_bounds__(256) void slice_sum_kernel(const float4 *__restrict__ part, const float4 *__restrict__ bias, u32x2 *__restrict__ out, int slices, int64_t n4, int cols4) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= n4) return;
  float4 s = part[i];
  int k = 1;
  for (; k + 3 < slices; k += 4) {
    float4 v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = part[(k + j) * n4 + i];
#pragma unroll
    for (int j = 0; j < 4; ++j) { s.x += v[j].x; s.y += v[j].y; s.z += v[j].z; s.w += v[j].w; }
  }
  for (; k < slices; ++k) {
    const float4 v = part[k * n4 + i];
    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
  }
  if (bias) {
    const float4 b = bias[i % cols4];
    s.x += b.x; s.y += b.y; s.z += b.z; s.w += b.w;
  }
  out[i] = u32x2{pack2(s.x, s.y), pack2(s.z, s.w)};
}

}  // namespace gated

using namespace gated;

// As many slices as give the chip two work-groups a compute unit, of at least five slabs of 64; none for short sums, where the second launch costs what
// the shorter loops save.  Output map of 1024 features over 2752, whole / in slices: 64 rows 38.7 / 24.3 us (with the first launch), 512 rows
// 42.7 / 30.0, 2000 rows 53.5 / 50.8; of 4096 over 10,944: 64 rows 195 / 90, 256 rows 219 / 113, 1000 rows 312 / 279, 2000 rows 423 / 487, where
// there are two tiles a compute unit without slices.
int gated_slices(int M, int N, int K) {
  const int64_t tiles = (static_cast<int64_t>(M) + 127) / 128 * ((N + 127) / 128);
  const int slabs = K / 64;
  if (slabs < 16) return 1;
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(2LL * g_num_cus / tiles, slabs / 5)));
}

hipError_t launch_gated_sliced(const void *a, const void *w, const float *bias, void *out, int M, int N, int K, float *part, hipStream_t st) {
  if (M <= 0 || N <= 0 || K <= 0 || K % 64 || N % 8) return hipErrorInvalidValue;
  GemmArgs g = {};
  g.A = a; g.W = w; g.out = part; g.ldo = N; g.tab_rows = 1; g.M = M; g.N = N; g.K = K;
  const int slabs = K / 64, want = gated_slices(M, N, K);
  g.k_slabs = (slabs + want - 1) / want;
  const hipError_t e = launch_bf16_tc<TileSmall, EPI_SLICE>(g, st);
  if (e != hipSuccess) return e;
  const int64_t n4 = static_cast<int64_t>(M) * N / 4;
  slice_sum_kernel<<<dim3(static_cast<unsigned>((n4 + 255) / 256)), dim3(256), 0, st>>>(reinterpret_cast<const float4 *>(part), reinterpret_cast<const float4 *>(bias),
                                                                                      static_cast<u32x2 *>(out), (slabs + g.k_slabs - 1) / g.k_slabs, n4, N / 4);
  return hipGetLastError();
}

hipError_t gated_gemm_init() {
  int dev = 0, cus = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (e == hipSuccess && cus > 0) g_num_cus = cus;
  if (e == hipSuccess) e = init_one<EPI_GATED>();
  if (e == hipSuccess) e = init_one<EPI_GATED + 1>();
  if (e == hipSuccess) e = init_one<EPI_GATED + kEpiKeep>();
  if (e == hipSuccess) e = init_one<EPI_GATED + kEpiKeep + 1>();
  if (e == hipSuccess) e = init_one<EPI_GATED + kEpiE4m3>();
  if (e == hipSuccess) e = init_one<EPI_GATED + kEpiE4m3 + 1>();
  if (e == hipSuccess) e = init_one<EPI_DGATE>();
  if (e == hipSuccess) e = init_one<EPI_DGATE + 1>();
  if (e == hipSuccess) e = set_attr<TileSmall, EPI_SLICE>();
  return e;
}

hipError_t launch_gated_in(const GatedIn &in, bool gelu, hipStream_t st) {
  const bool e4m3 = in.x_scale != nullptr;
  if (in.M <= 0 || in.D <= 0 || in.R <= 0 || in.D % (e4m3 ? 128 : 64) || in.R % 8 || (e4m3 && in.gu)) return hipErrorInvalidValue;
  GemmArgs g = {};
  g.A = in.x; g.W = in.w_in; g.bias = in.b_in; g.out = in.h; g.out2 = in.gu;
  g.ldo = in.R; g.tab_rows = 1; g.M = in.M; g.N = in.R; g.K = in.D;
  g.x_scale = in.x_scale; g.w_scale = in.in_scale;
  if (e4m3) return gelu ? launch<EPI_GATED + kEpiE4m3 + 1>(g, st) : launch<EPI_GATED + kEpiE4m3>(g, st);
  if (in.gu) return gelu ? launch<EPI_GATED + kEpiKeep + 1>(g, st) : launch<EPI_GATED + kEpiKeep>(g, st);
  return gelu ? launch<EPI_GATED + 1>(g, st) : launch<EPI_GATED>(g, st);
}

hipError_t launch_gated_dgate(const void *dy, const void *wt_out, const void *gu, void *d_gu, int M, int D, int R, bool gelu, hipStream_t st) {
  if (M <= 0 || D <= 0 || R <= 0 || D % 64 || R % 8) return hipErrorInvalidValue;
  GemmArgs g = {};
  g.A = dy; g.W = wt_out; g.out = d_gu; g.gu = gu;
  g.ldo = 2 * R; g.tab_rows = 1; g.M = M; g.N = R; g.K = D;
  return gelu ? launch<EPI_DGATE + 1>(g, st) : launch<EPI_DGATE>(g, st);
}

// ------------------------------------------------------------------ weight transposes of the gradient
// 64 x 64 tiles through LDS: 16-byte loads along the source's rows, 16-byte stores along the destination's.  A thread's eight
// values of a column are gathered from eight rows of LDS, two bytes each; rows are padded to 66 values so that they lie in
// different banks.  Sizes are multiples of 64 (2R, D) or of 8.
struct TransposeArgs {
  const bf16_t *src[2];
  bf16_t *dst[2];
  int rows[2], cols[2], tiles_c[2], first;      // `first`: tiles of matrix 0
};
__global__ __launch_bounds__(256) void gated_transpose_kernel(TransposeArgs a) {
  __shared__ bf16_t tile[64][66];
  const int w = static_cast<int>(blockIdx.x) >= a.first;
  const int L = blockIdx.x - (w ? a.first : 0);
  const bf16_t *src = w ? a.src[1] : a.src[0];
  bf16_t *dst = w ? a.dst[1] : a.dst[0];
  const int R = w ? a.rows[1] : a.rows[0], C = w ? a.cols[1] : a.cols[0], tc = w ? a.tiles_c[1] : a.tiles_c[0];
  const int r0 = L / tc * 64, c0 = L % tc * 64;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = (threadIdx.x >> 3) + 32 * i, c = (threadIdx.x & 7) * 8;
    if (r0 + r < R && c0 + c < C) {
      const u32x4 v = *reinterpret_cast<const u32x4 *>(src + static_cast<size_t>(r0 + r) * C + c0 + c);
#pragma unroll
      for (int k = 0; k < 4; ++k) *reinterpret_cast<uint32_t *>(&tile[r][c + 2 * k]) = v[k];
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int c = (threadIdx.x >> 3) + 32 * i, r = (threadIdx.x & 7) * 8;
    if (c0 + c < C && r0 + r < R) {
      u32x4 v;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = static_cast<uint32_t>(tile[r + 2 * k][c]) | (static_cast<uint32_t>(tile[r + 2 * k + 1][c]) << 16);
      *reinterpret_cast<u32x4 *>(dst + static_cast<size_t>(c0 + c) * R + r0 + r) = v;
    }
  }
}

hipError_t launch_gated_transpose(const void *w_in, void *wt_in, const void *w_out, void *wt_out, int D, int R, hipStream_t st) {
  if (D % 8 || R % 8) return hipErrorInvalidValue;
  TransposeArgs a = {};
  a.src[0] = static_cast<const bf16_t *>(w_in); a.dst[0] = static_cast<bf16_t *>(wt_in); a.rows[0] = 2 * R; a.cols[0] = D;
  a.src[1] = static_cast<const bf16_t *>(w_out); a.dst[1] = static_cast<bf16_t *>(wt_out); a.rows[1] = D; a.cols[1] = R;
  for (int i = 0; i < 2; ++i) a.tiles_c[i] = (a.cols[i] + 63) / 64;
  a.first = (a.rows[0] + 63) / 64 * a.tiles_c[0];
  const int total = a.first + (a.rows[1] + 63) / 64 * a.tiles_c[1];
  gated_transpose_kernel<<<dim3(total), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace reslim
