// What the product kernels of gemm.hip and gated_gemm.hip share beside their main loops (gemm_small.inc, gemm_pp.inc): vector
// types, the argument block, and what a main loop has to know of the epilogue behind it.
#pragma once

#include "common.h"
#include "gemm_cursor.h"

namespace reslim {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

struct GemmArgs {
  const void *A;
  const void *W;
  const float *bias;
  void *out;
  const float *tab;
  int ldo, tab_rows;
  int M, N, K;
  int grid_m, grid_n;
  float qscale;   // EPI_BIAS_QSCALE_ACT: factor applied to output columns n < qcols
  int qcols;
  int col_fast;            // one-tile-per-work-group kernel: tile order inside a band
  const void *aux;         // EPI_BIAS_RES_F32: skip input (fp32), layout of out unless res_map is set
  const int32_t *res_map;  // EPI_BIAS_RES_F32, optional: output row b*res_out + r reads skip row b*res_in + res_map[r]
  int res_out;
  int64_t res_in;
  void *out2;              // EPI_BIAS_ACT_GELU2: second output (act), layout of out
  // fp32 kernel with LayerNorm in front: gain and bias; rows of A through a map (see ResRowMap) where it is set
  const float *ln_g, *ln_b;
  const int32_t *a_map;
  int a_out;
  int64_t a_in;
  // gated feed-forward layer (gated_gemm.hip)
  const float *x_scale, *w_scale;      // e4m3 operands: one factor a row of A, one a row of W
  const void *gu;                      // gradient: the forward's [g | u], act [M, 2N]
  int k_slabs;                         // slices of k (blockIdx.y): slabs of 64 in each
};

template <int EPI>
__device__ __host__ constexpr bool epi_act_out() {
  return EPI == EPI_BIAS_ACT || EPI == EPI_BIAS_QSCALE_ACT || EPI == EPI_BIAS_GELU_ACT || EPI == EPI_BIAS_ACT_GELU2;
}
constexpr int kEpiStageBytes = 4096;    // per wave

// Epilogues of the gated feed-forward layer (gated_gemm.hip), numbered behind those of common.h.  A gated product has two
// weight matrices, gate and up, N rows each, one behind the other; a tile's rows of W are then half gate rows and half up rows
// of the same features, so that a wave's column half 0 is the gate and column half 1 the up projection of 32 features.
enum GatedEpilogue {
  EPI_GATED = 32,         // out(act) = act(gate + bias) * (up + bias); + 1: GELU instead of SiLU,
  kEpiGelu1 = 1,          // + 2: keeps [gate | up] in out2 too, + 4: A and W are e4m3 with scales
  kEpiKeep = 2,
  kEpiE4m3 = 4,
  EPI_DGATE = 64,         // acc = gradient of the hidden layer: out(act) = gradients of [gate | up]; + 1: GELU
  EPI_SLICE = 96          // out(f32) [slices, M, N] = the sum over a slice of k (128 x 128 and 64 x 64 tiles)
};
constexpr bool epi_gated(int epi) { return epi >= EPI_GATED && epi < EPI_DGATE; }
constexpr bool epi_dgate(int epi) { return epi >= EPI_DGATE && epi < EPI_SLICE; }
constexpr bool epi_e4m3(int epi) { return epi_gated(epi) && (epi & kEpiE4m3); }

// Stores of a wave's epilogue over 64 rb rows inside the matrix, or fewer: the persistent kernels' waits let them be in flight.
template <int EPI>
constexpr int epi_stores(int rb) {
  if (epi_gated(EPI)) return (EPI & kEpiKeep ? 12 : 4) * rb;
  if (epi_dgate(EPI)) return 16 * rb;      // of 32 rb: the count has six bits
  return (!epi_act_out<EPI>() || EPI == EPI_BIAS_ACT_GELU2 ? 16 : 8) * rb;
}

// tile id seen by the hardware dispatcher -> tile id in XCD-contiguous order
__device__ __forceinline__ int xcd_remap(int pid, int total) {
  constexpr int NXCD = 8;
  const int x = pid % NXCD, local = pid / NXCD;
  const int q = total / NXCD, r = total % NXCD;
  return x * q + (x < r ? x : r) + local;
}

}  // namespace reslim
