// The gated feed-forward layer's products on matrix tiles, bf16 and e4m3 operands (gfx950).
//
// Both projections, the activation and the product are one launch: the main loops of gemm_pp.inc and gemm_small.inc load
// half of a tile's weight rows from the gate matrix and half from the up matrix, interleaved so that every wave ends with
// the gate projection of 32 features in its column half 0 and the up projection of the same features in column half 1.  The
// hidden layer is then formed in the accumulators and written once, M R values instead of 2 M R written and read again.
//   Large products are bound by the matrix instructions at the power limit: 37,520 x 4096 x 2 x 10,944 in e4m3 2.44 ms, 2760 TFLOP/s (the library's
// 8192^3 2809); 80,704 x 1024 x 2 x 2752 in bf16 with [gate | up] kept 0.87-1.05 ms, 870-1050 TFLOP/s, where a tile has 16 slabs to 10 us
// of epilogue (the library's product of that shape alone 0.78-0.80 ms).  Few rows are bound by memory: see the 64 x 64 tiles.
#include <algorithm>
#include <type_traits>

#include "gated.h"
#include "gemm_kernel.h"

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

// One hidden value's gradient to those of its gate and up projection; half `odd` of the words holds what the forward kept.
template <bool GELU>
__device__ __forceinline__ void gate_gradient(float dh, uint32_t gates, uint32_t ups, bool odd, float &dg, float &du) {
  const float vg = __uint_as_float(odd ? gates & 0xffff0000u : gates << 16), vu = __uint_as_float(odd ? ups & 0xffff0000u : ups << 16);
  float act, slope;
  gate_act_slope<GELU>(vg, act, slope);
  dg = dh * vu * slope;
  du = dh * act;
}

// Gradients of gate and up projection from the hidden layer's (acc) and what the forward kept: 32 x 32 blocks in fp32 through the wave's
// LDS (row r at 128 r bytes, its 16-byte chunk c at c ^ ((r >> 1) & 7)), so that eight lanes hold 32 neighbouring columns of a row
// and read and write 64-byte segments.  The kept values come from memory while nothing else of the wave runs, so their loads go out as
// far ahead as registers allow: FIRST blocks before the first one, and for every block that has left the accumulators two more.  40,352 x 1024 x
// 2752 takes 343-367 us (620-660 TFLOP/s, 0.89 GB of gate, up and gradients; the library's product of that shape alone 242): 255 without the reads, 240 without reads and stores.
template <int EPI, bool GUARD, int MI, int NI>
__device__ __forceinline__ void epilogue_dgate(const GemmArgs &g, const f32x16 (&acc)[MI][NI], int m_base, int n_base, int lane, unsigned char *stg) {
  constexpr bool kGelu = EPI & kEpiGelu1;
  constexpr int BLOCKS = MI * NI, FIRST = GUARD || kGelu ? 1 : 2;      // at an edge the addresses take the registers, and GELU's slope does
  const int l32 = lane & 31, hi = lane >> 5, lr = lane >> 3, lc = lane & 7;
  const bf16_t *gu = static_cast<const bf16_t *>(g.gu);
  const unsigned at = static_cast<unsigned>(lr * 2 * g.N + lc * 4);
  u32x2 kept[BLOCKS][4][2];
  auto fetch = [&](int b) {
    const int i = b / NI, j = b % NI;
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      const int mu = m_base + i * 32 + it * 8;                 // uniform
      const bf16_t *p;
      if constexpr (GUARD) p = gu + static_cast<size_t>(min(mu + lr, g.M - 1)) * (2 * g.N) + min(n_base + j * 32 + lc * 4, g.N - 4);
      else p = gu + static_cast<size_t>(mu) * (2 * g.N) + n_base + j * 32 + at;      // uniform base, one 32-bit offset per lane
      kept[b][it][0] = *reinterpret_cast<const u32x2 *>(p);
      kept[b][it][1] = *reinterpret_cast<const u32x2 *>(p + g.N);
    }
  };
#pragma unroll
  for (int b = 0; b < FIRST; ++b) fetch(b);
  unsigned char *wrow = stg + l32 * 128;
  const int wsw = (l32 >> 1) & 7;
  bf16_t *out = static_cast<bf16_t *>(g.out);
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b) {
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
      for (int e = 0; e < 4; ++e) gate_gradient<kGelu>(dh[e], kept[b][it][0][e / 2], kept[b][it][1][e / 2], e % 2, dg[e], du[e]);
      if (!GUARD || (m < g.M && n < g.N)) {
        bf16_t *o = out + static_cast<size_t>(m_base + i * 32 + it * 8) * (2 * g.N) + n_base + j * 32 + at;
        *reinterpret_cast<u32x2 *>(o) = u32x2{pack2(dg[0], dg[1]), pack2(dg[2], dg[3])};
        *reinterpret_cast<u32x2 *>(o + g.N) = u32x2{pack2(du[0], du[1]), pack2(du[2], du[3])};
      }
      __builtin_amdgcn_sched_barrier(0);     // four rows' arithmetic at once does not fit beside the accumulators
    }
    // blocks requested once this one is done, and before it
    const int ahead = GUARD || kGelu ? b + FIRST + 1 : b < 1 ? 3 : 2 * b + 2, behind = GUARD || kGelu ? b + FIRST : b < 2 ? b + 2 : 2 * b;
#pragma unroll
    for (int k = 0; k < BLOCKS; ++k)
      if (k >= behind && k < ahead) fetch(k);
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

// ------------------------------------------------------------------ 64 x 64 tiles, for products that do not fill the chip
// One tile of 64 rows of A and 64 rows of W for a work-group of four waves (32 x 32 each), k in slabs of 128 bytes a row that go from
// memory straight into a ring of four LDS slots, so that three slabs are in flight while one is multiplied: what bounds such products
// is the latency of a slab, and the 128 x 128 tiles, which load the next slab into registers while they multiply one, take 0.75 us for each.  One
// barrier a slab: past it every wave's share of the slab has landed, and every wave has read the slab before it, whose slot
// the next loads fill.  Two work-groups lie on a compute unit.  Places of the 16-byte chunks as in gemm_pp.inc.  A gated wave's 32 rows
// of W are 16 gate and 16 up rows of the same features: registers r and r + 8 of a lane.  One row through 4096 x 10,944: 32 us for gate and up (5.7 TB/s
// of weights), 16 and 5 for the output map in slices (5.8 TB/s); 197 x 320 x 832, all latency, 4.6 and 6.7 us.
constexpr int kRing = 4, kRingSlab = 2 * 64 * 128;
constexpr int ring_lds() { return kRing * kRingSlab; }

// ACROSS: W lies as [K, N], its k across rows; a slot then holds 64 rows of k x 64 columns, and fragments come from the transposing read
// ds_read_b64_tr_b16 (four k of one column a lane, twice for the eight of an operand), whose 32 lanes touch four rows of 64 bytes at a time:
// the 16-byte chunks of every second pair of rows are moved by four.
template <int OFF>
__device__ __forceinline__ void read_across(uint64_t &d, unsigned addr) {
  static_assert(OFF >= 0 && OFF < 65536, "16-bit offset field");
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(d) : "v"(addr), "n"(OFF) : "memory");
}

template <int EPI, bool ACROSS>
__global__ __launch_bounds__(256, 2) void gemm_ring_kernel(GemmArgs g) {
  static_assert(!ACROSS || !epi_gated(EPI), "gated products have k along the rows of W");
  constexpr bool kGated = epi_gated(EPI), kE4m3 = epi_e4m3(EPI), kGelu = (kGated || epi_dgate(EPI)) && (EPI & kEpiGelu1);
  constexpr int BNO = kGated ? 32 : 64;        // output columns of a tile
  extern __shared__ __align__(1024) unsigned char smem[];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave >> 1, wn = wave & 1, l32 = lane & 31, hi = lane >> 5;
  const unsigned K2 = static_cast<unsigned>(g.K) * (kE4m3 ? 1 : 2);
  const int slabs = static_cast<int>(K2 / 128);
  const int first = EPI == EPI_SLICE ? blockIdx.y * g.k_slabs : 0;
  const int nk = EPI == EPI_SLICE ? min(g.k_slabs, slabs - first) : slabs;
  // tiles that share rows of W are neighbours and lie on one XCD
  const int pid = xcd_remap(blockIdx.x, g.grid_m * g.grid_n);
  const int m0 = pid % g.grid_m * 64, n0 = pid / g.grid_m * BNO;

  // A buffer covers exactly the tile's rows that exist: others are loaded as zeros.  Blocks of 8 rows, two of A and two of W a wave.
  auto rows_from = [&](const void *base, int row0, int rows, int most) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(static_cast<const unsigned char *>(base)) + static_cast<size_t>(row0) * K2, 0,
                                             min(most, rows - row0) * static_cast<int>(K2), 0x00020000);
  };
  const bool up = kGated && (wave & 2);      // this wave's blocks hold up rows
  const __amdgpu_buffer_rsrc_t a_rsrc = rows_from(g.A, m0, g.M, 64);
  __amdgpu_buffer_rsrc_t w_rsrc;
  if constexpr (!ACROSS) w_rsrc = rows_from(static_cast<const unsigned char *>(g.W) + (up ? static_cast<size_t>(g.N) * K2 : 0), n0, g.N, BNO);
  const int lrow = lane >> 3;
  const unsigned c16 = ((lane & 7) ^ lrow ^ (wave & 1)) << 4;
  unsigned vo_a[2], vo_w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = (wave + 4 * i) * 8 + lrow;
    vo_a[i] = r * K2 + c16;
    if constexpr (ACROSS) vo_w[i] = r * static_cast<unsigned>(g.N) * 2 + (((lane & 7) ^ (((r >> 1) & 1) << 2)) << 4);
    else vo_w[i] = (kGated ? i * 16 + (wave & 1) * 8 + lrow : r) * K2 + c16;
  }
  auto issue = [&](int s) {
    const int slot = s % kRing * kRingSlab, off = (first + s) * 128;
    if constexpr (ACROSS)                      // N is a multiple of 64: the tile's columns exist
      w_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t *>(static_cast<const bf16_t *>(g.W) + static_cast<size_t>(first + s) * 64 * g.N + n0), 0,
                                                 (63 * g.N + 64) * 2, 0x00020000);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      __builtin_amdgcn_raw_ptr_buffer_load_lds(a_rsrc, (__attribute__((address_space(3))) void *)(smem + slot + (wave + 4 * i) * 1024), 16, static_cast<int>(vo_a[i]), off, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(w_rsrc, (__attribute__((address_space(3))) void *)(smem + slot + 8192 + (wave + 4 * i) * 1024), 16, static_cast<int>(vo_w[i]),
                                               ACROSS ? 0 : off, 0, 0);
    }
  };
  const int fx = (l32 & 7) ^ ((l32 >> 3) & 1);
  unsigned a_at[4], w_at[4];
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) {
    const int c = ((2 * kk + hi) ^ fx) << 4;
    a_at[kk] = (wm * 32 + l32) * 128 + c;
    w_at[kk] = 8192 + (wn * 32 + l32) * 128 + c;
  }
  // ACROSS: this lane points at row 8 hi + 4 e + (lane % 16) / 4 of a step of 16 k, columns 32 wn + 16 ((lane / 16) & 1) + 4 (lane % 4) .. + 3
  unsigned across_at[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int r = 8 * hi + 4 * e + ((lane & 15) >> 2), o = 32 * wn + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    across_at[e] = static_cast<unsigned>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const unsigned char *)smem)) + 8192 + r * 128 +
                   (((o >> 3) ^ (((r >> 1) & 1) << 2)) << 4) + ((o >> 2) & 1) * 8;
  }
  f32x16 acc = {};
#pragma unroll
  for (int s = 0; s < kRing - 1; ++s)
    if (s < nk) issue(s);
  for (int k = 0; k < nk; ++k) {
    __builtin_amdgcn_sched_barrier(0);
    if (k + kRing - 2 < nk) wait_vm_lgkm0<4 * (kRing - 2)>();      // the loads of slab k have landed: four a slab, of the slabs behind it
    else wait_vm_lgkm0<0>();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    if (k + kRing - 1 < nk) issue(k + kRing - 1);
    __builtin_amdgcn_sched_barrier(0);
    const unsigned char *slot = smem + k % kRing * kRingSlab;
    bf16x8 a[4], w[4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) a[kk] = *reinterpret_cast<const bf16x8 *>(slot + a_at[kk]);
    if constexpr (ACROSS) {
      const unsigned base = k % kRing * kRingSlab;
      uint64_t f[4][2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        read_across<0>(f[0][e], base + across_at[e]);
        read_across<16 * 128>(f[1][e], base + across_at[e]);
        read_across<32 * 128>(f[2][e], base + across_at[e]);
        read_across<48 * 128>(f[3][e], base + across_at[e]);
      }
      __builtin_amdgcn_sched_barrier(0);
      wait_vm_lgkm0<63>();
      __builtin_amdgcn_sched_barrier(0);
      // the reads are complete from here on: nothing that uses them may move above
      asm volatile("" : "+v"(f[0][0]), "+v"(f[0][1]), "+v"(f[1][0]), "+v"(f[1][1]), "+v"(f[2][0]), "+v"(f[2][1]), "+v"(f[3][0]), "+v"(f[3][1]));
      typedef __attribute__((ext_vector_type(2))) uint64_t u64x2;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) w[kk] = __builtin_bit_cast(bf16x8, u64x2{f[kk][0], f[kk][1]});
    } else {
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) w[kk] = *reinterpret_cast<const bf16x8 *>(slot + w_at[kk]);
      __builtin_amdgcn_sched_barrier(0);       // all reads of the slab first, or each product waits for its own
    }
    if constexpr (kE4m3) {
      typedef __attribute__((ext_vector_type(4))) int i32x4;
      auto join = [](const bf16x8 &lo, const bf16x8 &hi8) {
        return __builtin_shufflevector(__builtin_bit_cast(i32x4, lo), __builtin_bit_cast(i32x4, hi8), 0, 1, 2, 3, 4, 5, 6, 7);
      };
#pragma unroll
      for (int kk = 0; kk < 4; kk += 2)
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(join(w[kk], w[kk + 1]), join(a[kk], a[kk + 1]), acc, 0, 0, 0, 0, 0, 0);
    } else {
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w[kk], a[kk], acc, 0, 0, 0);      // operands swapped: the block is C^T
    }
  }

  // Epilogue: the whole tile through LDS, then rows of 64 or 128 bytes.  A lane holds row wm 32 + l32, columns 8 q + 4 hi + 0..3 of the
  // wave's 32 in register quad q.
  const int ml = wm * 32 + l32;
  if constexpr (epi_dgate(EPI)) {              // thread: four columns of every fourth group of 16 rows; what the forward kept is requested first
    const int c = t & 15, r0 = t >> 4;
    u32x2 kept[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int m = min(m0 + r0 + 16 * i, g.M - 1), n = min(n0 + 4 * c, g.N - 4);
      const bf16_t *p = static_cast<const bf16_t *>(g.gu) + static_cast<size_t>(m) * 2 * g.N + n;
      kept[i][0] = *reinterpret_cast<const u32x2 *>(p);
      kept[i][1] = *reinterpret_cast<const u32x2 *>(p + g.N);
    }
    constexpr int P = 68;                      // floats of a staged row
    float *st = reinterpret_cast<float *>(smem);
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<float4 *>(st + ml * P + wn * 32 + 8 * q + 4 * hi) = make_float4(acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int m = m0 + r0 + 16 * i, n = n0 + 4 * c;
      const float4 v = *reinterpret_cast<const float4 *>(st + (r0 + 16 * i) * P + 4 * c);
      const float dh[4] = {v.x, v.y, v.z, v.w};
      float dg[4], du[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) gate_gradient<kGelu>(dh[e], kept[i][0][e / 2], kept[i][1][e / 2], e % 2, dg[e], du[e]);
      if (m < g.M && n < g.N) {
        bf16_t *o = static_cast<bf16_t *>(g.out) + static_cast<size_t>(m) * 2 * g.N + n;
        *reinterpret_cast<u32x2 *>(o) = u32x2{pack2(dg[0], dg[1]), pack2(dg[2], dg[3])};
        *reinterpret_cast<u32x2 *>(o + g.N) = u32x2{pack2(du[0], du[1]), pack2(du[2], du[3])};
      }
    }
  } else if constexpr (EPI == EPI_SLICE) {
    constexpr int P = 68;
    float *st = reinterpret_cast<float *>(smem);
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<float4 *>(st + ml * P + wn * 32 + 8 * q + 4 * hi) = make_float4(acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
    __syncthreads();
    float *out = static_cast<float *>(g.out) + static_cast<size_t>(blockIdx.y) * g.M * g.N;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = (t >> 4) + 16 * i, c = 4 * (t & 15);
      if (m0 + r < g.M && n0 + c < g.N) *reinterpret_cast<float4 *>(out + static_cast<size_t>(m0 + r) * g.N + n0 + c) = *reinterpret_cast<const float4 *>(st + r * P + c);
    }
  } else {
    constexpr bool kKeep = kGated && (EPI & kEpiKeep);
    constexpr int P = kGated ? 40 : 72;        // bf16 values of a staged row, 16-byte pieces in different banks
    bf16_t *st = reinterpret_cast<bf16_t *>(smem);
    __syncthreads();
    const float xs = kE4m3 ? g.x_scale[min(m0 + ml, g.M - 1)] : 1.0f;
#pragma unroll
    for (int q = 0; q < (kGated ? 2 : 4); ++q) {
      const int col = kGated ? wn * 16 + 8 * q + 4 * hi : wn * 32 + 8 * q + 4 * hi;
      const int n = min(n0 + col, g.N - 4);
      float v[2][4];
#pragma unroll
      for (int p = 0; p < (kGated ? 2 : 1); ++p) {
        const float4 b = g.bias ? *reinterpret_cast<const float4 *>(g.bias + p * g.N + n) : make_float4(0.f, 0.f, 0.f, 0.f);
        const float4 f = kE4m3 ? *reinterpret_cast<const float4 *>(g.w_scale + p * g.N + n) : make_float4(1.f, 1.f, 1.f, 1.f);
        const float bs[4] = {b.x, b.y, b.z, b.w}, fs[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) v[p][e] = kE4m3 ? fmaf(acc[8 * p + 4 * q + e], xs * fs[e], bs[e]) : acc[8 * p + 4 * q + e] + bs[e];
      }
      bf16_t *row = st + ml * P + col;
      if constexpr (kGated) {
        if constexpr (kKeep) {
#pragma unroll
          for (int p = 0; p < 2; ++p) *reinterpret_cast<u32x2 *>(row + (1 + p) * 64 * P) = u32x2{pack2(v[p][0], v[p][1]), pack2(v[p][2], v[p][3])};
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) v[0][e] = gate_act<kGelu>(v[0][e]) * v[1][e];
      }
      *reinterpret_cast<u32x2 *>(row) = u32x2{pack2(v[0][0], v[0][1]), pack2(v[0][2], v[0][3])};
    }
    __syncthreads();
    constexpr int LPR = BNO / 8;               // lanes to a row
#pragma unroll
    for (int i = 0; i < 64 * LPR / 256; ++i) {
      const int r = t / LPR + i * (256 / LPR), c = t % LPR * 8, m = m0 + r, n = n0 + c;
      if (m >= g.M || n >= g.N) continue;
      *reinterpret_cast<u32x4 *>(static_cast<bf16_t *>(g.out) + static_cast<size_t>(m) * g.N + n) = *reinterpret_cast<const u32x4 *>(st + r * P + c);
      if constexpr (kKeep) {
        bf16_t *gu = static_cast<bf16_t *>(g.out2) + static_cast<size_t>(m) * 2 * g.N + n;
        *reinterpret_cast<u32x4 *>(gu) = *reinterpret_cast<const u32x4 *>(st + 64 * P + r * P + c);
        *reinterpret_cast<u32x4 *>(gu + g.N) = *reinterpret_cast<const u32x4 *>(st + 128 * P + r * P + c);
      }
    }
  }
}

template <int EPI, bool ACROSS = false>
static hipError_t launch_ring(GemmArgs g, hipStream_t st) {
  constexpr int BNO = epi_gated(EPI) ? 32 : 64;
  g.grid_m = (g.M + 63) / 64;
  g.grid_n = (g.N + BNO - 1) / BNO;
  const int64_t total = static_cast<int64_t>(g.grid_m) * g.grid_n;
  if (total > INT32_MAX) return hipErrorInvalidValue;
  const int slices = EPI == EPI_SLICE ? (g.K / 64 + g.k_slabs - 1) / g.k_slabs : 1;
  gemm_ring_kernel<EPI, ACROSS><<<dim3(static_cast<unsigned>(total), slices), dim3(256), ring_lds(), st>>>(g);
  return hipGetLastError();
}

template <int EPI>
static hipError_t launch(const GemmArgs &g, int kernel, hipStream_t st) {
  if constexpr (!epi_dgate(EPI)) {             // with 64 x 64 tiles the gradient reads the output map as it lies
    if (kernel == kGatedRing) return launch_ring<EPI>(g, st);
  }
  if (kernel == kGemm256x256) return launch_bf16_pp<2, EPI>(g, st);
  if constexpr (!epi_e4m3(EPI)) {
    if (kernel == kGemm128) return launch_bf16_tc<TileSmall, EPI>(g, st);
  }
  return launch_bf16_pp<1, EPI>(g, st);
}

template <int EPI, bool ACROSS = false>
static hipError_t ring_attr() {
  return hipFuncSetAttribute(reinterpret_cast<const void *>(&gemm_ring_kernel<EPI, ACROSS>), hipFuncAttributeMaxDynamicSharedMemorySize, ring_lds());
}
template <int EPI>
static hipError_t init_one() {
  hipError_t e = set_attr_pp<2, EPI>();
  if constexpr (!epi_dgate(EPI)) {
    if (e == hipSuccess) e = ring_attr<EPI>();
  }
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
  if (e == hipSuccess) e = ring_attr<EPI_SLICE>();
  if (e == hipSuccess) e = ring_attr<EPI_BIAS_ACT>();
  if (e == hipSuccess) e = ring_attr<EPI_SLICE, true>();
  if (e == hipSuccess) e = ring_attr<EPI_BIAS_ACT, true>();
  if (e == hipSuccess) e = ring_attr<EPI_DGATE, true>();
  if (e == hipSuccess) e = ring_attr<EPI_DGATE + 1, true>();
  return e;
}

GatedChoice gated_choose_out(int M, int N, int K, double other) { return gated_choose(M, N, N, K / 64, kEpiAct, g_num_cus, true, false, other); }
GatedChoice gated_choose_dgate(int M, int D, int R, double other) { return gated_choose(M, R, 2 * R, D / 64, kEpiStream, g_num_cus, false, false, other); }

hipError_t launch_gated_out(const GatedChoice &how, const void *a, const void *w, bool across, const float *bias, const float *zeros, void *out, int M, int N, int K, float *part,
                            hipStream_t st) {
  if (M <= 0 || N <= 0 || K <= 0 || K % 64 || N % 64 || (across && how.kernel != kGatedRing)) return hipErrorInvalidValue;
  if (how.slices == 1 && how.kernel != kGatedRing) {
    const int whole = how.kernel == kGemm256x256 ? gated_whole_rounds(M, N, K / 64, kEpiAct, g_num_cus) : M;
    const hipError_t e = launch_gemm_act(how.kernel, a, w, bias ? bias : zeros, out, whole, N, K, st);
    if (e != hipSuccess || whole == M) return e;
    const int64_t at = whole;
    return launch_gated_out(gated_choose(M - whole, N, N, K / 64, kEpiAct, g_num_cus, false, false, 0.0), static_cast<const bf16_t *>(a) + at * K, w, false, bias, zeros,
                            static_cast<bf16_t *>(out) + at * N, M - whole, N, K, nullptr, st);
  }
  GemmArgs g = {};
  g.A = a; g.W = w; g.bias = bias; g.out = out; g.ldo = N; g.tab_rows = 1; g.M = M; g.N = N; g.K = K;
  if (how.slices == 1) return across ? launch_ring<EPI_BIAS_ACT, true>(g, st) : launch_ring<EPI_BIAS_ACT>(g, st);
  g.out = part;
  const int slabs = K / 64;
  g.k_slabs = (slabs + how.slices - 1) / how.slices;
  const hipError_t e = how.kernel != kGatedRing ? launch_bf16_tc<TileSmall, EPI_SLICE>(g, st) : across ? launch_ring<EPI_SLICE, true>(g, st) : launch_ring<EPI_SLICE>(g, st);
  if (e != hipSuccess) return e;
  const int64_t n4 = static_cast<int64_t>(M) * N / 4;
  slice_sum_kernel<<<dim3(static_cast<unsigned>((n4 + 255) / 256)), dim3(256), 0, st>>>(reinterpret_cast<const float4 *>(part), reinterpret_cast<const float4 *>(bias),
                                                                                      static_cast<u32x2 *>(out), (slabs + g.k_slabs - 1) / g.k_slabs, n4, N / 4);
  return hipGetLastError();
}

hipError_t launch_gated_in(const GatedIn &in, bool gelu, hipStream_t st) {
  const bool e4m3 = in.x_scale != nullptr;
  if (in.M <= 0 || in.D <= 0 || in.R <= 0 || in.D % (e4m3 ? 128 : 64) || in.R % 64 || (e4m3 && in.gu)) return hipErrorInvalidValue;
  GemmArgs g = {};
  g.A = in.x; g.W = in.w_in; g.bias = in.b_in; g.out = in.h; g.out2 = in.gu;
  g.ldo = in.R; g.tab_rows = 1; g.M = in.M; g.N = in.R; g.K = in.D;
  g.x_scale = in.x_scale; g.w_scale = in.in_scale;
  const int how = gated_choose(in.M, 2 * in.R, in.R, in.D / (e4m3 ? 128 : 64), in.gu ? kEpiTwo : kEpiGelu, g_num_cus, false, e4m3, 0.0).kernel;
  if (e4m3) return gelu ? launch<EPI_GATED + kEpiE4m3 + 1>(g, how, st) : launch<EPI_GATED + kEpiE4m3>(g, how, st);
  if (in.gu) return gelu ? launch<EPI_GATED + kEpiKeep + 1>(g, how, st) : launch<EPI_GATED + kEpiKeep>(g, how, st);
  return gelu ? launch<EPI_GATED + 1>(g, how, st) : launch<EPI_GATED>(g, how, st);
}

hipError_t launch_gated_dgate(const GatedChoice &how, const void *dy, const void *w, bool across, const void *gu, void *d_gu, int M, int D, int R, bool gelu, hipStream_t st) {
  if (M <= 0 || D <= 0 || R <= 0 || D % 64 || R % 64 || (across && how.kernel != kGatedRing)) return hipErrorInvalidValue;
  GemmArgs g = {};
  g.A = dy; g.W = w; g.out = d_gu; g.gu = gu;
  g.ldo = 2 * R; g.tab_rows = 1; g.M = M; g.N = R; g.K = D;
  if (across) return gelu ? launch_ring<EPI_DGATE + 1, true>(g, st) : launch_ring<EPI_DGATE, true>(g, st);
  return gelu ? launch<EPI_DGATE + 1>(g, how.kernel, st) : launch<EPI_DGATE>(g, how.kernel, st);
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
  if (!wt_in && !wt_out) return hipSuccess;
  TransposeArgs a = {};
  a.src[0] = static_cast<const bf16_t *>(w_in); a.dst[0] = static_cast<bf16_t *>(wt_in); a.rows[0] = 2 * R; a.cols[0] = D;
  a.src[1] = static_cast<const bf16_t *>(w_out); a.dst[1] = static_cast<bf16_t *>(wt_out); a.rows[1] = D; a.cols[1] = R;
  for (int i = 0; i < 2; ++i) a.tiles_c[i] = (a.cols[i] + 63) / 64;
  a.first = wt_in ? (a.rows[0] + 63) / 64 * a.tiles_c[0] : 0;
  const int total = a.first + (wt_out ? (a.rows[1] + 63) / 64 * a.tiles_c[1] : 0);
  gated_transpose_kernel<<<dim3(total), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace reslim
