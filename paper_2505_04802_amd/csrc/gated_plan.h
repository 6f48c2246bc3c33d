// Which kernel a product of the gated feed-forward layer gets, and into how many slices its sum is cut (gated_gemm.hip).  Arithmetic
// only: the CPU test compiles it too and holds the choice against measured times.
#pragma once

#include "gemm_plan.h"

namespace reslim {

constexpr int kGatedRing = 1;      // 64 x 64 tiles; beside the kernels of GemmKernel
struct GatedChoice {
  int kernel, slices;              // slices > 1: the ring or the 128 x 128 tiles
  double us;
};

constexpr double kMostTiles = 1 << 23;      // work-groups of 256 threads that one launch takes; the persistent kernels need one for every compute unit

// The smallest of the estimates of gemm_times and of those for the 64 x 64 tiles, in microseconds beside what every launch costs.  A slab of these takes
// a work-group 0.26 us, its latency over the three in flight, while two lie on a compute unit, and a compute unit 0.27, what it draws
// from L2 for one.  Slices of k make more work-groups of shorter sums, at the price of a second launch and of partial sums that are read
// again.  gemm_times is fitted to products whose weights lie in a cache; a model's come from memory, and where every work-group has one tile a slab
// then takes a persistent kernel 0.8 us (128 x 256) and 1.35 (256 x 256): 64 x 4096 x 10,944 140 us instead of 79.
//   Whole products of the output map and of dx that neither the ring nor slices win are hundreds of tiles reading the same rows of W, and there 0.8 and 1.35 us
// overrate memory: of 95 with cold weights the kernel that they would choose is 0.6 % slower than the best of the three, 1448 x 2112 x 4864 120 us instead of
// 115, the choice by gemm_times itself 0.4 %.  So that is what these get; where it sees no difference (0.2 %) between kernels with a tile or less for a
// compute unit, as at 1616 x 2048 x 2048 (62.6 and 62.4 us), 128 x 128, which leaves the launches around it their clock.
//   N: rows of W that are read (both matrices of a gated product); cols: columns of the result; slabs: K in slabs of 128 bytes a row; other: what the
// kernels beside the ring cost on top (copies of weights that it does without).
inline GatedChoice gated_choose(int M, int N, int cols, int slabs, GemmEpi epi, int cus, bool sliceable, bool e4m3, double other) {
  constexpr double ring_epi[] = {0.8, 1.0, 1.5, 1.0, 2.0};
  const GemmTimes g = gemm_times(M, N, slabs * 64, epi, cus);
  auto count = [&](int bm, int bn) { return static_cast<double>((M + bm - 1) / bm) * ((N + bn - 1) / bn); };
  const double tiles = count(64, 64), mid = count(128, 128);
  GatedChoice best = {kGemm256x256, 1, (count(256, 256) <= cus ? std::max(g.pp2, slabs * 1.35) : g.pp2) + other};
  auto offer = [&](int kernel, int slices, double us) {
    if (us < best.us) best = {kernel, slices, us};
  };
  offer(kGemm128x256, 1, (count(128, 256) <= cus ? std::max(g.pp1, slabs * 0.8) : g.pp1) + other);
  if (!e4m3 && mid <= kMostTiles) offer(kGemm128, 1, g.small + other);
  for (int s = 1; s <= 32 && (s == 1 || slabs / s >= 4); ++s) {
    if (s > 1 && !sliceable) break;
    const int per = (slabs + s - 1) / s, n = (slabs + per - 1) / per;
    if (tiles * n > kMostTiles) break;
    const double rounds = std::ceil(tiles * n / (2.0 * cus)), add = n > 1 ? 2.4 + 5e-6 / 4.5 * n * M * static_cast<double>(cols) : 0.0;
    offer(kGatedRing, n, 0.5 + std::max(rounds * per * 0.26, tiles * n * per * 0.27 / cus) + rounds * ring_epi[epi] + add);
    if (s > 1 && mid * n <= 3.0 * cus) {                   // 128 x 128 tiles, up to three on a compute unit
      const double ws = mid * n / cus, fs = std::min(1.0, std::max(0.0, (0.62 * std::ceil(ws) + 0.38 * ws - 1.0) / 2.0));
      offer(kGemm128, n, per * (0.73 + 1.07 * fs) + 5.99 * (0.12 + 0.88 * fs) + add + other);
    }
  }
  if (!e4m3 && epi == kEpiAct && best.kernel != kGatedRing && best.slices == 1) {
    const double persistent = std::min(g.pp1, g.pp2), tie = count(128, 256) <= cus ? 0.998 : 1.0;
    best.kernel = mid <= kMostTiles && tie * g.small <= persistent ? kGemm128 : g.pp1 < g.pp2 ? kGemm128x256 : kGemm256x256;
  }
  return best;
}

// Rows of a product on 256 x 256 tiles that fill whole rounds of them, where the rows of the last, part-filled round are faster in a launch of
// their own (any kernel, no slices) by 5 % of the whole; else all rows.  Every kernel sums k in the same order, so the result does not depend on it.
// Layers in one launch and in two: 17,000 x 2048 x 8192 1373 and 1276 us, 9000 x 4096 x 2752 534 and 522, 40,352 x 1024 x 2752 588 and 576, its
// gradient 1416 and 1391; where 3 % are promised (80,704 x 1536 x 2752) two lose up to 1 %.
inline int gated_whole_rounds(int M, int N, int slabs, GemmEpi epi, int cus) {
  const int64_t across = (N + 255) / 256, rounds = (M + int64_t{255}) / 256 * across / cus, rows = rounds * cus / across * 256;
  if (rounds < 1 || rows >= M) return M;
  const int whole = static_cast<int>(rows);
  const double all = gemm_times(M, N, slabs * 64, epi, cus).pp2, part = gemm_times(whole, N, slabs * 64, epi, cus).pp2;
  return part + gated_choose(M - whole, N, N, slabs, epi, cus, false, false, 0.0).us + 2.0 < 0.95 * all ? whole : M;
}

}  // namespace reslim
