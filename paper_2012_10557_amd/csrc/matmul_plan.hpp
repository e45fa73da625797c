// Which kernel a matrix product takes: the rules on its sizes, in host code alone.
#pragma once

#include <algorithm>

namespace ekya {

inline long long mm_ceil(long long a, long long b) { return (a + b - 1) / b; }

struct MmPlan {
  int tile;            // outputs of a tile in either direction
  int splits, stages;  // stages of a split (of a group of waves)
  int groups;          // of waves in a block
};
// Which tile, and into how many parts the reduction is split.
//
// 256 x 256 (bf16 with DMA only) takes about 10 us and 1.58 us a stage for every
// round of 256 tiles, one a CU; 128 x 128 about 5 us and 2.3 us and 0.46 us a
// stage for every 256 tiles, two at a time on a CU, so that no round is waited
// for.  Measured, 256 against 128: 8192^3 826 and 962 us, 4096^3 114 and 123,
// 6272 x 2048 x 512 (200 tiles of 256) 23.2 and 25.2, 25088 x 1024 x 256 30.4 and
// 31.1, 2048^3 (64 tiles of 256) 53.6 and 27.4.
//
// Up to 256 tiles of 128 with a reduction long enough for 512 parts of 8 stages,
// two ways of giving every CU two parts: two groups of waves a block, each with a
// part of the reduction, whose sums meet in LDS, or two blocks of one group.  A
// stage takes 1.42 us in the two groups and 1.10 in the two blocks, which in turn
// leave twice the partial sums and fill CUs that 256 / tiles rounded down leaves
// idle.  Two groups against two blocks: 2040^2 x 2264 33.7 and 39.9 us, 760^2 x 7448
// 28.0 and 29.5, 500^2 x 35992 39.6 and 41.4, but 1500^2 x 3992 (144 tiles) 47.8 and
// 38.6, 1280 x 1150 x 12760 83.5 and 62.9, 896 x 900 x 18008 60.6 and 53.8.  One
// group unsplit or 64 x 64 against the better of the two: 2040^2 x 2264 36.8 and 33.7,
// 1500^2 x 3992 52.0 and 38.6, 760^2 x 7448 31.6 and 28.0; dw of 6272 x 512 x 2048 31.5 and
// 28.0, of 25088 x 256 x 1024 30.7 and 27.1.
//
// With less than 192 tiles of 128 most CUs hold one block or none: 64 x 64, and
// the reduction split until 512 blocks run where a part is still 32 stages
// long, else until 256 do (one a CU, three stages in flight).  128 against 64:
// 1000^3 14.8 and 9.2 us, 512^3 10.3 and 6.0, but with 256 tiles of 128 2048^3
// 27.4 and 28.0.  256 against 512 blocks: 128 x 2048 x 8192 (parts of 32 and 16
// stages) 12.6 and 15.7, 256 x 1024 x 25088 (98 and 49) 40.6 and 33.4.  A part has
// 16 stages at least (1024 x 512 x 4096 in parts of 32, 16 and 8: 21.6, 17.5 and
// 19.2), 4 without DMA, whose stages take longer.
//
// fp32 is bound by the matrix cores with a block or two a CU already, so tile and
// parts are those with the least estimated time: a launch and what surrounds the
// stages (4 us, 128 x 128 6), stages at what they take alone on a CU and with
// other blocks beside them, adding up the parts (2 us and their traffic at 5.7
// TB/s).  The constants are fitted to either tile and up to 16 parts of 70 sizes
// (on those and 50 more the choice is 0.3% slower than the best of them on average,
// 5% at most).  Without DMA a block alone on its CU waits for its loads.
// 1000^3 in one part of 64 x 64 23.7 us, in two 27.3; 1500^3 78.6 and, in three, 73.2;
// 1001 x 513 x 771 20.2 and, in two, 22.4; 212 x 5079 x 2955 in four parts of 64 x 64
// 82.1, in ten of 128 x 128 89.7; 2048 x 520 x 2048 in 128 x 128 42.8, in 64 x 64 46.6;
// 25088 x 256 x 256 dw in 8 parts 80.7, in 16 45.4; 7 x 320 x 976 dx in 7 parts of 5
// stages 9.7, in 16 of 2 7.9.
inline MmPlan mm_fp32_plan(long long R, long long C, long long ns, bool dma) {
  MmPlan best{};
  double least = 1e30;
  for (int tile : {64, 128}) {
    const double alone = tile == 64 ? (dma ? 0.64 : 0.91) : dma ? 1.95 : 2.7;
    const double beside = tile == 64 ? (dma ? 0.56 : 0.68) : dma ? 1.95 : 2.4;
    for (int s = 1; s <= 16 && s <= ns; ++s) {
      const long long stages = mm_ceil(ns, s), blocks = mm_ceil(mm_ceil(R, tile) * mm_ceil(C, tile) * s, 256);
      const double us = (tile == 64 ? 4 : 6) + stages * (blocks == 1 ? alone : beside * blocks) +
                        (s > 1 ? 2 + s * (double)R * C * 8 / 5.7e6 : 0);
      if (us < least) {
        least = us;
        best = {tile, (int)mm_ceil(ns, stages), (int)stages, 1};
      }
    }
  }
  return best;
}
inline MmPlan mm_plan(long long R, long long C, long long Tn, bool fp32, bool dma) {
  const long long ns = std::max(1LL, mm_ceil(Tn, fp32 ? 32 : 64));
  const long long t256 = mm_ceil(R, 256) * mm_ceil(C, 256), t128 = mm_ceil(R, 128) * mm_ceil(C, 128);
  if (fp32) return mm_fp32_plan(R, C, ns, dma);
  if (dma && t256 >= 192 &&
      mm_ceil(t256, 256) * (10 + 1.58 * ns) <= 5 + t128 / 256. * (2.3 + 0.46 * ns))
    return {256, 1, (int)ns, 1};
  if (dma && std::min(R, C) >= 128 && t128 <= 256 && ns * t128 >= 512 * 8) {
    const long long parts = 256 / t128, blocks = 512 / t128;  // of the reduction, for two groups and for one
    const long long two = mm_ceil(ns, 2 * parts), one = mm_ceil(ns, blocks);
    const double adding = (double)R * C * 8 / 5.7e6;  // a part's sums, written and read
    if (1.42 * two + (parts > 1 ? 2 + parts * adding : 0) <= 1.10 * one + 2 + blocks * adding)
      return {128, (int)mm_ceil(ns, 2 * two), (int)two, 2};
    return {128, (int)mm_ceil(ns, one), (int)one, 1};
  }
  if (t128 >= 192) return {128, 1, (int)ns, 1};
  const long long t64 = std::max(1LL, mm_ceil(R, 64) * mm_ceil(C, 64));
  const long long blocks = !dma || ns * t64 >= 512 * 32 ? 512 : 256;
  const long long want = std::max(1LL, std::min(blocks / t64, ns / (dma ? 16 : 4)));
  const int stages = (int)mm_ceil(ns, want);
  return {64, (int)mm_ceil(ns, stages), stages, 1};
}

// Whether operands off 16 bytes are worth a padded copy.  Through registers a
// bf16 product runs at about 300 TFLOP/s, with copies to LDS at 1100; a copied
// element costs 4 bytes of traffic, so both directions of the result have to
// be some hundreds long, and the product long enough for two more launches
// (16384 x 2047 x 8192: 1812 us without).
inline bool mm_pack(bool fp32, long long R, long long C, long long Tn) {
  return !fp32 && R * C >= 256 * (R + C) && (double)R * C * Tn >= 2e9;
}

}  // namespace ekya
