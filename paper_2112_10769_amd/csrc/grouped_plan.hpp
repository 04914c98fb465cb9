// Tiles and splits of the products grouped by expert (gemm_grouped.hip), from what the host
// knows of the groups: how many there are, and of how many rows in all.
#pragma once

#include "gemm_kernel.hpp"

namespace luq {

// A grid has below 2^32 threads: 2^23 workgroups of 512.
constexpr int64_t kMostWorkgroups = (int64_t)1 << 23;

// Workgroups of a product of grouped rows: whole tiles of T rows, and one partly filled tile
// for each group that can have rows and for the rows of no group.
static int64_t rows_grid(GemmTile t, int64_t T, int64_t N, int64_t experts) {
  const TileCost& c = kTileCost[kPlanOne][t];
  return ((T >> c.lm) + (experts < T ? experts : T) + 1) * (((N - 1) >> c.ln) + 1);
}

// Workgroups of a split of the weight gradient: every group's tiles, in eighths for the XCDs.
static int64_t depth_grid(GemmTile t, int64_t M, int64_t N, int64_t experts) {
  const TileCost& c = kTileCost[kPlanOne][t];
  return ((((M - 1) >> c.lm) + 1) * (((N - 1) >> c.ln) + 1) + 7) / 8 * 8 * experts;
}

// The tile with the least time by the ungrouped products' cost table.  The host knows the
// mean group only; a group of m rows is taken to need m / BM + 0.6 tiles, and at least one
// (with 1/2, groups of half a tile were taken to fill one each, which unequal ones exceed:
// 64 groups of 127 rows, 4096 -> 1024, took 97 us in 256 x 256 tiles, 59 in 128 x 128).
// Over 420 drawn shapes (1 to 32768 rows, 1 to 128 experts of equal to very unequal load, N
// and K 128 to 16384) the choice loses 3.4% in the geometric mean against the best of the
// eight tiles, 15% at the 95th percentile, 42% at worst; the 128 x 128 tile for all loses
// 40%, 202% and 294%.  Without the 128 x 256 and 64 x 64 tiles the best lose 0.4%: left out.
static GemmTile plan_rows(int64_t T, int64_t N, int64_t K, int64_t experts) {
  const float groups = (float)(experts < T ? experts : T), mean = (float)T / groups;
  GemmTile best = kTile128x128;
  float least = 0.0f;
  for (GemmTile t : {kTile256x256, kTile128x128, kTile64x128, kTile32x64, kTile32x32, kTile64x64k1}) {
    const TileCost& c = kTileCost[kPlanOne][t];
    if (rows_grid(t, T, N, experts) >= kMostWorkgroups) continue;
    const float tiles = mean / (float)(1 << c.lm) + 0.6f;
    const int64_t nb = (int64_t)(groups * (tiles > 1.0f ? tiles : 1.0f)) * (((N - 1) >> c.ln) + 1);
    const int64_t stages = ((K - 1) >> c.lk) + 1;
    float cost = tile_time(c, kPlanOne, nb, (float)(stages << c.lk) * (1.0f / 128));
    if (T * N > kCachedOutputs && c.ln < 7) cost *= kNarrowBeyondCache;
    if (least == 0.0f || cost < least) {
      least = cost;
      best = t;
    }
  }
  return best;
}

struct DepthPlan {
  GemmTile tile;
  int splits;
};

// One group may have all T rows, so a batch beyond the int32-exact length takes at least
// T / kMaxExactK splits: a chunk of any group's stages is then within that length, which
// every stage depth divides.
constexpr int kMostSplits = 16;
constexpr int64_t kMostDepth = kMostSplits * kMaxExactK;

// As plan_rows, for a group of the mean length plus half a stage (its ends lie anywhere in
// one), split where the tiles leave CUs idle.  Over 300 drawn shapes the choice loses 2.9%
// in the geometric mean against the best of eight tiles in 1 to 16 splits, 18% at the 95th
// percentile, 37% at worst; the 128 x 128 tile for all loses 14%, 71% and 456%.
static DepthPlan plan_depth(int64_t T, int64_t M, int64_t N, int64_t experts) {
  DepthPlan best{kTile128x128, 1};
  float least = 0.0f;
  const int64_t outputs = experts * M * N;
  for (GemmTile t : {kTile256x256, kTile128x256, kTile128x128, kTile64x128, kTile32x64, kTile64x64k1}) {
    const TileCost& c = kTileCost[kPlanOne][t];
    if (depth_grid(t, M, N, experts) >= kMostWorkgroups) continue;
    const int64_t tiles = experts * (((M - 1) >> c.lm) + 1) * (((N - 1) >> c.ln) + 1);
    int least_splits = 1;
    while (least_splits * kMaxExactK < T) least_splits *= 2;
    for (int splits = least_splits; splits <= kMostSplits; splits *= 2) {
      const float k = (float)T / (float)experts + 64.0f;
      if (splits > least_splits && (splits * tiles >= 2 * kCus || k < (float)(splits << c.lk))) break;
      const int64_t stages = ((int64_t)(k / (float)splits) >> c.lk) + 1;
      float cost = tile_time(c, kPlanOne, tiles * splits, (float)(stages << c.lk) * (1.0f / 128));
      if (outputs > kCachedOutputs && c.ln < 7) cost *= kNarrowBeyondCache;
      if (splits > 1)
        cost += kSplitCost[kPlanOne].launch + kSplitCost[kPlanOne].per_mout * 1e-6f * (float)outputs * (float)splits;
      if (least == 0.0f || cost < least) {
        least = cost;
        best = DepthPlan{t, splits};
      }
    }
  }
  return best;
}

}  // namespace luq
