// The tiles, splits and pieces of the cross entropy of the last layer (cross_entropy.hip), and its workspace,
// from the sizes and types alone.
#pragma once

#include "bf16_tile.hpp"

namespace luq {

namespace {

// Eight waves on 256 x 256 (128 KB of LDS: one workgroup a CU), or four on 128 x 128 (two a CU) where there
// are few tiles: both gradients of 8192 rows on 32000 x 4096 bf16 take 5550 us with 256 x 256 (the products
// 1140 to 1180 TFLOP/s traced), 6580 with 128 x 128; the loss of 8192 on 50021 x 1024 745 and 843.
using BigTile = Bf16Tile<2, 4, 4, 2, 64, 2>;
using SmallTile = Bf16Tile<2, 2, 2, 2, 64, 2>;
// The same alone on its CU: eight waves and three stages under way (the gradients of 300 tokens on 3000 x
// 700 in fp32: 103 us, 112 with four waves and one stage, 111 with three).
using DeepTile = Bf16Tile<4, 2, 1, 2, 64, 4>;
// A few rows, bound by the read of the table, or a few tiles: six stages are under way (two workgroups a CU).
using ThinTile = Bf16Tile<1, 2, 1, 1, 64, 6>;

int64_t up8(int64_t n) { return (n + 7) & ~(int64_t)7; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
// Elements from a laid out row to the next: whole 128-byte lines (the loss of 1000 tokens on 1000 x 1000 in
// fp32: 64 us, 74 with rows of 2000 bytes).
int64_t pitch(int64_t cols) { return ceil_div(cols, 64) * 64; }

// All pairs of na and nb terms whose product is not below 2^-24 of the largest; the smallest
// first, while the sums are small (509 tokens in fp32, gradient of the table: 1.5e-6 of its norm off,
// with the largest first 2.4e-6).
PlanePairs pairs_of(int na, int nb) {
  PlanePairs p{0, 0, 0};
  for (int sum = 2; sum >= 0; --sum)
    for (int i = 0; i < na; ++i) {
      const int j = sum - i;
      if (j < 0 || j >= nb) continue;
      p.a |= (uint32_t)i << (4 * p.count);
      p.b |= (uint32_t)j << (4 * p.count);
      ++p.count;
    }
  return p;
}

// A product's tile and the splits of its reduction, by predicted time: a CU's one large tile takes
// 1.65 us a stage of 64 k, its two small ones 1.0 (0.6 alone), and beginning and end 4 us; the splits'
// sums are written and read again.
enum class Edge { kThin, kSmall, kDeep, kBig };
struct Choice {
  Edge edge;
  int splits;
  double us;   // predicted
};
Choice choose(int64_t M, int64_t N, int64_t stages, int most_splits) {
  Choice best{Edge::kSmall, 1, 1e300};
  for (int big = 0; big < 2; ++big) {
    const int64_t edge = big ? 256 : 128, tiles = ceil_div(M, edge) * ceil_div(N, edge);
    for (int s = 1; s <= most_splits && (s == 1 || stages / s >= 2); ++s) {
      const int64_t groups = tiles * s, slots = big ? 256 : 512;
      const double stage = big ? 1.65 : groups <= 256 ? 0.6 : 1.0;
      double t = (double)ceil_div(groups, slots) * ((double)ceil_div(stages, s) * stage + 4.0);
      if (s > 1) t += 3.0 + (double)s * M * N * 8.0 / 4.5e6;
      if (t < best.us) best = {big ? Edge::kBig : groups <= 256 ? Edge::kDeep : Edge::kSmall, s, t};
    }
  }
  return best;
}

// The logits' tile: up to kThinRows rows are bound by the table's read (one row on 32000 x 4096: 58.6 us, 59.9
// with the tile of 128 x 128; the gradients of 32 rows on 50021 x 1024 118 and 121; the loss of 64 there
// 39 and 28).  So are few tiles with long rows, bound by a CU's loads (0.3 us a stage, 0.36 with two
// tiles a CU): the loss of 1000 rows on 1000 x 1000 fp32 takes 48 us, 65 with 128 x 128, of 3812 on 206 x
// 3144 121 and 176, but of 323 on 6004 x 3364 304 and 199.
constexpr int64_t kThinRows = 32;
Choice choose_logits(int64_t T, int64_t V, int64_t stages) {
  const int64_t groups = ceil_div(T, ThinTile::BM) * ceil_div(V, ThinTile::BN);
  const Choice thin{Edge::kThin, 1, (double)ceil_div(groups, 512) * ((double)stages * (groups <= 256 ? 0.3 : 0.36) + 4.0)};
  if (T <= kThinRows) return thin;
  const Choice other = choose(T, V, stages, 1);
  return thin.us < other.us ? thin : other;
}

// Calls f with the tile.
template <typename F>
auto with_tile(Edge edge, F f) {
  return edge == Edge::kBig     ? f(BigTile{})
         : edge == Edge::kSmall ? f(SmallTile{})
         : edge == Edge::kDeep  ? f(DeepTile{})
                                : f(ThinTile{});
}
static_assert(BigTile::BK == SmallTile::BK && BigTile::BK == ThinTile::BK, "one stage");
constexpr int kStage = BigTile::BK;

struct Carver {
  size_t at = 0;
  size_t take(size_t bytes) {
    const size_t p = at;
    at += (bytes + 255) & ~(size_t)255;
    return p;
  }
};

// How a call is laid out; the same for its workspace query and its launches.
struct Layout {
  int64_t T, V, D, D8, ld;    // ld: of laid out rows
  int xn, tn;                 // terms of x and the table
  bool pack_x, pack_t;        // laid out in rows: fp32, or rows that are no whole 16-byte pieces
  size_t x_rows, t_rows;      // offsets in the workspace
  // forward
  Choice z;                   // the logits' tile
  int64_t parts;
  size_t part, at_target;
  // backward
  int64_t piece, pieces;
  int g_x, g_w;               // terms of g in the product for dx, and in that for dtable
  int tx, xt;                 // terms of the table and of x in these products: two of an fp32 one for a bf16 output
  Choice by_x, by_w;          // the tiles of the products for dx and dtable
  size_t g, sum_x, sum_w;
  bool sums_x;
  size_t bytes;
  // x is laid out in the backward call too where it need not be: a row that is padding becomes
  // zeros, since 0 times what it holds need not be 0.
  Layout(int64_t T_, int64_t V_, int64_t D_, int x_bf16, int t_bf16, bool back) : T(T_), V(V_), D(D_), D8(up8(D_)), ld(pitch(D8)) {
    xn = x_bf16 ? 1 : 3;
    tn = t_bf16 ? 1 : 3;
    pack_x = back || !x_bf16 || (D & 7);
    pack_t = !t_bf16 || (D & 7);
    x_rows = c.take(pack_x ? (size_t)xn * T * ld * 2 : 0);
    t_rows = c.take(pack_t ? (size_t)tn * V * ld * 2 : 0);
  }
  void forward() {
    z = choose_logits(T, V, logits_stages());
    parts = with_tile(z.edge, [&](auto tile) { return ceil_div(V, decltype(tile)::BN); });
    part = c.take((size_t)parts * 3 * T * sizeof(float));
    at_target = c.take((size_t)T * sizeof(float));
    bytes = c.at;
  }
  // The piece: g of 2^27 elements (256 MiB a term), a thousand columns at least.
  void backward(int x_bf16, int g_bf16) {
    int64_t most = ((int64_t)1 << 27) / (T > 0 ? T : 1) & ~(int64_t)127;
    if (most < 1024) most = 1024;
    if (most > (int64_t)1 << 21) most = (int64_t)1 << 21;   // a tile's rows lie within 32-bit offsets
    const int64_t all = ceil_div(V, 128) * 128;
    if (most > all) most = all;
    pieces = ceil_div(V, most);
    piece = ceil_div(ceil_div(V, pieces), 128) * 128;
    pieces = ceil_div(V, piece);
    g_x = x_bf16 ? 1 : 3;
    tx = x_bf16 && tn > 2 ? 2 : tn;
    g_w = g_bf16 ? 1 : 3;
    xt = g_bf16 && xn > 2 ? 2 : xn;
    const int64_t rows = piece < V ? piece : V;
    z = choose_logits(T, rows, logits_stages());
    by_x = choose(T, D, pairs_of(g_x, tx).count * ceil_div(up8(rows), kStage), 64);
    by_w = choose(rows, D, pairs_of(g_w, xt).count * ceil_div(T, kStage), 64);
    g = c.take((size_t)g_terms() * T * piece * 2);
    sums_x = by_x.splits > 1 || pieces > 1;
    sum_x = c.take(sums_x ? (size_t)by_x.splits * T * D * sizeof(float) : 0);
    sum_w = c.take(by_w.splits > 1 ? (size_t)by_w.splits * piece * D * sizeof(float) : 0);
    bytes = c.at;
  }

  int g_terms() const { return g_x > g_w ? g_x : g_w; }
  int64_t logits_stages() const { return pairs_of(xn, tn).count * ceil_div(D8, kStage); }

 private:
  Carver c;
};

}  // namespace

}  // namespace luq
