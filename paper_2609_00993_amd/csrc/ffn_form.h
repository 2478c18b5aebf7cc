// Which tiles a product of the gated feed-forward block takes (ffn_block.hip), by sizes alone.  Plain
// arithmetic, compiled for the host too, where a test asks for it.
#pragma once

namespace moepd {

enum FfnKind : int { kFfnGateUp = 0, kFfnDown = 1, kFfnDownGrad = 2, kFfnGateUpGrad = 3, kFfnWeightGrad = 4 };

// kFfnFew8, kFfnFew32: up to 8 or 32 rows and 32 or 64 columns, K dealt among the waves; kFfnMid: up to `rows`
// (32 to 160) rows and 256 columns (gate/up: 128 of each), cut to the 32-row blocks they hold; kFfnWide: 256 rows.
enum FfnTiles : int { kFfnFew8 = 0, kFfnFew32 = 1, kFfnMid = 2, kFfnWide = 3 };

constexpr int kFfnMidRows = 160, kFfnWideRows = 256, kFfnCus = 256;

// Columns of a few tile: gate/up of up to 8 rows 16 of each, which spreads one token's weights over twice the CUs (I
// 2048: 128).
constexpr int ffn_few_columns(int kind, int rows) {
  return kind == kFfnGateUp ? (rows == 8 ? 16 : 32) : kind == kFfnDown ? 32 : 64;
}

struct FfnForm {
  int tiles;          // FfnTiles
  int rows, columns;  // of a tile at most
  int run;            // consecutive tiles that go to one XCD
  int n_tiles;
  long long count;    // workgroups at most
  int threads() const { return tiles == kFfnFew8 ? 512 : 256; }
};

// Whether groups of `mean` rows, of which some have a few more or less, suit wide tiles: not around a
// full tile and a small rest, where tiles of 160 rows share the rows better.  32 groups, H 7168, I 2048, gate/up and down,
// us, mid / wide: 200 rows 501 / 428 and 256 / 244; 257 559 / 558 and 291 / 294 (drawn lengths: 527 / 579 and 300 / 269);
// 300 597 / 614 and 316 / 322; 400 812 / 777 and 428 / 385; 550 1086 / 1024 and 553 / 514.  One rule for
// every kind: down alone would take wide tiles at 257 drawn rows too.
constexpr bool ffn_wide_fits(int mean) {
  return (mean > kFfnMidRows && mean <= kFfnWideRows - 24) || mean >= kFfnWideRows + 96;
}

// rows in `groups` groups, n columns, K values to a sum.  The times behind the rule, in ns with every CU at work:
// a slice of 64 of K takes a mid tile 300 + 105 for each 32-row block, a wide one 1170, a few tile's start and
// join 3000 and each value of K 2; mid and wide tiles start and end in 3000.  Measured, one group, us, mid / few: 128 rows, H
// 7168, I 2048, gate/up 79 / 20, down 26 / 19; 512 rows, H 2048, I 1024, 46 / 14 and 24 / 14; 1000 rows, H 7168, I 2048,
// gate/up 131 (wide) / 138, down 43 / 118, and what the rule takes there, mid tiles of 64 and 128 rows, 69 and 33; 500 rows
// there, mid tiles of 160 / 96 / 64 rows, 81 / 68 / 57 (the rule's, of 32: 52).  32 groups of one row, H 2560, I 768: gate/up
// 37 / 41.
inline FfnForm ffn_form(int kind, long long rows, int groups, int n, int k) {
  const long long touched = groups < rows ? groups : rows;  // groups that have a row, if shared evenly
  const int mean = (int)((rows + touched - 1) / touched);
  auto up = [](long long a, long long b) { return (a + b - 1) / b; };
  FfnForm best{};
  double least = 0;
  auto consider = [&](int tiles, int bm, int bn, auto&& tile_ns) {
    const int here = (int)up(mean, bm);  // row tiles of a group
    const long long count = touched * here * up(n, bn);
    const double rounds = count <= 4 * kFfnCus ? (double)up(count, kFfnCus) : (double)count / kFfnCus;
    const double ns = rounds * tile_ns((int)up(up(mean, 32), here));
    if (best.columns && ns >= least) return;
    least = ns;
    best.tiles = tiles;
    best.rows = bm;
    best.columns = bn;
    best.n_tiles = (int)up(n, bn);
    best.run = count >= 8 * 32 ? 32 : count >= 16 ? (int)(count / 8) : 2;
    best.count = (rows / bm + touched) * best.n_tiles;
  };
  const int bn = kind == kFfnGateUp ? 128 : 256;
  const double slices = (double)up(k, 64);
  if (ffn_wide_fits(mean)) {
    // full tiles, and a rest of its own height or, a small one, half and half with a full one
    const int full = mean / kFfnWideRows, rest = (int)up(mean % kFfnWideRows, 32);
    auto mid_ns = [](int blocks) { return blocks ? 300.0 + 105 * blocks : 0; };
    const double ns = rest > kFfnMidRows / 32 ? 1170.0 * (full + 1)
                      : rest <= 2 && rest && full ? 1170.0 * (full - 1) + mid_ns((9 + rest) / 2) + mid_ns((8 + rest) / 2)
                                                  : 1170.0 * full + mid_ns(rest);
    consider(kFfnWide, kFfnWideRows, bn, [&](int) { return 3000 + ns / (full + (rest ? 1 : 0)) * slices; });
  }
  for (int bm = kFfnMidRows; bm >= 32; bm -= 32)
    consider(kFfnMid, bm, bn, [&](int blocks) { return 3000 + (300 + 105 * blocks) * slices; });
  const bool few8 = rows <= 8;
  consider(few8 ? kFfnFew8 : kFfnFew32, few8 ? 8 : 32, ffn_few_columns(kind, few8 ? 8 : 32), [&](int) { return 3000 + 2.0 * k; });
  return best;
}

constexpr int kFfnWeightRows = 128, kFfnWeightCols = 256;  // of a tile of the weights' gradients
constexpr long long kFfnPartBytes = 1LL << 27;            // of the parts' sums, at most

// Parts that a group's rows are cut into, each with float32 sums of its own which a second launch
// adds: where tiles are few and rows many.  In ns: a slice of 32 rows takes a tile 500 alone on
// its CU and 830 beside another, the parts' sums 8 bytes a value to write and read at 4500 bytes, a launch 4000.
// Measured, one group, us: 1000 rows, 2048 x 2048, one part 20, three 38; 16000 rows, 512 x 512, 20 parts 24, 62 parts 66;
// 16000 rows, 2048 x 2048, two 147, four 137.
inline int ffn_weight_parts(long long rows, int groups, int m, int n) {
  const long long tiles = (long long)groups * ((m + kFfnWeightRows - 1) / kFfnWeightRows) *
                          ((n + kFfnWeightCols - 1) / kFfnWeightCols);
  const double values = (double)groups * m * n;
  const long long slices = (rows / groups + 31) / 32;
  int best = 1;
  double least = 0;
  for (int s = 1; s <= 64 && (s == 1 || (s <= slices / 4 && 4 * s * values <= kFfnPartBytes)); ++s) {
    const long long wgs = tiles * s;
    const double rounds = wgs <= kFfnCus ? 500 : 830.0 * ((wgs + 2 * kFfnCus - 1) / (2 * kFfnCus));
    const double ns = rounds * ((slices + s - 1) / s) + (s > 1 ? 4000 + s * values * 8 / 4500 : 0);
    if (s > 1 && ns >= least) continue;
    least = ns;
    best = s;
  }
  return best;
}

}  // namespace moepd
