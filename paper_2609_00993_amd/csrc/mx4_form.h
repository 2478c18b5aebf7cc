// Sizes of held MX FP4 matrices, and the tiles that a product of them takes.  Host
// arithmetic and constants only, so that a test without a GPU can check them, and that the
// shapes of the GPU tests reach every form.
#pragma once

#include <limits.h>

namespace moepd {

constexpr int kMx4Rows = 32;    // rows of a held block
constexpr int kMx4Slice = 256;  // K values that share scale words; the padding of K
constexpr int kMx4SliceBytes = 4096;  // codes of 32 rows x 256 values
constexpr int kMx4SliceScales = 256;  // their scales
constexpr int kMx4StepBytes = 1024;   // codes of 32 rows x 64 values, one MFMA's operand
constexpr int kMx4MaxSlices = (1 << 20) / kMx4Slice;

constexpr int kRingSlots = 3, kRingBlocks = 4;  // of a ring tile: slices in LDS, blocks of 32 rows

// A tile's rows start anywhere in a held block, so they lie in one block more than they fill.
// What a lane adds to its place within the first: whole blocks, and one of the four steps of a
// slice, which a ring's wave adds once and a streaming tile's loads each.
constexpr long long kMx4MostBytes = (kRingBlocks + 1LL) * kMx4MaxSlices * kMx4SliceBytes;
constexpr long long kMx4MostAdded = (kRingBlocks - 1LL) * kMx4MaxSlices * kMx4SliceBytes + 2 * 3 * kMx4StepBytes;

// The place of a lane whose row does not count: past every resource, and with all that is
// added still a positive int.
constexpr int kMx4Nowhere = 0x7c000000;
static_assert(kMx4Nowhere >= kMx4MostBytes, "within a resource");
static_assert(kMx4Nowhere + kMx4MostAdded <= INT_MAX, "the sum passes 31 bits");

// The tiles of a launch.
struct Mx4Form {
  bool ring;         // LDS ring tiles, else streaming tiles
  int blocks;        // 32-row blocks of a tile at most: 4, streaming 1 or 2
  int panels;        // panels of 32 weight rows that a wave takes
  int waves;         // waves of a workgroup: ring side by side along the weights, streaming along K
  int n_tiles;       // column tiles (streaming: rounded up to a multiple of 8)
  int run;           // consecutive ring tiles that go to one XCD
  long long groups;  // workgroups

  int threads() const { return 64 * waves; }
  // Dynamic LDS: where a streaming tile's waves meet.
  int lds() const { return ring || waves == 1 ? 0 : waves * blocks * panels * 4096; }
  bool fits() const { return groups <= 0x7fff0000LL; }
};

constexpr int kStreamWaves = 8;

// width: output columns, whole slices of them where they are MX FP4; expect: how many of the
// `rows` rows are expected to be in use, 1 at least.
inline Mx4Form mx4_form(bool gated, long long width, long long rows, int weights, int slices, long long expect) {
  const long long touched = weights < expect ? weights : expect;  // groups that have a row
  const int mean = (int)(expect / touched);
  // Expected tiles of bm rows and bn columns.
  auto tiles_of = [&](int bm, int bn) { return (width + bn - 1) / bn * (expect / bm + touched); };
  Mx4Form f{};
  int bn = gated ? 128 : 256;
  // Ring tiles from 16 rows a group on (32 gated), if there are enough for many CUs.  us, ring / streaming tiles: 18
  // rows in each of 64 groups, 2560 x 768, 18.4 / 19.3; 20 in each of 32, 7168 x 2048, 41.8 / 42.9, and
  // gated, 2048 x 7168, 89.7 / 88.0; 28 in each of 64, gated, 768 x 2560, 31.4 / 29.0.  One matrix of
  // 7168 x 7168: 128 rows (28 ring tiles) 28.6 / 18.2, 256 (56) 28.1 / 22.2, 512 (112) 28.6 / 36.1.
  f.ring = mean >= (gated ? 32 : 16) && tiles_of(32 * kRingBlocks, bn) >= 100;
  if (f.ring) {
    f.blocks = kRingBlocks;
    f.panels = 2;
    f.waves = 4;
  } else {
    f.blocks = mean > 32 ? 2 : 1;
    // panels of 32 columns where those of 64 would leave CUs idle
    f.panels = gated || tiles_of(32 * f.blocks, 64) >= 256 ? 2 : 1;
    bn = gated ? 32 : 32 * f.panels;
    // waves to share a tile, enough to keep the memory busy, 8 to a CU
    f.waves = 1;
    while (f.waves < kStreamWaves && tiles_of(32 * f.blocks, bn) * f.waves < 8 * 256 && f.waves * 2 <= slices) f.waves *= 2;
  }
  const int round = f.ring ? 1 : 8;
  f.n_tiles = (int)((width + bn - 1) / bn + round - 1) / round * round;
  f.run = mean >= 512 ? 64 : 32;
  // row tiles: at most one that is not full for each group that may have a row
  const long long tiles = (rows / (32 * f.blocks) + (weights < rows ? weights : rows)) * f.n_tiles;
  f.groups = f.ring ? (tiles + 8 * f.run - 1) / (8 * f.run) * (8 * f.run) : tiles;  // ring: whole rounds
  return f;
}

}  // namespace moepd
