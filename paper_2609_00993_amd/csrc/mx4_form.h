// Sizes of held MX FP4 matrices and of the products' tiles.  Host arithmetic and
// constants only, so that a test without a GPU can check them.
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

}  // namespace moepd
