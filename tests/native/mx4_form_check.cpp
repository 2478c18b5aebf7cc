// Host side of the MX FP4 products' tiles (csrc/mx4_form.h).
//
// Without arguments: checks, in 64 bits, that the byte offsets a lane forms stay within
// 31 bits whatever the matrix's width, that those of a row which counts lie within its
// tile's resource, and that those of a row which does not lie past every resource.
// With "form gated width rows groups slices expect": prints the form of a launch.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <initializer_list>

#include "mx4_form.h"

using namespace moepd;

int main(int argc, char** argv) {
  if (argc == 8 && !std::strcmp(argv[1], "form")) {
    const Mx4Form f = mx4_form(std::atoi(argv[2]), std::atoll(argv[3]), std::atoll(argv[4]), std::atoi(argv[5]),
                               std::atoi(argv[6]), std::atoll(argv[7]));
    std::printf("%d %d %d %d\n", f.ring, f.blocks, f.panels, f.waves);
    return 0;
  }
  int bad = 0;
  auto check = [&](const char* what, bool holds, int slices, int block, long long at) {
    if (holds) return;
    std::printf("%s: slices %d, block %d: %lld\n", what, slices, block, at);
    ++bad;
  };
  for (int slices : {1, 2, 3, 28, 4095, kMx4MaxSlices})
    for (int first = 0; first < kMx4Rows; ++first)      // where in its block a tile's first row lies
      for (int wave = 0; wave < 4; ++wave)              // ring: the step that a wave moves
        for (int step = 0; step < 4; ++step)            // streaming: the step of a load
          for (int b = 0; b < kRingBlocks; ++b)         // the tile's b-th 32 rows
            for (int row : {0, 31}) {
              const long long bytes = (long long)((first + kMx4Rows * kRingBlocks + 31) / 32) * slices * kMx4SliceBytes;
              const long long unit = (long long)slices * kMx4SliceBytes, added = (wave + step) * kMx4StepBytes;
              const long long none = kMx4Nowhere + b * unit + added;
              check("a row that does not count, past 31 bits", none <= INT_MAX, slices, b, none);
              check("a row that does not count, within the resource", none >= bytes, slices, b, none);
              const long long in = (long long)((first + row) / 32 + b) * unit + 512 + (first + row) % 32 * 16;
              check("a row that counts, past its resource", wave + step > 3 || in + added + 16 <= bytes, slices, b, in + added);
            }
  if (bad) return 1;
  std::printf("ok\n");
  return 0;
}
