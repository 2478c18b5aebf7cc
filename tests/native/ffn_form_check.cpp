// Host side of the feed-forward block's tiles (csrc/ffn_form.h).
//
// "form kind rows groups n k": prints the tiles, rows, columns and run of a product.
// "parts rows groups m n": prints the parts of a weight gradient's rows.
// Without arguments: over a range of sizes, checks that every launch covers its rows and columns whatever
// the groups' lengths, and that the parts' sums fit their workspace.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <initializer_list>

#include "ffn_form.h"

using namespace moepd;

int main(int argc, char** argv) {
  if (argc == 7 && !std::strcmp(argv[1], "form")) {
    const FfnForm f = ffn_form(std::atoi(argv[2]), std::atoll(argv[3]), std::atoi(argv[4]), std::atoi(argv[5]),
                               std::atoi(argv[6]));
    std::printf("%d %d %d %d\n", f.tiles, f.rows, f.columns, f.run);
    return 0;
  }
  if (argc == 6 && !std::strcmp(argv[1], "parts")) {
    std::printf("%d\n", ffn_weight_parts(std::atoll(argv[2]), std::atoi(argv[3]), std::atoi(argv[4]), std::atoi(argv[5])));
    return 0;
  }
  int bad = 0;
  auto check = [&](bool holds, const char* what, long long rows, int groups, int n, int k) {
    if (holds) return;
    std::printf("%s: rows %lld, groups %d, n %d, k %d\n", what, rows, groups, n, k);
    ++bad;
  };
  for (long long rows : {1LL, 2LL, 7LL, 8LL, 9LL, 31LL, 33LL, 160LL, 161LL, 1000LL, 30001LL, 1LL << 20, (1LL << 31) - 512})
    for (int groups : {1, 2, 31, 64, 65, 256, 1024})
      for (int n : {8, 16, 24, 264, 768, 7168, 32768})
        for (int k : {8, 64, 72, 520, 7168, 32768}) {
          for (int kind = kFfnGateUp; kind <= kFfnGateUpGrad; ++kind) {
            const FfnForm f = ffn_form(kind, rows, groups, n, k);
            // the most row tiles that any offsets can make: full ones, and one more for each group with a row
            const long long touched = groups < rows ? groups : rows;
            check(f.count >= (rows / f.rows + touched) * f.n_tiles, "too few workgroups", rows, groups, n, k);
            check((long long)f.n_tiles * f.columns >= n && (f.n_tiles - 1LL) * f.columns < n, "columns", rows, groups, n, k);
            check(f.run >= 1 && f.run <= 64, "run", rows, groups, n, k);
            check(f.tiles != kFfnFew8 || (rows <= 8 && f.rows == 8), "rows of the smallest tiles", rows, groups, n, k);
            check(f.tiles != kFfnMid || (f.rows >= 32 && f.rows <= kFfnMidRows && f.rows % 32 == 0), "rows", rows, groups, n, k);
          }
          const int s = ffn_weight_parts(rows, groups, n, k);
          check(s >= 1 && (s == 1 || 4LL * s * groups * n * k <= kFfnPartBytes), "parts", rows, groups, n, k);
        }
  if (bad) return 1;
  std::printf("ok\n");
  return 0;
}
