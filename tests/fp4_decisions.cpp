// Decisions of the host about 4-bit products by groups whose sizes no test can run: rows of a group and of its tiles.
#include <cstdio>

#include "fp4_internal.h"

using namespace b2c;

int main() {
  int wrong = 0;
  auto check = [&](bool ok, const char* what, long long n) {
    if (!ok && ++wrong <= 10) std::printf("%s, %lld\n", what, n);
  };
  const int32_t offsets[2] = {0, 0};
  // (half as many rows again as a group has on average pass 32 bits from 1431655766 rows on)
  for (long long rows : {1ll, 10ll, 11ll, 21ll, 22ll, 42ll, 43ll, 44ll, 1000ll, 1ll << 30, 1431655765ll, 1431655766ll, 1ll << 31, kMaxRows - 1000, kMaxRows})
    for (int groups : {1, 2, 3, 256, 257, 700, kMaxExperts}) {
      if (rows > kMaxRows) continue;
      Matmul4Args a = {};
      a.rows = (int)rows;
      a.groups = groups;
      a.offsets = offsets;
      const long long n = rows_of_a_group(a), tile = rows_of_a_group_tile(a);
      check(n * groups >= rows && (n - 1) * groups < rows, "rows of a group", rows);
      check(tile >= std::min(n + n / 2, 128ll) && (tile == 16 || tile / 2 < n + n / 2), "rows of a tile", rows);
      // the kernel for few rows can launch its tiles
      check(tile == 128 || rows / tile + std::min<long long>(groups, rows) <= 65535, "tiles of few rows", rows);
      a.offsets = nullptr;
      check(rows_of_a_group(a) == rows, "rows without groups", rows);
    }
  return wrong ? 1 : 0;
}
