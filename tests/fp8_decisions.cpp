// Decisions of the host about products whose sizes no test can run: which results the copy engine takes out, rows of a group.
#include <cstdio>

#include "fp8_internal.h"

using namespace b2c;

int main() {
  int wrong = 0;
  auto check = [&](bool ok, const char* what, long long n) {
    if (!ok && ++wrong <= 10) std::printf("%s, %lld\n", what, n);
  };
  // a copy's coordinate is a byte of the row, in 32 bits with a sign
  const int types[3] = {B2C_F32, B2C_F16, B2C_BF16};
  for (int t : types)
    for (long long n = 64; n <= 1 << 30; n *= 2)
      for (long long d = -64; d <= 64; d += 16) {
        MatmulArgs a = {};
        a.y = (void*)4096;
        a.y_type = t;
        a.N = (int)std::min(n + d, 1ll << 30);
        if (a.N < 16) continue;
        a.ldy = a.N;
        const long long last = (a.N - 1ll) * type_bytes(t);
        check(results_by_copy(a) == (last < (1ll << 31) && a.N * (long long)type_bytes(t) < (1ll << 31)), "copied columns", a.N);
        a.ldy = a.N + 1;
        check(!results_by_copy(a), "rows off the grid", a.N);
        a.ldy = a.N;
        a.y = (void*)(4096 + type_bytes(t));
        check(!results_by_copy(a), "first row off the grid", a.N);
      }
  // with groups the average chooses the kernel
  const int32_t offsets[2] = {0, 0};
  for (long long rows : {1ll, 1000ll, 1ll << 30, kMaxRows - 1000, kMaxRows})
    for (int groups : {1, 2, 3, 256, 257, 700, kMaxExperts}) {
      MatmulArgs a = {};
      a.rows = (int)rows;
      a.groups = groups;
      a.offsets = offsets;
      const long long n = rows_of_a_group(a);
      check(n * groups >= rows && (n - 1) * groups < rows, "rows of a group", rows);
      a.offsets = nullptr;
      check(rows_of_a_group(a) == rows, "rows without groups", rows);
    }
  return wrong ? 1 : 0;
}
