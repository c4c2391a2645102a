// Decisions of the host about products whose sizes no test can run: which results the copy engine takes out.
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
  return wrong ? 1 : 0;
}
