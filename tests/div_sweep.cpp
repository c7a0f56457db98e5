// Sweep of the division by a number from the host: (n m) >> s against n / d over divisors and dividends at their edges.
#include "bbmm_div.h"

#include <cstdio>

int main() {
  uint64_t checked = 0;
  auto check = [&](uint32_t d) {
    Div v = div_by(d);
    auto one = [&](uint64_t n) {
      if (n >= ((uint64_t)1 << 31)) return true;
      uint32_t q = (uint32_t)((n * v.m) >> v.s);
      ++checked;
      if (q != n / d) std::printf("%u / %u: %u\n", (unsigned)n, d, q);
      return q == n / d;
    };
    uint64_t most = (((uint64_t)1 << 31) - 1) / d;
    for (uint64_t k = 0; k <= most; k = k < 64 ? k + 1 : k + k / 7 + 1)
      for (int64_t e = -1; e <= 1; ++e)
        if ((int64_t)(k * d) + e >= 0 && !one(k * d + e)) return false;
    for (int64_t e = -2; e <= 1; ++e)
      if ((int64_t)(most * d) + e >= 0 && !one(most * d + e)) return false;
    return one(((uint64_t)1 << 31) - 1) && one(((uint64_t)1 << 31) - 2);
  };
  for (uint32_t d = 1; d <= 70000; ++d)
    if (!check(d)) return 1;
  for (int l = 1; l < 31; ++l)
    for (int64_t e = -3; e <= 3; ++e) {
      int64_t d = ((int64_t)1 << l) + e;
      if (d >= 1 && d < ((int64_t)1 << 31) && !check((uint32_t)d)) return 1;
    }
  for (uint32_t d = 70001; d < 2000000000u; d += d / 5 + 1)
    if (!check(d)) return 1;
  std::printf("ok %llu\n", (unsigned long long)checked);
  return 0;
}
