// Division by a number that a kernel gets from the host.  No device code here: the host's tests sweep it.
#pragma once

#include <stdint.h>

// n / d for 0 <= n < 2^31 and 1 <= d < 2^31 as (n m) >> s: s = 31 + ceil(log2 d), m = ceil(2^s / d), whose product with n is too large by less than
// n d < 2^s.
struct Div {
  uint32_t d, m;
  int s;
};
inline Div div_by(uint32_t d) {
  int l = 0;
  while (((uint64_t)1 << l) < d) ++l;
  uint64_t p = (uint64_t)1 << (31 + l);
  return Div{d, (uint32_t)((p + d - 1) / d), 31 + l};
}
