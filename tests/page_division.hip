// Divider on the host, for tests: built without device code and called through ctypes.
#include "../paper_2307_05908_amd/csrc/ppd_divide.h"

extern "C" uint32_t t_divided(uint32_t x, uint32_t size) { return ppd::Divider(size)(x); }

// the first x below 2^31 beside a multiple of `size` whose quotient is not the compiler's; -1: none (every `step`th multiple is tried, and the last ones)
extern "C" int64_t t_first_wrong(uint32_t size, uint32_t step) {
  const ppd::Divider d(size);
  for (uint64_t m = 0; m < 1ull << 31; m += (uint64_t)size * step)
    for (int64_t x = (int64_t)m - 1; x <= (int64_t)m + 1; ++x)
      if (x >= 0 && x < 1ll << 31 && d((uint32_t)x) != (uint32_t)x / size) return x;
  for (int64_t x = (1ll << 31) - 1; x > (1ll << 31) - 1000; --x)
    if (d((uint32_t)x) != (uint32_t)x / size) return x;
  return -1;
}
