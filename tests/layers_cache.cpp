// When rows that are packed, unpacked or activated go past the last cache of 256 MB.
// Prints what is wrong; 0: nothing.
#include <cstdio>

#include "../paper_2608_16329_amd/csrc/layers.h"

namespace {
int wrong = 0;
// n rows of `width` values, k entries each in the experts' order (0: no order).
void need(bool want, int64_t n, int k, int width, bool bf16) {
  static const int32_t order = 0;
  mlip::Pack8Args a{};
  a.n = n * (k ? k : 1);
  a.E = 16;
  a.K = k ? k : 1;
  a.width = width;
  a.bf16 = bf16;
  a.order = k ? &order : nullptr;
  if (mlip::pack8_streams(a) != want)
    std::printf("%lld rows of %d values in %d bits, %d entries: not %s the cache\n", (long long)n, width, bf16 ? 16 : 32, k, want ? "past" : "through"), ++wrong;
}
}  // namespace

int main() {
  // without an order: the values' bytes
  need(false, 65536, 0, 2048, true);
  need(true, 65537, 0, 2048, true);
  need(false, 65536, 0, 1024, false);
  need(true, 65536, 0, 1025, false);
  need(true, int64_t(1) << 30, 0, 65536, false);
  need(false, 1, 0, 65536, false);
  // few rows for many experts: rows and codes stay
  need(false, 10240, 16, 1024, true);
  need(false, 20000, 8, 1024, true);
  need(false, 45000, 3, 1024, true);
  need(false, 22000, 3, 1024, false);
  need(false, 40000, 2, 1000, false);
  // they do not fit together
  need(true, 40000, 6, 1000, true);
  need(true, 65536, 4, 1024, true);
  need(true, 131072, 2, 1024, true);
  need(true, 100000, 8, 512, false);
  need(true, 262144, 1, 1024, true);
  need(true, (int64_t(1) << 27) - 1, 16, 65536, false);
  // entries that would fit themselves do so with their codes or not
  need(false, 30000, 4, 1024, true);
  need(false, 131072, 1, 1024, true);
  return wrong != 0;
}
