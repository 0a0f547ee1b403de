// The page of a group of 16 rows by the library's own division (page_internal.hpp), on the host:
// every page size, at each border of a quotient that lies near the ends of the groups that a
// table may have, or at one of `every` borders between.
#include <cstdio>

#include "page_internal.hpp"

int main() {
  const int top = (1 << 25) + 4096;   // groups of a table of 2^29 rows, rounded up to whole pages
  const int every = 997;
  long long checked = 0, wrong = 0;
  for (int D = 1; D <= 4096; ++D) {
    const vase::PageDiv v = vase::page_div(16 * D);
    const int last = top / D;
    auto check = [&](int q) {
      for (int n = q * D - 1; n <= q * D + 1; ++n)
        if (n >= 0 && n <= top) {
          ++checked;
          if (vase::page_of_group(v, n) != n / D) {
            if (!wrong++) std::printf("group %d, %d to a page: %d\n", n, D, vase::page_of_group(v, n));
          }
        }
    };
    for (int q = 0; q < last - 40; q += q < 40 ? 1 : every) check(q);
    for (int q = last > 40 ? last - 40 : 0; q <= last; ++q) check(q);
    if (v.groups != (uint32_t)D) ++wrong;
  }
  std::printf("%lld checked, %lld wrong\n", checked, wrong);
  return wrong != 0;
}
