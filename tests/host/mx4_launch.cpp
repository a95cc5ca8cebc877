// Prints what csrc/mx4_rules.h launches for m rows, n columns and k: the form (-1: the kernel of few rows) and the threads it asks for.
#include <algorithm>
#include <cstdio>
#include "mx4_rules.h"

int main() {
  long long m, n, k;
  while (std::scanf("%lld %lld %lld", &m, &n, &k) == 3) {
    const int slabs = (int)((k + 255) / 256);
    if (pahq::mx4_few(m, n, slabs) && pahq::mx4_few_fits(n)) {
      std::printf("-1 %lld\n", (n + 15) / 16 * 512);
      continue;
    }
    const int form = pahq::mx4_form(m, n, slabs);
    const pahq::Mx4Form& f = pahq::mx4_forms[form];
    const long long tiles = ((m + f.tile - 1) / f.tile * ((n + f.tile - 1) / f.tile) + 7) / 8 * 8;
    // one wave a group, a workgroup a tile; the large tiles' workgroups walk: at most two for each of 256 compute units
    std::printf("%d %lld\n", form, f.groups > 1 ? tiles * f.groups * 64 : std::min(tiles, 512ll) * 512);
  }
  return 0;
}
