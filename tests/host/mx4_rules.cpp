// Prints what csrc/mx4_rules.h picks: m, n and k in, a form out (-1: the kernel of few rows).
#include <cstdio>
#include "mx4_rules.h"

int main() {
  long long m, n, k;
  while (std::scanf("%lld %lld %lld", &m, &n, &k) == 3) {
    const int slabs = (int)((k + 255) / 256);
    std::printf("%d\n", pahq::mx4_few(m, n, slabs) ? -1 : pahq::mx4_form(m, n, slabs));
  }
  return 0;
}
