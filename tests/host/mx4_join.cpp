// Prints the rows a workgroup that joins partial sums reads of a residual: per line of input (tile, threads, columns, elements of an
// access, rows left in the matrix) every row of the tile a thread is let have, with the element it starts at.
#include <cstdio>
#include "mx4_rules.h"

int main() {
  int tile, threads, columns, each, left;
  while (std::scanf("%d %d %d %d %d", &tile, &threads, &columns, &each, &left) == 5) {
    const int across = columns / each, down = threads / across;
    for (int t = 0; t < threads; t++)
      for (int r = 0; r < (tile + down - 1) / down; r++)
        if (pahq::mx4_in_tile(t / across + r * down, tile, left)) std::printf("%d:%d ", t / across + r * down, t % across * each);
    std::printf("\n");
  }
  return 0;
}
