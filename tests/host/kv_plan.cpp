// csrc/kv_plan.h by itself.  A line "plan slots least over brief enough unit n (tiles heads length) * n" is followed as the workgroups follow it;
// answers: ranges, units, most tiles of a range, whether every tile's units lie in ranges in order, once, and are held by whom they should.
#include <algorithm>
#include <cstdio>
#include <vector>
#include "kv_plan.h"
using namespace pahq;

// A line "n length rows group unit over": tiles, a couple's units, and the most and the fewest that two tiles of one have
int couples() {
  int n, length, rows, group, unit, over;
  while (std::scanf("%d %d %d %d %d %d", &n, &length, &rows, &group, &unit, &over) == 6) {
    const int tiles = kv_tiles((long long)n * group, rows), base = length - n;
    int most = 0, fewest = 1 << 30;
    for (int i = 0; i < tiles / 2; i++) {
      int sum = 0;
      for (const int tile : {i, tiles - 1 - i}) sum += kv_units_of(kv_tile_end(n, base, tile, rows, group), unit, over);
      most = std::max(most, sum);
      fewest = std::min(fewest, sum);
    }
    std::printf("%d %d %d %d\n", tiles, kv_couple_units(base, tiles, rows, group, unit, over), most, fewest);
  }
  return 0;
}

int main(int argc, char**) {
  if (argc > 1) return couples();
  int slots, least, over, brief, enough, unit, n;
  while (std::scanf("%d %d %d %d %d %d %d", &slots, &least, &over, &brief, &enough, &unit, &n) == 7) {
    std::vector<uint32_t> of;                       // units of each tile, in the line's order
    uint32_t units = 0, pairs = 0, longest = 0;
    for (int i = 0; i < n; i++) {
      int tiles, heads, length;
      if (std::scanf("%d %d %d", &tiles, &heads, &length) != 3) return 1;
      const uint32_t p = kv_pairs(tiles, heads), u = kv_units_of(length, unit, over);
      pairs += p;
      units += kv_units(p, u);
      if (p) longest = std::max(longest, u);
      of.insert(of.end(), p, u);
    }
    const KvPlan plan = kv_plan(units, longest > kv_cut_from(units, pairs, slots, enough, brief), slots, least);
    bool fine = plan.units == units && plan.wgs <= (uint32_t)slots;
    int most = 0;
    if (plan.wgs) {
      std::vector<int> seen(plan.wgs, 0);           // kv_wg_of: every range by one workgroup of the launch
      for (uint32_t block = 0; block < (uint32_t)slots; block++)
        if (const int w = kv_wg_of(block, plan.wgs); w >= 0) fine &= (uint32_t)w < plan.wgs && seen[w]++ == 0;
      for (const int s : seen) fine &= s == 1;
      fine &= kv_from(plan, 0) == 0 && kv_from(plan, plan.wgs) == units;
      uint32_t at = 0;
      for (const uint32_t u : of) {                 // where a tile's parts lie is what the join goes by: neighbouring ranges from its first one on
        uint32_t done = 0;
        int first = -1, parts = 0;
        const int w0 = kv_holder(plan, at), last = kv_holder(plan, at + u - 1);
        for (int w = w0; w <= last; w++) {
          const uint32_t lo = std::max(at, kv_from(plan, w)), hi = std::min(at + u, kv_from(plan, w + 1));
          fine &= lo < hi && lo == at + done;
          done = hi - at;
          if (hi - at <= (uint32_t)over) continue;  // ends among what beginning costs
          if (first < 0) first = w;
          fine &= w == first + parts;
          parts++;
        }
        fine &= done == u && first >= 0 && parts == last - first + 1;
        at += u;
      }
      for (uint32_t w = 0; w < plan.wgs; w++) fine &= kv_holder(plan, kv_from(plan, w)) == (int)w || kv_from(plan, w) == kv_from(plan, w + 1);
      for (uint32_t w = 0; w < plan.wgs; w++) most = std::max(most, (int)(kv_from(plan, w + 1) - kv_from(plan, w)));
    }
    std::printf("%u %u %u %d %d\n", plan.wgs, units, longest, most, (int)fine);
  }
}
