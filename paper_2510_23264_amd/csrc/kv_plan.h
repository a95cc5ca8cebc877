// How the attention over a paged cache is shared out to workgroups.  No GPU type in it, so that CPU tests compile it.
//
// The rows of a sequence and a cache head are (new token, query head of the group) pairs, in tiles of `rows`; a tile's work is its
// sequence's length, in units of some rows of the cache.  The host knows neither the lengths nor how the tokens are spread over the
// sequences, so each workgroup finds its part from the batch.  Where no tile is longer than what a workgroup would do on average, tiles
// are given out whole, as workgroups end.  Otherwise the units of all tiles, heads and sequences stand in one line, which is cut into
// equal ranges for at most `slots` workgroups, about as many as the chip holds at a time: one long sequence beside short ones, or
// one alone, takes the whole chip.  A range ends inside tiles at its ends only, so every workgroup leaves at most two parts
// of tiles in the workspace: in slot 2 w what it began inside of a tile, in slot 2 w + 1 what it left unfinished.
#pragma once
#include <stdint.h>

#ifndef PAHQ_HD
#ifdef __HIPCC__
#define PAHQ_HD __host__ __device__ __forceinline__
#else
#define PAHQ_HD inline
#endif
#endif

namespace pahq {

constexpr int KV_MOST_ITEMS = 1 << 24;              // workgroups of a launch, whose threads are counted in 32 bits
PAHQ_HD int kv_tiles(long long rows, int tile) { return (int)((rows + tile - 1) / tile); }
PAHQ_HD int kv_units_of(int length, int unit) { return length <= unit ? 1 : (int)(((uint32_t)length + (uint32_t)unit - 1) / (uint32_t)unit); }
// Of a sequence; starts that do not grow can name more tiles than there are, and no sum over a batch may pass 64 bits
PAHQ_HD uint64_t kv_units(int tiles, int heads, int length, int unit) {
  const uint64_t pairs = (uint64_t)(uint32_t)tiles * (uint32_t)heads, most = 1ull << 47, each = (uint64_t)kv_units_of(length, unit);
  return pairs < most / each ? pairs * each : most;
}

struct KvPlan { uint64_t units; int wgs; };        // wgs 0: tiles are given out whole
PAHQ_HD KvPlan kv_plan(uint64_t units, int longest, int slots, int least) {
  if ((uint64_t)(uint32_t)longest * (uint32_t)slots <= units) return {units, 0};
  const uint64_t parts = units / (uint32_t)least;
  return {units, parts >= (uint64_t)slots ? slots : parts > 1 ? (int)parts : 1};
}
// Where range w begins: units * w / wgs, rounded down
PAHQ_HD uint64_t kv_from(uint64_t units, int wgs, int w) {
  const uint64_t each = units / (uint32_t)wgs, rest = units - each * (uint32_t)wgs;
  return each * (uint32_t)w + rest * (uint32_t)w / (uint32_t)wgs;
}
// Whose range a unit lies in: the last w that begins at or in front of it
PAHQ_HD int kv_holder(uint64_t units, int wgs, uint64_t unit) {
  const uint64_t w = ((unit + 1) * (uint32_t)wgs - 1) / units;
  return w < (uint64_t)wgs ? (int)w : wgs - 1;      // also where a batch that makes no sense has more units than that holds
}
// The range of a workgroup of the launch, -1 for none: neighbouring ranges, which share rows of the cache where tiles do, on one of the eight
// XCDs, to which workgroups go in turn
PAHQ_HD int kv_wg_of(unsigned block, int wgs) {
  const unsigned each = ((unsigned)wgs + 7) / 8, w = block % 8 * each + block / 8;
  return block / 8 < each && w < (unsigned)wgs ? (int)w : -1;
}

// For the worst case: every sequence that has tokens ends in a tile of its own
PAHQ_HD long long kv_most_tiles(int tokens, int batch, int group, int tile) {
  return (long long)tokens * group / tile + (batch < tokens ? batch : tokens);
}

}  // namespace pahq
