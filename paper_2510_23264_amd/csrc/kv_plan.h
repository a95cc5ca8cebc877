// How the attention over a paged cache is shared out to workgroups.  No GPU type in it, so that CPU tests compile it.
//
// The rows of a sequence and a cache head are (new token, query head of the group) pairs, in tiles of `rows`; a tile's work is its
// sequence's length, in units of some rows of the cache.  The host knows neither the lengths nor how the tokens are spread over the
// sequences, so each workgroup finds its part from the batch.  Where it does not pay to cut them (kv_cut_from) tiles
// are given out whole, as workgroups end.  Otherwise the units of all tiles, heads and sequences stand in one line, which is cut into
// equal ranges for at most `slots` workgroups, about as many as the chip holds at a time: one long sequence beside short ones, or
// one alone, takes the whole chip.  A range ends inside tiles at its ends only, so every workgroup leaves at most two parts
// of tiles in the workspace: in slot 2 w what it began inside of a tile, in slot 2 w + 1 what it left unfinished.  A tile's first `over`
// units stand for what it costs to begin one; a range that ends among them leaves the tile to the next.
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
PAHQ_HD int kv_units_of(int length, int unit, int over) { return over + (length <= unit ? 1 : (int)(((uint32_t)length + (uint32_t)unit - 1) / (uint32_t)unit)); }
// Of a sequence: tiles of all heads, and their units.  Sums over a batch stick at 2^32 - 1, with more units than that tiles are given out
// whole; starts that do not grow can name more tiles than there are, which is why a sequence's own are bounded.
PAHQ_HD uint32_t kv_pairs(int tiles, int heads) {
  const uint64_t pairs = (uint64_t)(uint32_t)tiles * (uint32_t)heads;
  return pairs < KV_MOST_ITEMS ? (uint32_t)pairs : (uint32_t)KV_MOST_ITEMS;
}
PAHQ_HD uint32_t kv_units(uint32_t pairs, int each) {
  const uint64_t units = (uint64_t)pairs * (uint32_t)each;
  return units < 0xFFFFFFFFull ? (uint32_t)units : 0xFFFFFFFFu;
}

// Tiles are cut if one has more units than this.  Given out whole, they take as long as the longest of them, or as the average range, or,
// where there are some more than can run at a time, until the last ones are done; cut, the average range and `brief` units more.
constexpr uint32_t KV_FEW_TILES = 256;              // one for each compute unit
PAHQ_HD uint32_t kv_cut_from(uint32_t units, uint32_t pairs, int slots, int enough, int brief) {
  return pairs > KV_FEW_TILES && pairs < (uint32_t)enough ? 0 : units / (uint32_t)slots + (uint32_t)brief;
}
// How many rows of the cache a tile sees at most, its sequence having n new tokens behind base others; (token, query head) pairs are fewer than
// KV_MAX_LENGTH, so that a tile more of them is counted in 32 bits
PAHQ_HD int kv_tile_end(int n, int base, int tile, int rows, int group) {
  const int last = (int)((((uint32_t)tile + 1) * (uint32_t)rows - 1) / (uint32_t)group), end = base + (last < n - 1 ? last : n - 1) + 1;
  return end > 0 ? end : 0;
}
// Of a causal sequence's T > 1 tiles the late ones see more, and a line of tiles that count the same would leave those who find early ones idle.  Tile T - 1 - i
// and tile i together see about as much for every i, so the line is made of such couples, whose units this bounds: their ends add up to at
// most 2 base + ((T + 1) rows - 2) / group + 2, and two quotients rounded up are at most two above the rounded-down quotient of their sum.  What is
// left of a couple's units, or of the middle tile's, is nobody's work.  A prompt of 4096 tokens in fp32, 12 heads of 64 columns: 260 us, 385 with tiles
// that count the same.
PAHQ_HD int kv_couple_units(int base, int tiles, int rows, int group, int unit, int over) {
  const uint32_t behind = base > 0 ? (uint32_t)base : 0, ends = (((uint32_t)tiles + 1) * (uint32_t)rows - 2) / (uint32_t)group + 2;
  return 2 * over + (int)(behind / (uint32_t)unit * 2 + (ends + behind % (uint32_t)unit * 2) / (uint32_t)unit) + 2;
}
struct KvPlan { uint32_t units, wgs; };            // wgs 0: tiles are given out whole
PAHQ_HD KvPlan kv_plan(uint32_t units, bool cut, int slots, int least) {
  if (!cut || units == 0xFFFFFFFFu) return {units, 0};
  const uint32_t parts = units / (uint32_t)least;
  return {units, parts >= (uint32_t)slots ? (uint32_t)slots : parts > 1 ? parts : 1u};
}
// Where range w begins: units * w / wgs, rounded down
PAHQ_HD uint32_t kv_from(const KvPlan& p, uint32_t w) { return (uint32_t)((uint64_t)p.units * w / p.wgs); }
// Whose range a unit lies in: the last w that begins at or in front of it
PAHQ_HD int kv_holder(const KvPlan& p, uint32_t unit) {
  const uint64_t w = (((uint64_t)unit + 1) * p.wgs - 1) / p.units;
  return w < p.wgs ? (int)w : (int)p.wgs - 1;
}
// The range of a workgroup of the launch, -1 for none: neighbouring ranges, which share rows of the cache where tiles do, on one of the eight
// XCDs, to which workgroups go in turn
PAHQ_HD int kv_wg_of(uint32_t block, uint32_t wgs) {
  const uint32_t each = (wgs + 7) / 8, w = block % 8 * each + block / 8;
  return block / 8 < each && w < wgs ? (int)w : -1;
}

// For the worst case: every sequence that has tokens ends in a tile of its own
PAHQ_HD long long kv_most_tiles(int tokens, int batch, int group, int tile) {
  return (long long)tokens * group / tile + (batch < tokens ? batch : tokens);
}

}  // namespace pahq
