// How the attention over a paged cache is shared out to workgroups.  No GPU type in it, so that CPU tests compile it.
//
// The rows of a sequence and a cache head are (new token, query head of the group) pairs, in tiles of `rows`; a tile's work is its
// sequence's length, in units of some rows of the cache.  The host knows neither the lengths nor how the tokens are spread over the
// sequences, so each workgroup finds its part from the batch.  Where it does not pay to cut them (kv_cut_from) tiles
// are given out whole, as workgroups end.  Otherwise the units of all tiles, heads and sequences stand in one line, which is cut into
// equal ranges for at most `slots` workgroups: one long sequence beside short ones, or one alone, takes the whole chip.  That is as many as the chip
// holds at a time, but for heads of more than 128 columns and, in tiles of 128 rows, of more than 64 in fp32: LDS or registers leave room for
// one workgroup on a compute unit there, and 512 ranges take two rounds.  A range ends inside tiles at its ends only, so every workgroup leaves at most two parts
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

// ---------------------------------------------------------------- a call
constexpr int KV_MAX_LENGTH = 0x7FFF0000;           // rows of a sequence: a tile behind the last one is still counted in 31 bits
PAHQ_HD int kv_least(int a, int b) { return a < b ? a : b; }
PAHQ_HD int kv_most(int a, int b) { return a > b ? a : b; }
// A sequence: its new tokens are rows t0 .. t0 + n - 1 of the operator's, its rows base .. base + n - 1 (base may be negative).  `starts` and `length` as the
// batch has them, whatever they are; `most`: rows a list of pages has room for.
struct KvSequence { int t0, n, length, base; };
PAHQ_HD int kv_clipped_start(int start, int tokens) { return kv_least(kv_most(start, 0), tokens); }
PAHQ_HD KvSequence kv_clipped(int start, int next, int length, int tokens, int most) {
  KvSequence s;
  s.t0 = kv_clipped_start(start, tokens);
  s.n = kv_most(kv_clipped_start(next, tokens) - s.t0, 0);
  s.length = kv_least(kv_most(length, 0), most);
  s.base = s.length - s.n;
  return s;
}
// What of a call decides how it is shared out
struct KvCall { bool causal; int heads, group, slots, over; };
// A sequence's part of the line: tiles a head, and units of a tile, or of a couple of them (0 where no line is made)
struct KvShare { int tiles, each; uint32_t pairs, units; };
PAHQ_HD bool kv_in_couples(const KvCall& c, int tiles) { return c.causal && tiles > 1; }
PAHQ_HD int kv_lines(const KvCall& c, int tiles) { return kv_in_couples(c, tiles) ? (tiles + 1) / 2 : tiles; }
PAHQ_HD KvShare kv_share(const KvCall& c, const KvSequence& s, int rows, int unit) {
  KvShare x = {};
  x.tiles = kv_tiles((long long)s.n * c.group, rows);
  x.pairs = kv_pairs(x.tiles, c.heads);
  if (c.slots) {
    const bool couples = kv_in_couples(c, x.tiles);
    x.each = couples ? kv_couple_units(s.base, x.tiles, rows, c.group, unit, c.over) : kv_units_of(s.length, unit, c.over);
    x.units = kv_units(couples ? kv_pairs(kv_lines(c, x.tiles), c.heads) : x.pairs, x.each);
  }
  return x;
}
PAHQ_HD int kv_end_of(const KvCall& c, const KvSequence& s, int tile, int rows) { return c.causal ? kv_tile_end(s.n, s.base, tile, rows, c.group) : s.length; }
// Of tiles that are given out whole the `local`-th of a sequence: heads in turn, and the last tiles, which see the most rows, first
struct KvTile { int h, tile; };
PAHQ_HD KvTile kv_whole_tile(const KvCall& c, int tiles, uint32_t local) {
  return {(int)(local % (uint32_t)c.heads), (int)((uint32_t)tiles - 1 - local / (uint32_t)c.heads)};
}
// What lies at unit `local` of a sequence's part of the line: from unit `off` of a tile's `whole` on, `take` of them up to `left` at most; no work
// where a couple's bound is more than its tiles have
struct KvStretch { int h, tile; uint32_t off, whole, take; bool work; };
PAHQ_HD KvStretch kv_stretch(const KvCall& c, const KvSequence& s, int tiles, uint32_t each, int rows, int unit, uint32_t local, uint32_t left) {
  const bool couples = kv_in_couples(c, tiles);
  const uint32_t lines = kv_lines(c, tiles), line = local / each, in = local - line * each;
  KvStretch x;
  x.h = line / lines;
  const int i = line - x.h * lines;
  x.tile = couples ? tiles - 1 - i : i;
  x.off = in;
  x.whole = kv_units_of(kv_end_of(c, s, x.tile, rows), unit, c.over);
  if (x.off >= x.whole && i != x.tile) {            // behind the late tile the early one
    x.off -= x.whole;
    x.tile = i;
    x.whole = kv_units_of(kv_end_of(c, s, i, rows), unit, c.over);
  }
  x.work = x.off < x.whole;
  const uint32_t rest = x.work ? x.whole - x.off : each - in;
  x.take = rest < left ? rest : left;
  return x;
}
// Of a stretch that reaches past what beginning a tile costs: whether the tile begins and ends in it, and the rows of the cache it takes of the
// tile's `end` where that is not so
PAHQ_HD bool kv_begins(const KvCall& c, const KvStretch& x) { return x.off <= (uint32_t)c.over; }
PAHQ_HD bool kv_ends(const KvStretch& x) { return x.off + x.take == x.whole; }
PAHQ_HD int kv_begin_of(const KvCall& c, const KvStretch& x, int unit, int end) {
  const uint64_t from = (uint64_t)(x.off - (uint32_t)c.over) * (uint32_t)unit;
  const uint32_t begin = from < KV_MAX_LENGTH ? (uint32_t)from : (uint32_t)KV_MAX_LENGTH;
  return begin < (uint32_t)end ? (int)begin : end;
}
PAHQ_HD int kv_stop_of(const KvCall& c, const KvStretch& x, int unit, int end) { return kv_least(end, (int)((x.off + x.take - (uint32_t)c.over) * (uint32_t)unit)); }

// How a call is cut.  What the host sees of it decides, as the size of the workspace does too.
struct KvCut {
  int rows;                                         // of a tile
  bool waves;                                       // of few rows: a workgroup has a compute unit to itself, and so many waves
  int slots;                                        // ranges at most, 0: tiles are given out whole in any case
  int least, over;                                  // units of a range at least, and what beginning a tile counts
  int enough, brief;                                // where that pays, see kv_cut_from
};
inline long long kv_call_tiles(int tokens, int batch, int group, int heads, int rows) { return kv_most_tiles(tokens, batch, group, rows) * heads; }
inline KvCut kv_cut(int tokens, int batch, int group, int heads, int most, int d, int eb) {
  KvCut k;
  // Rows a sequence and head.  Every tile reads its sequence's rows of the cache, so they decide: 8 sequences of 64 tokens, 4 heads of a
  // group, over up to 8000 rows take 44 us in tiles of 128 and 140 us in tiles of 16; 64 single tokens of 4 heads over up to 16384 rows
  // take 172 us in tiles of 16 and 198 us in tiles of 128, which then mostly hold nothing.
  const long long mean = (((long long)tokens + batch - 1) / kv_most(batch, 1)) * group;
  // heads of more than 128 columns in fp32 stay with 16: more rows of theirs do not fit the registers
  k.rows = mean <= 16 || (eb == 4 && d > 128) ? 16 : mean <= 32 ? 32 : 128;
  const long long tiles = kv_call_tiles(tokens, batch, group, heads, k.rows);
  // Few tiles: one workgroup of many waves on a compute unit has half the parts to join, and 4 us less of 94 to do for a token over 131072
  // rows.  Many short ones hide each other's beginnings in two workgroups (256 tokens over 1024 rows, 8 heads: 181 us instead of 198).
  k.waves = k.rows < 128 && tiles < 1024;
  k.slots = k.waves ? 256 : 512;
  k.least = 4;
  k.over = k.rows < 128 ? 2 : 5;
  // Equal tiles, some for each range, are cut for the last ones would leave workgroups idle: 40 tokens over 4096 rows, 8 heads, 109 us
  // instead of 138, 200 over 512 80 instead of 90, 200 over 2048 274 instead of 291; at eight for a range (500 over 1024) it would lose 2 %.
  // Prompts' do not: the first tiles see little, and are done while the last ones run.
  k.enough = k.rows < 128 ? 5 * k.slots : 0;
  // What cutting costs in units: the parts' way through memory and the join, 5 to 15 us.  One token of 4 heads over 500 rows takes 12.5 us
  // whole and 16.5 cut, over 1000 rows 19 and 17; 1500 tokens of a prompt 42 and 67; 128 behind 640 others 22 and 24, behind 1372 37 and 27.
  // In fp32, whose units take longer, 300 tokens of a prompt 28 and 32, 100 behind 300 others 66 and 36.
  k.brief = k.rows < 128 ? 8 : eb == 2 ? 18 : 12;
  // Not even the longest sequence that the lists of pages have room for would be cut, or the new tokens alone are so much work that a range is as
  // long as any sequence can be
  const int wide = eb * (d <= 64 ? 64 : d <= 128 ? 128 : 256), unit = k.rows < 128 ? 32768 / wide : wide <= 256 ? 64 : 32;
  const bool few = k.rows == 128 || tiles <= KV_FEW_TILES;
  const double work = (double)tokens * tokens * group / ((double)k.rows * kv_most(batch, 1)) * heads / k.slots;
  if (most <= 256 || (few && kv_units_of(most, unit, k.over) <= k.brief) || most <= work) {
    k.slots = 0;
    k.waves = k.rows < 128 && tiles <= KV_FEW_TILES;
  }
  return k;
}

}  // namespace pahq
