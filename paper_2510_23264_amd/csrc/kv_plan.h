// How the attention over a paged cache is cut into workgroups.  No GPU type in it, so that CPU tests compile it.
//
// The rows of a sequence and a cache head are (new token, query head of the group) pairs, in tiles of `rows`; a tile's work is the
// sequence's length.  The host knows neither the lengths nor how the tokens are spread over the sequences, so a launch counts workgroups for
// the worst case and each finds its part from the batch: tiles are cut along the sequence into pieces of `piece` rows of the cache, one size
// for the whole batch, chosen so that all of them together are about the `slots` workgroups that the chip holds at a time.  So one long
// sequence beside short ones, or one alone, takes the whole chip, and a batch whose tiles fill it already is not cut.
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
PAHQ_HD int kv_pieces(int length, int piece) { return length <= piece ? 1 : (int)(((uint32_t)length + (uint32_t)piece - 1) / (uint32_t)piece); }

// The first guess: the work (rows of the cache over all tiles and heads) over the slots, in whole units, at least `least`.  A tile longer than a
// piece has fewer than 2 * length / piece of them, so those of all cut tiles and heads are fewer than 2 * slots, whatever the
// batch holds: work that a double does not hold exactly makes a piece as long as any sequence.
PAHQ_HD int kv_first_piece(double work, int slots, int unit, int least) {
  const double even = work / slots;
  if (!(even < 2e9)) return 0x7FFF0000;
  uint64_t p = (uint64_t)even + 1;
  if (p < (uint64_t)least) p = (uint64_t)least;
  p = (p + unit - 1) / unit * unit;
  return p >= 0x7FFF0000u ? 0x7FFF0000 : (int)p;
}
// The next guess, where the pieces of a batch of few tiles are more than the slots: an eighth longer
PAHQ_HD int kv_longer_piece(int piece, int unit) {
  const uint64_t p = (uint64_t)piece + (uint64_t)(piece / 8 > unit ? piece / 8 : unit) + unit - 1;
  return p >= 0x7FFF0000u ? 0x7FFF0000 : (int)(p / unit * unit);
}
constexpr int KV_GUESSES = 8;                       // after which a batch of tiles below half the slots fits twice over

// For the worst case: every sequence that has tokens ends in a tile of its own; pieces are fewer than the slots' share and one a tile
PAHQ_HD long long kv_most_tiles(int tokens, int batch, int group, int tile) {
  return (long long)tokens * group / tile + (batch < tokens ? batch : tokens);
}
PAHQ_HD long long kv_most_items(long long tiles, int heads, int slots) { return tiles + slots / heads + 1; }

}  // namespace pahq
