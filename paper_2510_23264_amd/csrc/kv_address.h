// Where the attention over a paged cache reads and writes: in the cache, in LDS, in its operands' rows and in the workspace.  Everything that
// becomes an address is here or in kv_plan.h, without a GPU type, so that a CPU test can follow every lane of every kernel and see that it stays
// inside of what there is, and that what a lane reads from LDS is what was brought there.
#pragma once
#include <stddef.h>
#include <stdint.h>
#include "kv_plan.h"

namespace pahq {

// ---------------------------------------------------------------- rows of a sequence in the cache
// ceil(2^(31 + s) / p), 2^s the power of two at or above p: fits 32 bits, and j * (its excess over the exact quotient) stays
// below 2^(31 + s) for every j < 2^31, so the shifted product is the quotient.
inline void kv_divider(uint32_t p, uint32_t* magic, int* shift) {
  int s = 0;
  while ((1ull << s) < p) s++;
  *magic = (uint32_t)(((1ull << (31 + s)) + p - 1) / p);
  *shift = 31 + s;
}
// The cache as kernels take it: strides in bytes
struct KvCache {
  char *keys, *values;
  long long page, head, slot;
  int pages, page_size, heads, d;
  uint32_t magic;                                   // j / page_size = j * magic >> shift for j < 2^31
  int shift;
};
PAHQ_HD int kv_in_list(const KvCache& c, int j) { return (int)((unsigned long long)(uint32_t)j * c.magic >> c.shift); }
// Bytes from the cache's start to row j of a sequence in head 0, `page` being what its list says for it; KV_ROW_NONE where that is no page
constexpr long long KV_ROW_BEHIND = -2, KV_ROW_NONE = -1;
PAHQ_HD bool kv_is_page(const KvCache& c, int page) { return (uint32_t)page < (uint32_t)c.pages; }
PAHQ_HD long long kv_row_of_page(const KvCache& c, int j, int page) {
  const int slot = j - kv_in_list(c, j) * c.page_size;
  return page * c.page + slot * c.slot;
}
PAHQ_HD long long kv_row_in(const KvCache& c, int j, int page) { return kv_is_page(c, page) ? kv_row_of_page(c, j, page) : KV_ROW_NONE; }
// Attention asks for the page of every row of a block, also of rows behind `end`: of the last row in front of it, or the first one
PAHQ_HD int kv_asked(const KvCache& c, int row, int end) { return kv_in_list(c, kv_most(kv_least(row, end - 1), 0)); }
PAHQ_HD long long kv_row_or_behind(const KvCache& c, int row, int end, int page) { return row >= end ? KV_ROW_BEHIND : kv_row_in(c, row, page); }

// ---------------------------------------------------------------- a block of rows in LDS
// Where chunk c (16 bytes) of a row lies among the row's CH chunks: c ^ swizzle.  Rows 4 apart in the low bits, so that four rows' 64 neighbouring
// bytes (what a transposing read takes) lie in different quarters of the 64 banks, and so do one chunk of sixteen rows (what K's reads take).
template <int CH> PAHQ_HD int kv_swizzle(int row) {
  static_assert(CH >= 8, "rows of 128 bytes and more");
  return CH >= 16 ? (row & 3) << 2 | (row >> 2 & 3) : (row >> 1 & 1) << 2 | (row >> 2 & 3);
}
// Rows r0 .. of a block, 64 / CH of them (r0 a multiple of that), come chunk by chunk, lane l's behind lane l - 1's: lane l's row behind r0 and its chunk
template <int CH> PAHQ_HD int kv_asks_row(int lane) { return lane / CH; }
template <int CH> PAHQ_HD int kv_asks_chunk(int lane, int r0) { return (lane % CH ^ kv_swizzle<CH>(lane / CH)) ^ kv_swizzle<CH>(r0); }

// A kernel for up to 16 RT rows of queries: EB bytes an element, D columns, NW waves.  LDS: [NW][2][STAGE], then [NW][4][64] pages' numbers;
// a stage is keys [HALF] and values [HALF].  Addresses in a stage are given as a lane's first one, from which the others differ in the
// chunk, which XOR changes in place (rows begin at multiples of their size), and in rows a constant apart.
template <int EB, int D, int RT, int NW> struct KvFew {
  static constexpr int CH = D * EB / 16, KT = EB == 2 ? 2 : 1, KVB = 16 * KT, ROWS = 16 * RT, ROW = D * EB;
  static constexpr int HALF = KVB * ROW, STAGE = 2 * HALF, ASKS = HALF / 1024, DT = D / 16;
  static constexpr int IDS = NW * 2 * STAGE, LDS = IDS + NW * 1024, UNIT = KVB * NW;
  // of a wave, and in it of its n-th block
  static PAHQ_HD int stages(int wave) { return wave * 2 * STAGE; }
  static PAHQ_HD int stage(int n) { return (n & 1) * STAGE; }
  static PAHQ_HD int ids(int wave) { return IDS + wave * 4 * 256; }
  static PAHQ_HD int ids_of(int n) { return (n & 3) * 256; }
  // the operand of a product of 16 rows from 16 t on: chunk h4 + 4 c of row l16
  static PAHQ_HD uint32_t key0(int l16, int h4) { return l16 * ROW + ((h4 ^ kv_swizzle<CH>(l16)) * 16); }
  static PAHQ_HD uint32_t key(uint32_t key0, int t, int c) { return (key0 ^ (4 * c * 16)) + 16 * t * ROW; }
  // of 16 columns from 16 d on, 16 bits: four of them of row 4 h4 + l16 / 4, which the read transposes; fp32: column l16 of row 4 h4 + i
  static PAHQ_HD uint32_t value0(int l16, int h4) {
    const int row = 4 * h4 + (EB == 2 ? l16 / 4 : 0);
    return EB == 2 ? HALF + row * ROW + (((l16 & 3) / 2 ^ kv_swizzle<CH>(row)) * 16) + (l16 & 1) * 8
                   : HALF + row * ROW + ((l16 / 4 ^ kv_swizzle<CH>(row)) * 16) + (l16 & 3) * 4;
  }
  static PAHQ_HD uint32_t value_16_bit(uint32_t value0, int t, int d) { return (value0 ^ (2 * d * 16)) + 16 * t * ROW; }
  static PAHQ_HD uint32_t value_fp32(uint32_t value0, int i, int d) { return (value0 ^ ((4 * d ^ kv_swizzle<CH>(i)) * 16)) + i * ROW; }
  // the wave's sums, [row][D] of fp32 in its stages: columns 4 c and on, swizzled by the row
  static PAHQ_HD int sum(int wave, int row, int c) { return stages(wave) + row * (D * 4) + ((c ^ (row & 15)) * 16); }
  static_assert(2 * STAGE >= ROWS * D * 4 && 2 * ASKS + 1 < 64, "the waves' sums fit their stages");
};
// The kernel for many rows: four waves of 32 rows share blocks of KVB rows.  LDS: [2] keys [HALF] and values [HALF], [NW][2][64] pages' numbers.
template <int EB, int D> struct KvWide {
  static constexpr int NW = 4, ROWS = 32 * NW, CH = D * EB / 16, KVB = D * EB <= 256 ? 64 : 32, KT = KVB / 32, N = 16 / EB, ROW = D * EB;
  static constexpr int HALF = KVB * ROW, MINE = KVB / NW, ASKS = HALF / 1024 / NW, DT = D / 32, STEPS = 16 / N;      // a step: 16 rows, or 8
  static constexpr int IDS = 4 * HALF, LDS = IDS + NW * 512, UNIT = KVB;
  // of the n-th block, in it the wave's share of MINE rows, and a wave's pages' numbers
  static PAHQ_HD int stage(int n) { return (n & 1) * 2 * HALF; }
  static PAHQ_HD int share(int wave) { return wave * ASKS * 1024; }
  static PAHQ_HD int ids(int wave) { return IDS + wave * 2 * 256; }
  static PAHQ_HD int ids_of(int n) { return (n & 1) * 256; }
  // the operand of a product of 32 rows from 32 t on: chunk h2 + 2 c of row l32
  static PAHQ_HD uint32_t key0(int l32, int h2) { return l32 * ROW + ((h2 ^ kv_swizzle<CH>(l32)) * 16); }
  static PAHQ_HD uint32_t key(uint32_t key0, int t, int c) { return (key0 ^ (2 * c * 16)) + 32 * t * ROW; }
  // of 32 columns from 32 d on and the 2 N rows from `row` on, 16 bits: four columns of row 4 h2 + (lane & 15) / 4 + 8 j; fp32: column l32 of row 4 h2 + j
  static PAHQ_HD uint32_t value0(int lane) {
    const int l32 = lane & 31, row = 4 * (lane >> 5) + (EB == 2 ? (lane & 15) / 4 : 0);
    return HALF + row * ROW +
           (EB == 2 ? ((2 * (lane >> 4 & 1) + (lane & 3) / 2 ^ kv_swizzle<CH>(row)) * 16) + (lane & 1) * 8 : ((l32 / 4 ^ kv_swizzle<CH>(row)) * 16) + (l32 & 3) * 4);
  }
  static PAHQ_HD uint32_t value_16_bit(uint32_t value0, int row, int j, int d) { return (value0 ^ ((4 * d ^ kv_swizzle<CH>(8 * j)) * 16)) + (row + 8 * j) * ROW; }
  static PAHQ_HD uint32_t value_fp32(uint32_t value0, int row, int j, int d) { return (value0 ^ ((8 * d ^ kv_swizzle<CH>(row % 32 + j)) * 16)) + (row + j) * ROW; }
  // Rows in one page, as those of a wave are where pages hold whole shares of a block: their place is the wave's, a lane's chunk an offset of 32 bits
  static bool PAHQ_HD simple(const KvCache& c) { return c.page_size % MINE == 0 && c.d == D && c.slot < 1 << 24; }
  static PAHQ_HD bool simple_block(int k0, int end) { return k0 + KVB <= end; }
  static PAHQ_HD uint32_t simple_offset(int lane, int r0, uint32_t slot) { return (uint32_t)kv_asks_chunk<CH>(lane, r0) * 16 + (uint32_t)kv_asks_row<CH>(lane) * slot; }
  static_assert(ASKS >= 1 && MINE * CH == ASKS * 64 && KVB <= 64, "a wave asks for whole rows");
};
// Waves of the kernels for few rows: as many as hold 64 KB of stages, or 128 KB where a workgroup has a compute unit to itself
template <int EB, int D> struct KvWaves {
  static constexpr int STAGES = 4 * (EB == 2 ? 32 : 16) * D * EB;       // a wave's
  static constexpr int NW = 65536 / STAGES > 2 ? 65536 / STAGES : 2, MANY = 131072 / STAGES > NW ? 131072 / STAGES : NW;
};

// ---------------------------------------------------------------- rows of queries and results, parts
// Row `row` of a sequence and cache head: (new token, query head of the group)
struct KvQuery { int token, g; };
PAHQ_HD int kv_token(long long row, int group) { return (int)(row / group); }
PAHQ_HD KvQuery kv_query(long long row, int token, int group) { return {token, (int)(row - (long long)token * group)}; }
// Where it is among rows of a tile's operand, strides in bytes
PAHQ_HD long long kv_query_at(int t0, const KvQuery& q, int h, int group, long long token, long long head) { return (t0 + q.token) * token + (h * group + q.g) * head; }
// Bit x: whether new token i sees row k0 + x of the cache; none for i < 0.  `tree` [tokens][words] or NULL.  Without branches, so that lanes do not
// part here: registers that hold what is every lane's are to stay out of code in which some lanes are off.
PAHQ_HD unsigned long long kv_low_bits(int n) { return n >= 64 ? ~0ull : (1ull << kv_most(n, 0)) - 1; }
PAHQ_HD unsigned long long kv_seen(const unsigned long long* tree, int words, const KvSequence& s, int i, int k0, int end) {
  const unsigned long long here = kv_low_bits(end - k0) & (i < 0 ? 0ull : ~0ull);
  if (!tree) return kv_low_bits(s.base + i + 1 - k0) & here;
  const int ahead = k0 - s.base, word = ahead >> 6, shift = ahead & 63;            // rounded down
  const unsigned long long* const w = tree + (long long)(s.t0 + kv_most(i, 0)) * words;
  const unsigned long long first = w[kv_least(kv_most(word, 0), words - 1)], second = w[kv_least(kv_most(word + 1, 0), words - 1)];
  const unsigned long long of_first = word >= 0 && word < words ? ~0ull : 0ull, of_second = shift && word + 1 >= 0 && word + 1 < words ? ~0ull : 0ull;
  return (kv_low_bits(s.base - k0) | (first >> shift & of_first) | (second << (64 - shift & 63) & of_second)) & here;
}
// The workspace: [2 slots][rows][d] sums of a part, [2 slots][rows][2] maximum and sum, how many of KvLeft there are (32 bytes), and they
struct KvLeft { int t0, rows, tile, h, pieces, w0, unused[2]; };        // pieces 0: of a tile that does not lie in several ranges, of which `w0` is the first
PAHQ_HD long long kv_part_at(int slot, int rows, int row, int d) { return ((long long)slot * rows + row) * d; }                          // in floats
PAHQ_HD long long kv_stat_at(int slots, int slot, int rows, int row, int d) { return 2ll * slots * rows * d + ((long long)slot * rows + row) * 2; }
PAHQ_HD long long kv_count_at(int slots, int rows, int d) { return 2ll * slots * rows * (d + 2); }
PAHQ_HD long long kv_left_at(int slots, int rows, int d) { return kv_count_at(slots, rows, d) + 8; }
inline size_t kv_part_bytes(int slots, int rows, int d) { return slots ? (size_t)kv_left_at(slots, rows, d) * 4 + (size_t)slots * sizeof(KvLeft) : 0; }
// Which slot a stretch of a tile that is not whole goes to, and in which slots a tile's parts lie
PAHQ_HD int kv_slot(int wg, bool starts) { return 2 * wg + starts; }
PAHQ_HD int kv_slot_of(int w0, int part) { return 2 * (w0 + part) + (part == 0); }
// The row of KvLeft of a tile: its number among all, or the range it begins in
PAHQ_HD uint32_t kv_number(uint32_t pairs_before, int h, int tiles, int tile) { return pairs_before + h * tiles + tile; }

// ---------------------------------------------------------------- the join's launch
struct KvJoin { int left, per, few; };
// As many rows of a workgroup that its launch, a workgroup in 3 to 4 ns, does not take longer than what they do
inline KvJoin kv_join(long long tiles, int slots, int rows, int d) {
  KvJoin j = {(int)(tiles < slots ? tiles : slots), 1, 1};
  while (j.per < rows && j.left * (rows / j.per) > 2048) j.per *= 2;
  while (j.few * 2 <= (j.per < 8 ? j.per : 8) && j.few * 2 * (d / 4) <= 256) j.few *= 2;
  return j;
}

}  // namespace pahq
