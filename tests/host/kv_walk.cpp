// csrc/kv_address.h and kv_plan.h followed as the attention's kernels follow them, every lane of them, on the CPU.
//   quotient   a line is a page size: j / p by product and shift against the division
//   seen       lines "words base n k0 end seed": the bits of every new token against their definition
//   stages     for every kernel that is built: what a block's requests put into LDS is what the products' reads find there
//   walk       a line is a call: who does what of it, and that every address lies inside of what it is an address of
// An answer a line; one that begins with a letter says what is wrong.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <string>
#include <vector>
#include "kv_address.h"
using namespace pahq;

struct Wrong { std::string what; };
static void need(bool ok, const char* what, long long a = 0, long long b = 0, long long c = 0) {
  if (!ok) throw Wrong{std::string(what) + " " + std::to_string(a) + " " + std::to_string(b) + " " + std::to_string(c)};
}
static uint64_t state;
static uint32_t rnd(uint32_t below) {
  state = state * 6364136223846793005ull + 1442695040888963407ull;
  return (uint32_t)((state >> 33) % below);
}

// ---------------------------------------------------------------- quotient, seen
static void quotient(uint32_t p) {
  KvCache c = {};
  c.page_size = (int)p;
  kv_divider(p, &c.magic, &c.shift);
  const uint32_t top = 0x7FFFFFFF;
  auto at = [&](uint64_t j) { if (j <= top) need(kv_in_list(c, (int)j) == (int)(j / p), "quotient", p, j); };
  for (const uint64_t j : {(uint64_t)0, (uint64_t)1, (uint64_t)p - 1, (uint64_t)p, (uint64_t)top, (uint64_t)top / p * p, (uint64_t)top / p * p - (top >= p)}) at(j);
  for (int i = 0; i < 100; i++) {
    at(rnd(top));
    const uint64_t m = (uint64_t)rnd(top / p + 1) * p;
    at(m);
    if (m) at(m - 1);
  }
}
static void seen(int words, int base, int n, int k0, int end) {
  std::vector<unsigned long long> tree((size_t)(n + 3) * words);
  for (auto& w : tree) w = (uint64_t)rnd(1u << 31) << 33 ^ (uint64_t)rnd(1u << 31) << 10 ^ rnd(1u << 31);
  const KvSequence s = {3, n, base + n, base};
  for (int i = -1; i < n; i++)
    for (int masked = 0; masked < 2; masked++) {
      const unsigned long long got = kv_seen(masked ? tree.data() : nullptr, masked ? words : 0, s, i, k0, end);
      for (int x = 0; x < 64; x++) {
        const int j = k0 + x, ahead = j - base;
        bool want = i >= 0 && j < end;
        if (want && ahead >= 0) want = masked ? ahead / 64 < words && tree[(size_t)(3 + i) * words + ahead / 64] >> (ahead % 64) & 1 : ahead <= i;
        need((got >> x & 1) == want, "seen", i, x, masked);
      }
    }
}

// ---------------------------------------------------------------- stages
struct Held { int row, chunk; bool value; };                    // what lies in 16 bytes of a stage
template <int EB, int D, int RT, int NW> void few_stages() {
  typedef KvFew<EB, D, RT, NW> L;
  for (int wave = 0; wave < NW; wave++)
    for (int n = 0; n < 2; n++) {
      const int stage = L::stages(wave) + L::stage(n);
      std::map<int, Held> lds;
      for (int j = 0; j < L::ASKS; j++)
        for (int lane = 0; lane < 64; lane++)
          for (int v = 0; v < 2; v++) {
            const int r0 = j * (64 / L::CH), at = stage + v * L::HALF + j * 1024 + lane * 16, chunk = kv_asks_chunk<L::CH>(lane, r0);
            need(at >= stage && at + 16 <= stage + L::STAGE && at + 16 <= L::IDS && !lds.count(at) && chunk >= 0 && chunk < L::CH, "few: asked", wave, j, lane);
            need(r0 + kv_asks_row<L::CH>(lane) < L::KVB, "few: row", j, lane);
            lds[at] = {r0 + kv_asks_row<L::CH>(lane), chunk, v == 1};
          }
      need((int)lds.size() == L::STAGE / 16, "few: a stage is filled");
      auto find = [&](uint32_t at, int row, int byte, int bytes, bool value, const char* what) {
        const auto h = lds.find((int)(at & ~15u));
        need(at % bytes == 0 && h != lds.end() && h->second.row == row && h->second.value == value && h->second.chunk * 16 + (int)(at & 15) == byte, what, at, row, byte);
      };
      for (int lane = 0; lane < 64; lane++) {
        const int l16 = lane & 15, h4 = lane >> 4;
        const uint32_t ks = stage + L::key0(l16, h4), vs = stage + L::value0(l16, h4);
        for (int t = 0; t < L::KT; t++)
          for (int c = 0; c < L::CH / 4; c++) find(L::key(ks, t, c), 16 * t + l16, (h4 + 4 * c) * 16, 16, false, "few: key");
        for (int d = 0; d < L::DT; d++)
          if (EB == 2) for (int t = 0; t < 2; t++) find(L::value_16_bit(vs, t, d), 16 * t + 4 * h4 + l16 / 4, 2 * (16 * d + 4 * (l16 % 4)), 8, true, "few: value");
          else for (int i = 0; i < 4; i++) find(L::value_fp32(vs, i, d), 4 * h4 + i, 4 * (16 * d + l16), 4, true, "few: value");
      }
      need(L::ids(wave) >= L::IDS && L::ids(wave) + L::ids_of(3) + 256 <= L::LDS, "few: ids", wave);
    }
  for (int wave = 0; wave < NW; wave++) {
    std::map<int, int> sums;
    for (int row = 0; row < L::ROWS; row++)
      for (int c = 0; c < D / 4; c++) {
        const int at = L::sum(wave, row, c);
        need(at >= L::stages(wave) && at + 16 <= L::stages(wave) + 2 * L::STAGE && at % 16 == 0 && !sums.count(at), "few: sums", wave, row, c);
        sums[at] = 1;
      }
  }
  need(L::LDS + NW * L::ROWS * 8 + NW * 4 + 1024 <= 160 * 1024, "few: LDS of a compute unit", L::LDS);
}
template <int EB, int D> void wide_stages() {
  typedef KvWide<EB, D> L;
  for (int n = 0; n < 2; n++) {
    std::map<int, Held> lds;
    for (int wave = 0; wave < L::NW; wave++)
      for (int j = 0; j < L::ASKS; j++)
        for (int lane = 0; lane < 64; lane++)
          for (int v = 0; v < 2; v++) {
            const int first = j * (64 / L::CH), r0 = wave * L::MINE + first, at = L::stage(n) + L::share(wave) + v * L::HALF + j * 1024 + lane * 16;
            const int chunk = kv_asks_chunk<L::CH>(lane, r0);
            need(at >= L::stage(n) && at + 16 <= L::stage(n) + 2 * L::HALF && at + 16 <= L::IDS && !lds.count(at) && chunk >= 0 && chunk < L::CH, "wide: asked", wave, j, lane);
            need(first + kv_asks_row<L::CH>(lane) < L::MINE, "wide: row", j, lane);
            lds[at] = {r0 + kv_asks_row<L::CH>(lane), chunk, v == 1};
            // by offset from the place of the wave's first row of 64 / CH
            need(L::simple_offset(lane, r0, 4096) == (uint32_t)(chunk * 16 + kv_asks_row<L::CH>(lane) * 4096), "wide: offset", lane);
          }
    need((int)lds.size() == 2 * L::HALF / 16, "wide: a stage is filled");
    auto find = [&](uint32_t at, int row, int byte, int bytes, bool value, const char* what) {
      const auto h = lds.find((int)(at & ~15u));
      need(at % bytes == 0 && h != lds.end() && h->second.row == row && h->second.value == value && h->second.chunk * 16 + (int)(at & 15) == byte, what, at, row, byte);
    };
    for (int lane = 0; lane < 64; lane++) {
      const int l32 = lane & 31, h2 = lane >> 5;
      const uint32_t ks = L::stage(n) + L::key0(l32, h2), vs = L::stage(n) + L::value0(lane);
      for (int t = 0; t < L::KT; t++)
        for (int c = 0; c < L::CH / 2; c++) find(L::key(ks, t, c), 32 * t + l32, (h2 + 2 * c) * 16, 16, false, "wide: key");
      for (int i = 0; i < L::KT * L::STEPS * L::DT; i++) {
        const int d = i % L::DT, row = i / L::DT * 2 * L::N;
        if (EB == 2) for (int j = 0; j < 2; j++) find(L::value_16_bit(vs, row, j, d), row + 8 * j + 4 * h2 + (lane & 15) / 4, 2 * (32 * d + 16 * (lane >> 4 & 1) + 4 * (lane & 3)), 8, true, "wide: value");
        else for (int j = 0; j < 4; j++) find(L::value_fp32(vs, row, j, d), row + j + 4 * h2, 4 * (32 * d + l32), 4, true, "wide: value");
      }
    }
  }
  for (int wave = 0; wave < L::NW; wave++) need(L::ids(wave) >= L::IDS && L::ids(wave) + L::ids_of(1) + 256 <= L::LDS, "wide: ids", wave);
  need(L::LDS + 1024 <= 160 * 1024, "wide: LDS of a compute unit", L::LDS);
}
template <int EB, int D> void stages_of() {
  few_stages<EB, D, 1, KvWaves<EB, D>::NW>();
  few_stages<EB, D, 1, KvWaves<EB, D>::MANY>();
  if constexpr (D * EB <= 512) {
    few_stages<EB, D, 2, KvWaves<EB, D>::NW>();
    few_stages<EB, D, 2, KvWaves<EB, D>::MANY>();
    wide_stages<EB, D>();
  }
}

// ---------------------------------------------------------------- walk
struct Call {
  int eb, causal, words, tokens, batch, heads, group, d, page_size, pages, width, layout, sane;
  std::vector<int> starts, lengths, table;
  KvCache c;
  long long extent, token, head;                                // of the cache; strides of queries and results
  int most;
};
struct Item { KvSequence s; int b, tile, h, begin, end, slot; };
struct Cover { int begin, end, slot; };

struct Walk {
  const Call& q;
  KvCut cut;
  KvCall call;
  int unit;
  bool by_pair;
  KvPlan plan;
  uint32_t pairs = 0, units = 0, longest = 0;
  std::vector<KvSequence> s;
  std::vector<KvShare> share;
  std::vector<uint32_t> pairs_to, units_to;
  std::vector<KvLeft> left;
  int count = -1;
  std::map<std::vector<int>, std::vector<Cover>> tiles;          // (sequence, head, tile)
  std::map<int, std::vector<int>> slots;                         // slot -> whose part
  long long items = 0;

  static uint32_t sum(uint32_t a, uint32_t b) { const uint64_t x = (uint64_t)a + b; return x > 0xFFFFFFFFull ? 0xFFFFFFFFu : (uint32_t)x; }
  Walk(const Call& c, const KvCut& k, int u) : q(c), cut(k), unit(u) {
    call = {q.causal != 0, q.heads, q.group, cut.slots, cut.over};
    by_pair = kv_call_tiles(q.tokens, q.batch, q.group, q.heads, cut.rows) <= cut.slots;
    for (int b = 0; b < q.batch; b++) {
      s.push_back(kv_clipped(q.starts[b], q.starts[b + 1], q.lengths[b], q.tokens, q.most));
      share.push_back(kv_share(call, s[b], cut.rows, unit));
      pairs = sum(pairs, share[b].pairs);
      units = sum(units, share[b].units);
      pairs_to.push_back(pairs);
      units_to.push_back(units);
      if (share[b].tiles) longest = std::max(longest, (uint32_t)kv_units_of(s[b].length, unit, cut.over));
    }
    plan = kv_plan(units, cut.slots && longest > kv_cut_from(units, pairs, cut.slots, cut.enough, cut.brief), cut.slots, cut.least);
    // whatever the memory held
    left.assign(cut.slots, KvLeft{(int)0x80000000, 0x7FFFFFFF, -1, -1, 0x7FFFFFFF, -1, {}});
  }
  // Finder::next
  uint32_t next(int wg, uint32_t at, uint32_t stop, Item* it) {
    const uint32_t begun = at;
    KvStretch x;
    int l;
    for (;;) {
      const std::vector<uint32_t>& to = plan.wgs ? units_to : pairs_to;
      for (l = 0; l < q.batch && !(at < to[l]); l++) {}
      if (l == q.batch) return 0;
      *it = {s[l], l, 0, 0, 0, 0, -1};
      if (!plan.wgs) {
        const KvTile t = kv_whole_tile(call, share[l].tiles, at - (pairs_to[l] - share[l].pairs));
        it->h = t.h;
        it->tile = t.tile;
        it->end = kv_end_of(call, it->s, it->tile, cut.rows);
        return 1;
      }
      x = kv_stretch(call, it->s, share[l].tiles, share[l].each, cut.rows, unit, at - (units_to[l] - share[l].units), stop - at);
      need(x.take > 0 && at + x.take <= stop, "a stretch goes on", at, x.take, stop);
      it->h = x.h;
      it->tile = x.tile;
      at += x.take;
      if (x.work && x.off + x.take > (uint32_t)cut.over) break;
      if (at >= stop) return 0;
    }
    it->end = kv_end_of(call, it->s, it->tile, cut.rows);
    const bool starts = kv_begins(call, x), ends = kv_ends(x);
    if (!starts) it->begin = kv_begin_of(call, x, unit, it->end);
    if (!ends) it->end = kv_stop_of(call, x, unit, it->end);
    if (!starts || !ends) it->slot = kv_slot(wg, starts);
    if (starts && (!ends || by_pair)) {
      const uint32_t number = kv_number(pairs_to[l] - share[l].pairs, it->h, share[l].tiles, it->tile);
      if (!by_pair || number < (uint32_t)cut.slots) {
        const uint32_t at_left = by_pair ? number : (uint32_t)wg;
        need(at_left < left.size(), "a place among what is left", at_left, cut.slots);
        left[at_left] = {it->s.t0, (int)std::min((long long)it->s.n * q.group - (long long)it->tile * cut.rows, (long long)cut.rows), it->tile, it->h,
                         ends ? 0 : kv_holder(plan, at - x.take - x.off + x.whole - 1) - wg + 1, wg, {}};
      }
    }
    return at - begun;
  }
  // rows of queries and results, and parts
  void rows_of(const Item& it) {
    need(it.h >= 0 && it.h < q.heads && it.tile >= 0 && it.tile < share[it.b].tiles && it.s.n > 0, "a tile", it.h, it.tile);
    const long long out = (q.tokens - 1) * q.token + ((long long)q.heads * q.group - 1) * q.head + (long long)q.d * q.eb;
    for (int r = 0; r < cut.rows; r++) {
      const long long row = (long long)it.tile * cut.rows + r;
      const bool there = row < (long long)it.s.n * q.group;
      const int token = there ? kv_token(row, q.group) : -1;
      const long long at = kv_query_at(it.s.t0, there ? kv_query(row, token, q.group) : KvQuery{0, 0}, it.h, q.group, q.token, q.head);
      need(at >= 0 && at + (long long)q.d * q.eb <= out, "a row of queries", it.tile, r, at);
      if (there) need(kv_query(row, token, q.group).g < q.group && token < it.s.n, "a query", row);
      if (it.slot >= 0) {
        need(it.slot < 2 * cut.slots, "a slot", it.slot);
        const long long part = kv_part_at(it.slot, cut.rows, r, q.d), st = kv_stat_at(cut.slots, it.slot, cut.rows, r, q.d);
        need(part >= 0 && part % 4 == 0 && part + q.d <= 2ll * cut.slots * cut.rows * q.d, "a part", part);
        need(st >= 2ll * cut.slots * cut.rows * q.d && st + 2 <= kv_count_at(cut.slots, cut.rows, q.d), "a part's sum", st);
      }
    }
    if (cut.slots) need((size_t)(kv_left_at(cut.slots, cut.rows, q.d) * 4 + cut.slots * (long long)sizeof(KvLeft)) <= kv_part_bytes(cut.slots, cut.rows, q.d) && kv_left_at(cut.slots, cut.rows, q.d) % 8 == 0, "the workspace");
  }
  // a chunk of a row: list, page, place
  int page_asked(const Item& it, int row, int end) {
    const int i = kv_asked(q.c, row, end);
    need(i >= 0 && i < q.width, "an entry of the list", i, row, end);
    if (row < end) need(i == row / q.page_size, "the row's entry", i, row);
    return q.table[(size_t)it.b * q.width + i];
  }
  void chunk(const Item& it, int row, int end, int page, int chunk_of_row) {
    const long long at = kv_row_or_behind(q.c, row, end, page);
    if (at == KV_ROW_BEHIND) { need(row >= end, "behind", row); return; }
    if (at == KV_ROW_NONE) { need(page < 0 || page >= q.pages, "no page", page); return; }
    if (chunk_of_row * 16 >= q.d * q.eb) return;                 // zeros
    const long long from = it.h * q.c.head + at + chunk_of_row * 16;
    need(from >= 0 && from + 16 <= q.extent, "a chunk of the cache", row, page, from);
    need(at == page * q.c.page + (row % q.page_size) * q.c.slot, "a row's place", row, page, at);
  }
  template <typename F> void blocks_of(int blocks, F f) {        // the first and the last ones, some between
    for (int n = 0; n < blocks && n < 2; n++) f(n);
    for (int i = 0; i < 4 && blocks > 4; i++) f(2 + (int)rnd(blocks - 4));
    for (int n = std::max(2, blocks - 2); n < blocks; n++) f(n);
  }
  template <typename L, int NW> void few(const Item& it) {
    const int begin = it.begin, end = it.end, blocks = end > begin ? (end - begin + L::KVB - 1) / L::KVB : 0;
    for (int wave = 0; wave < NW; wave++) {
      const int turns = blocks > wave ? (blocks - wave + NW - 1) / NW : 0;
      auto first_row = [&](int n) { return begin + (wave + n * NW) * L::KVB; };
      if (turns) for (int n = turns; n < turns + 3; n++) for (int lane = 0; lane < L::KVB; lane++) {      // asked for even behind the last block
        const long long row = (long long)begin + ((long long)wave + (long long)n * NW) * L::KVB + lane;
        need(row < 0x7FFFFFFF, "rows in 31 bits", row);
        page_asked(it, (int)row, end);
      }
      blocks_of(turns, [&](int n) {
        for (int j = 0; j < L::ASKS; j++)
          for (int lane = 0; lane < 64; lane++) {
            const int first = j * (64 / L::CH), holder = first + kv_asks_row<L::CH>(lane);
            need(holder < 64, "a lane that holds the row", holder);
            const int row = first_row(n) + (holder & (L::KVB - 1));
            chunk(it, row, end, page_asked(it, row, end), kv_asks_chunk<L::CH>(lane, first));
          }
      });
    }
  }
  template <typename L> void wide(const Item& it) {
    const int begin = it.begin, end = it.end, blocks = end > begin ? (end - begin + L::KVB - 1) / L::KVB : 0;
    const bool simple = L::simple(q.c);
    for (int wave = 0; wave < L::NW; wave++) {
      auto row_of = [&](int n) { return begin + n * L::KVB + wave * L::MINE; };
      if (blocks) for (int lane = 0; lane < 64; lane++) page_asked(it, row_of(blocks) + (lane & (L::MINE - 1)), end);
      blocks_of(blocks, [&](int n) {
        const bool whole = simple && L::simple_block(begin + n * L::KVB, end);
        const int page = page_asked(it, row_of(n), end);
        for (int j = 0; j < L::ASKS; j++)
          for (int lane = 0; lane < 64; lane++) {
            const int first = j * (64 / L::CH), r0 = wave * L::MINE + first, row = row_of(n) + first + kv_asks_row<L::CH>(lane);
            if (whole && kv_is_page(q.c, page)) {
              const long long at = kv_row_of_page(q.c, row_of(n), page) + first * q.c.slot + L::simple_offset(lane, r0, (uint32_t)q.c.slot);
              need(row < end && page_asked(it, row, end) == page && row / q.page_size == row_of(n) / q.page_size, "rows of one page", row, page);
              need(at == kv_row_or_behind(q.c, row, end, page) + kv_asks_chunk<L::CH>(lane, r0) * 16, "a chunk by offset", row, lane, at);
              need(it.h * q.c.head + at >= 0 && it.h * q.c.head + at + 16 <= q.extent, "a chunk of the cache", row, page, at);
            } else {
              chunk(it, row, end, page_asked(it, row, end), kv_asks_chunk<L::CH>(lane, r0));
            }
          }
      });
    }
  }
  template <typename F> void run(F kernel) {
    const long long given = kv_call_tiles(q.tokens, q.batch, q.group, q.heads, cut.rows);
    const unsigned grid = (unsigned)std::max<long long>(given, cut.slots);
    if (q.sane) need(pairs <= given, "tiles beyond the launch", pairs, given);
    for (unsigned block = 0; block < grid; block++) {
      const int wg = plan.wgs ? kv_wg_of(block, plan.wgs) : 0;
      if (wg < 0) continue;
      if (cut.slots) {
        if (plan.wgs && !by_pair) { need((uint32_t)wg < left.size(), "a range's place", wg); left[wg].pieces = 0; }
        if (plan.wgs ? wg == 0 : block == 0) count = plan.wgs ? (int)(by_pair ? std::min(pairs, (uint32_t)cut.slots) : plan.wgs) : 0;
      }
      uint32_t at = plan.wgs ? kv_from(plan, wg) : block;
      const uint32_t stop = plan.wgs ? kv_from(plan, wg + 1) : at + 1;
      while (at < stop) {
        Item it;
        const uint32_t take = next(wg, at, stop, &it);
        if (!take) break;
        at += take;
        items++;
        const int whole_end = kv_end_of(call, it.s, it.tile, cut.rows);
        need(it.begin >= 0 && it.begin <= it.end && it.end <= whole_end && whole_end <= q.most && it.begin % unit == 0 || it.begin == it.end, "rows of a tile", it.begin, it.end, whole_end);
        tiles[{it.b, it.h, it.tile}].push_back({it.begin, it.end, it.slot});
        if (it.slot >= 0) {
          need(!slots.count(it.slot), "a slot used twice", it.slot);
          slots[it.slot] = {it.b, it.h, it.tile};
        }
        if (items <= 40 || rnd(8) == 0) rows_of(it), kernel(it);
      }
    }
    joins(given);
    if (q.sane) covered();
  }
  // every row of every tile once
  void covered() {
    size_t all = 0;
    for (int b = 0; b < q.batch; b++) all += (size_t)share[b].tiles * q.heads;
    need(all == tiles.size(), "every tile is somebody's", all, tiles.size());
    for (auto& t : tiles) {
      const int end = kv_end_of(call, s[t.first[0]], t.first[2], cut.rows);
      std::sort(t.second.begin(), t.second.end(), [](const Cover& a, const Cover& b) { return a.begin != b.begin ? a.begin < b.begin : a.end < b.end; });
      int at = 0;
      for (const Cover& c : t.second) {
        need(c.begin == at, "rows of a tile once", t.first[2], c.begin, at);
        at = c.end;
        need((c.slot < 0) == (t.second.size() == 1), "a tile's part in the workspace", t.first[2], c.slot);
      }
      need(at == end, "a tile's end", t.first[2], at, end);
    }
  }
  // what the join reads was written, by the tile's parts in order, and every cut tile is joined once
  void joins(long long given) {
    if (!cut.slots) return;
    const KvJoin j = kv_join(given, cut.slots, cut.rows, q.d);
    need(count >= 0 && count <= cut.slots && j.left <= cut.slots && j.few * (q.d / 4) <= 256 && 256 / (j.few * (q.d / 4)) >= 1 && cut.rows % j.per == 0, "the join's launch", count, j.left, j.per);
    std::map<std::vector<int>, int> joined;
    for (int i = 0; i < j.left && i < count; i++) {
      const KvLeft& t = left[i];
      if (t.pieces <= 1) continue;
      if (!q.sane && t.w0 < 0) need(false, "an entry that nobody wrote", i);
      need(t.w0 >= 0 && t.rows > 0 && t.rows <= cut.rows && t.h >= 0 && t.h < q.heads, "an entry", i, t.w0, t.rows);
      const std::vector<int>* whose = nullptr;
      for (int p = 0; p < t.pieces; p++) {
        const int slot = kv_slot_of(t.w0, p);
        need(slot >= 0 && slot < 2 * cut.slots, "a part's slot", slot);
        if (q.sane) {
          need(slots.count(slot), "a part that nobody wrote", i, p, slot);
          if (p == 0) whose = &slots[slot];
          need(*whose == slots[slot] && (*whose)[1] == t.h && (*whose)[2] == t.tile && s[(*whose)[0]].t0 == t.t0, "a part of the same tile", i, p, slot);
        }
      }
      for (int r = 0; r < t.rows; r++) {
        const long long row = (long long)t.tile * cut.rows + r, at = kv_query_at(t.t0, kv_query(row, kv_token(row, q.group), q.group), t.h, q.group, q.token, q.head);
        need(at >= 0 && at + (long long)q.d * q.eb <= (q.tokens - 1) * q.token + ((long long)q.heads * q.group - 1) * q.head + (long long)q.d * q.eb, "a joined row", i, r, at);
      }
      if (q.sane) {
        const auto& cover = tiles[*whose];
        need((int)cover.size() == t.pieces, "a tile's parts", cover.size(), t.pieces);
        joined[*whose]++;
      }
    }
    if (!q.sane) return;
    for (const auto& t : tiles) need((t.second.size() > 1) == (joined.count(t.first) && joined[t.first] == 1), "a cut tile is joined", t.first[2], t.second.size());
  }
};

template <int EB, int D> void walk_of(const Call& q, const KvCut& k, long long* items, uint32_t* wgs) {
  auto go = [&](auto layout, auto kernel) {
    typedef decltype(layout) L;
    Walk w(q, k, L::UNIT);
    w.run([&](const Item& it) { kernel(w, it); });
    *items = w.items;
    *wgs = w.plan.wgs;
  };
  constexpr int NW = KvWaves<EB, D>::NW, MANY = KvWaves<EB, D>::MANY;
  if (k.rows == 16 && k.waves) go(KvFew<EB, D, 1, MANY>(), [](Walk& w, const Item& it) { w.few<KvFew<EB, D, 1, MANY>, MANY>(it); });
  else if (k.rows == 16) go(KvFew<EB, D, 1, NW>(), [](Walk& w, const Item& it) { w.few<KvFew<EB, D, 1, NW>, NW>(it); });
  else if constexpr (D * EB <= 512) {
    if (k.rows == 32 && k.waves) go(KvFew<EB, D, 2, MANY>(), [](Walk& w, const Item& it) { w.few<KvFew<EB, D, 2, MANY>, MANY>(it); });
    else if (k.rows == 32) go(KvFew<EB, D, 2, NW>(), [](Walk& w, const Item& it) { w.few<KvFew<EB, D, 2, NW>, NW>(it); });
    else go(KvWide<EB, D>(), [](Walk& w, const Item& it) { w.wide<KvWide<EB, D>>(it); });
  } else {
    need(false, "a kernel that is not built", k.rows, D, EB);
  }
}
// eb causal tokens batch heads group d page_size pages width layout sane, then starts [batch + 1], lengths [batch]
static bool walk() {
  Call q = {};
  if (std::scanf("%d %d %d %d %d %d %d %d %d %d %d %d", &q.eb, &q.causal, &q.tokens, &q.batch, &q.heads, &q.group, &q.d, &q.page_size, &q.pages, &q.width, &q.layout, &q.sane) != 12) return false;
  q.starts.resize(q.batch + 1);
  q.lengths.resize(q.batch);
  for (int& x : q.starts) if (std::scanf("%d", &x) != 1) std::exit(2);
  for (int& x : q.lengths) if (std::scanf("%d", &x) != 1) std::exit(2);
  q.table.resize((size_t)q.batch * q.width);
  for (int& x : q.table) x = rnd(20) ? (int)rnd(q.pages) : rnd(2) ? -1 - (int)rnd(1000) : q.pages + (int)rnd(1000);
  KvCache& c = q.c;
  c.pages = q.pages, c.page_size = q.page_size, c.heads = q.heads, c.d = q.d;
  const long long row = (long long)q.d * q.eb;
  if (q.layout == 0) c.slot = row, c.head = row * q.page_size, c.page = c.head * q.heads;           // [pages][heads][slots]
  else if (q.layout == 1) c.head = row, c.slot = row * q.heads, c.page = c.slot * q.page_size;      // [pages][slots][heads]
  else c.slot = row * 2 + 16, c.page = c.slot * q.page_size + 48, c.head = c.page * q.pages;        // [heads][pages][slots], with gaps
  kv_divider((uint32_t)q.page_size, &c.magic, &c.shift);
  q.extent = (q.pages - 1) * c.page + (q.heads - 1) * c.head + (q.page_size - 1) * c.slot + row;
  q.head = row + (q.layout == 2 ? q.eb : 0);
  q.token = q.head * q.heads * q.group;
  const long long room = (long long)q.width * q.page_size;
  q.most = room < KV_MAX_LENGTH ? (int)room : KV_MAX_LENGTH;
  const KvCut k = kv_cut(q.tokens, q.batch, q.group, q.heads, q.most, q.d, q.eb);
  long long items = 0;
  uint32_t wgs = 0;
  try {
    if (q.eb == 2) (q.d <= 64 ? walk_of<2, 64> : q.d <= 128 ? walk_of<2, 128> : walk_of<2, 256>)(q, k, &items, &wgs);
    else (q.d <= 64 ? walk_of<4, 64> : q.d <= 128 ? walk_of<4, 128> : walk_of<4, 256>)(q, k, &items, &wgs);
    std::printf("%d %u %lld\n", k.rows, wgs, items);
  } catch (const Wrong& w) {
    std::printf("wrong: %s\n", w.what.c_str());
  }
  return true;
}

int main(int argc, char** argv) {
  const std::string mode = argc > 1 ? argv[1] : "";
  state = 12345;
  if (mode == "walk") {
    while (walk()) {}
    return 0;
  }
  auto said = [](auto f) {
    try {
      f();
      std::printf("0\n");
    } catch (const Wrong& w) {
      std::printf("wrong: %s\n", w.what.c_str());
    }
  };
  if (mode == "quotient")
    for (uint32_t p; std::scanf("%u", &p) == 1;) said([&] { quotient(p); });
  if (mode == "seen")
    for (int words, base, n, k0, end; std::scanf("%d %d %d %d %d", &words, &base, &n, &k0, &end) == 5;) said([&] { seen(words, base, n, k0, end); });
  if (mode == "stages") {
    said(stages_of<2, 64>);
    said(stages_of<2, 128>);
    said(stages_of<2, 256>);
    said(stages_of<4, 64>);
    said(stages_of<4, 128>);
    said(stages_of<4, 256>);
  }
  return 0;
}
