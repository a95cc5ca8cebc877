// Attention of new tokens over a paged cache (the definition is in include/pahq.h).
//
// Both kernels work on transposed products: S^T = K Q^T and O^T = V^T P^T.  The matrix instruction leaves of S^T in a lane one row
// of queries and several rows of the cache, so a softmax row's maximum and sum stay in a lane but for an exchange or two, and the
// weights P are, as they lie in the registers, the right operand of the second product, if V's rows are taken in the
// same order: rows 4 h .. 4 h + 3 of every eight (or sixteen) for lane group h.  LDS reads that transpose (DS_READ_B64_TR_B16) give V that way.
// Rows of the cache reach LDS without registers (global_load_lds), each 16 bytes a lane at an address of its own, which is what pages
// need; their 16-byte chunks are XOR-swizzled by the row so that both products' reads spread over the banks.  What lies behind a
// sequence's end comes from a chunk of zeros, what lies in a page that is none from a chunk of NaN.
//
// Scores, the running maxima, the sums and the output's sums are fp32.  The weights P are rounded once to the cache's 16-bit type, at most
// half a step of each, because the second product then takes one pass of the matrix cores instead of three; the
// fp32 cache has fp32 products and no such rounding.  exp2 instead of exp: log2 e is part of the scale.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>
#include "../../include/pahq.h"
#include "device_util.h"
#include "mma_util.h"
#include "kv.h"

namespace pahq {

struct AttendArgs {
  KvCache c;
  KvBatch b;
  KvRows q, out;
  const unsigned long long* tree;
  int words, group;                                 // group: query heads of a cache head
  float scale, sign;                                // of the scores: times log2 e and positive; of the queries: its sign, 0 for a scale of 0, which multiplies them
  float* part;                                      // [slot][rows][d] sums of a part, [slot][rows][2] maximum and sum, then how many of Left there are, and they
  int slots, least, over, enough, brief;            // of ranges (kv_plan.h); slots 0: nothing is cut
  int by_pair;                                      // Left are counted by tile and head, or by range: whichever are fewer
};

// The kernel's one argument, read again where it is asked for: kept for the whole kernel it would take more scalar registers than there are.
// The kernels take nothing but it, so it begins their argument memory.
template <typename T> __device__ __forceinline__ void in_global(T*& p) {       // memory loads know only that it is some address
  p = (T*)(__attribute__((address_space(1))) T*)(uintptr_t)p;
}
__device__ __forceinline__ AttendArgs args_again() {
  uintptr_t p = (uintptr_t)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  static_assert(sizeof(AttendArgs) % 8 == 0, "whole words");
  struct Words { uint64_t w[sizeof(AttendArgs) / 8]; } x;
#pragma unroll
  for (unsigned i = 0; i < sizeof(AttendArgs) / 8; i++) x.w[i] = ((const __attribute__((address_space(4))) uint64_t*)p)[i];
  AttendArgs a = __builtin_bit_cast(AttendArgs, x);
  in_global(a.c.keys);
  in_global(a.c.values);
  in_global(a.b.starts);
  in_global(a.b.lengths);
  in_global(a.b.pages);
  in_global(a.q.at);
  in_global(a.out.at);
  in_global(a.tree);
  in_global(a.part);
  return a;
}

// ---------------------------------------------------------------- a workgroup's part
__device__ __forceinline__ int lane_of(int v, int l) { return __builtin_amdgcn_readlane(v, l); }
__device__ __forceinline__ uint32_t lane_of(uint32_t v, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); }
// Sums up to and with the own lane, sticking at 2^32 - 1: shifts by 1, 2, 4, 8 in rows of 16 lanes, then a row's last lane to the next row
// and the second row's to the last two
__device__ __forceinline__ uint32_t wave_sum_up_to(uint32_t v) {
#define STEP(control, rows) v = __builtin_elementwise_add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, control, rows, 0xF, false))
  STEP(0x111, 0xF);
  STEP(0x112, 0xF);
  STEP(0x114, 0xF);
  STEP(0x118, 0xF);
  STEP(0x142, 0xA);
  STEP(0x143, 0xC);
#undef STEP
  return v;
}
__device__ __forceinline__ KvCall call_of(const AttendArgs& a) { return {!a.tree, a.c.heads, a.group, a.slots, a.over}; }
// Sequences in lanes, 64 at a time from b0 on, and the sums of their tiles (with heads) and units up to and with each
struct Share { KvSequence s; int tiles, each; uint32_t pairs, units, pairs_to, units_to; };
template <int UNIT> __device__ __forceinline__ Share share_of(const AttendArgs& a, int rows, int b0, uint32_t pairs_before, uint32_t units_before) {
  const int b = b0 + (threadIdx.x & 63);
  Share x = {};
  if (b < a.b.batch) {
    x.s = kv_sequence(a.b, b);
    const KvShare y = kv_share(call_of(a), x.s, rows, UNIT);
    x.tiles = y.tiles;
    x.each = y.each;
    x.pairs = y.pairs;
    x.units = y.units;
  }
  x.pairs_to = __builtin_elementwise_add_sat(wave_sum_up_to(x.pairs), pairs_before);
  x.units_to = __builtin_elementwise_add_sat(wave_sum_up_to(x.units), units_before);
  return x;
}
__device__ __forceinline__ int* count_of(const AttendArgs& a, int rows) { return (int*)(a.part + kv_count_at(a.slots, rows, a.c.d)); }
__device__ __forceinline__ KvLeft* left_of(const AttendArgs& a, int rows) { return (KvLeft*)(a.part + kv_left_at(a.slots, rows, a.c.d)); }
struct Item {
  KvSequence s;
  int b, tile, h, begin, end, slot;                 // rows of the cache; slot in the workspace, -1: the whole tile
};
// Where a workgroup finds its part; every wave looks by itself.  Of up to 64 sequences KEEP keeps what was read.
template <int UNIT, bool KEEP> struct Finder {
  Share x;
  KvPlan plan;
  uint32_t pairs;
  __device__ __forceinline__ bool kept(const AttendArgs& a) const { return KEEP && a.b.batch <= 64; }
  __device__ __forceinline__ void look(const AttendArgs& a, int rows) {
    uint32_t units = 0;
    int longest = 0;
    pairs = 0;
    for (int b0 = 0; b0 < a.b.batch && (a.slots || kept(a)); b0 += 64) {
      x = share_of<UNIT>(a, rows, b0, pairs, units);
      pairs = lane_of(x.pairs_to, 63);
      units = lane_of(x.units_to, 63);
      longest = max(longest, x.tiles ? kv_units_of(x.s.length, UNIT, a.over) : 0);
    }
    // a long tile somewhere, asked for every lane's longest
    const uint32_t from = a.slots ? kv_cut_from(units, pairs, a.slots, a.enough, a.brief) : 0;
    plan = kv_plan(units, a.slots && __any((uint32_t)longest > from), a.slots, a.least);
  }
  // Sequence with the `at`-th unit, or tile and head where tiles are given out whole: its lane of x, -1 for none
  __device__ __forceinline__ int lane_with(const AttendArgs& a, int rows, uint32_t at, bool by_units, int* b0) {
    uint32_t pairs = 0, units = 0;
    for (*b0 = 0; *b0 < a.b.batch; *b0 += 64) {
      if (!kept(a)) x = share_of<UNIT>(a, rows, *b0, pairs, units);
      const unsigned long long behind = __ballot(at < (by_units ? x.units_to : x.pairs_to));
      if (behind) return __builtin_ctzll(behind);
      pairs = lane_of(x.pairs_to, 63);
      units = lane_of(x.units_to, 63);
    }
    return -1;
  }
  __device__ __forceinline__ KvSequence sequence(int l) const { return {lane_of(x.s.t0, l), lane_of(x.s.n, l), lane_of(x.s.length, l), lane_of(x.s.base, l)}; }
  // What workgroup `wg` does at `at`, up to `stop` at most.  Returns how many units that takes, 0 if there is nothing.
  __device__ __forceinline__ uint32_t next(const AttendArgs& a, int rows, int wg, uint32_t at, uint32_t stop, Item* it) {
    const uint32_t begun = at;
    const KvCall c = call_of(a);
    int b0, l, tiles;
    KvStretch x;
    for (;;) {
      l = lane_with(a, rows, at, plan.wgs, &b0);
      if (l < 0) return 0;
      it->b = b0 + l;
      it->s = sequence(l);
      it->begin = 0;
      it->slot = -1;
      tiles = lane_of(this->x.tiles, l);
      if (!plan.wgs) {
        const KvTile t = kv_whole_tile(c, tiles, at - (lane_of(this->x.pairs_to, l) - lane_of(this->x.pairs, l)));
        it->h = t.h;
        it->tile = t.tile;
        it->end = kv_end_of(c, it->s, it->tile, rows);
        return 1;
      }
      x = kv_stretch(c, it->s, tiles, lane_of(this->x.each, l), rows, UNIT, at - (lane_of(this->x.units_to, l) - lane_of(this->x.units, l)), stop - at);
      it->h = x.h;
      it->tile = x.tile;
      at += x.take;
      if (x.work && x.off + x.take > (uint32_t)c.over) break;
      if (at >= stop) return 0;
    }
    it->end = kv_end_of(c, it->s, it->tile, rows);
    const bool starts = kv_begins(c, x), ends = kv_ends(x);
    if (!starts) it->begin = kv_begin_of(c, x, UNIT, it->end);
    if (!ends) it->end = kv_stop_of(c, x, UNIT, it->end);
    if (!starts || !ends) it->slot = kv_slot(wg, starts);
    if (starts && (!ends || a.by_pair) && threadIdx.x == 0) {
      const uint32_t number = kv_number(lane_of(this->x.pairs_to, l) - lane_of(this->x.pairs, l), it->h, tiles, it->tile);
      if (!a.by_pair || number < (uint32_t)a.slots)
        left_of(a, rows)[a.by_pair ? number : wg] = {it->s.t0, (int)min((long long)it->s.n * a.group - (long long)it->tile * rows, (long long)rows), it->tile, it->h,
                                                     ends ? 0 : kv_holder(plan, at - x.take - x.off + x.whole - 1) - wg + 1, wg, {}};
    }
    return at - begun;
  }
  // A range says first that it left nothing; the first one how many Left there are
  __device__ __forceinline__ void begin(const AttendArgs& a, int rows, int wg) const {
    if (!a.slots || threadIdx.x) return;
    if (plan.wgs && !a.by_pair) left_of(a, rows)[wg].pieces = 0;
    if (plan.wgs ? wg == 0 : blockIdx.x == 0) *count_of(a, rows) = plan.wgs ? (int)(a.by_pair ? min(pairs, (uint32_t)a.slots) : plan.wgs) : 0;
  }
};
__device__ __forceinline__ unsigned long long seen_bits(const AttendArgs& a, const KvSequence& s, int i, int k0, int end) {
  return kv_seen(a.tree, a.words, s, i, k0, end);
}
// x where bit n of seen is set, else -infinity
__device__ __forceinline__ float seen_score(uint32_t seen, int n, float x) {
  const uint32_t keep = (uint32_t)((int)(seen << (31 - n)) >> 31);
  return __uint_as_float((__float_as_uint(x) & keep) | (0xFF800000u & ~keep));
}

#define INLINE __attribute__((always_inline))

// ---------------------------------------------------------------- fragments
// Sixteen bytes of a row are one operand of a step of the 16-bit products and of four steps of the fp32 products
template <typename T> struct Frag;
typedef float v16f __attribute__((ext_vector_type(16)));
typedef short v4s __attribute__((ext_vector_type(4)));
template <> struct Frag<bf16_t> {
  typedef v8bf type;
  static __device__ __forceinline__ v4f mma16(v8bf a, v8bf b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ v16f mma32(v8bf a, v8bf b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Frag<f16_t> {
  typedef v8h type;
  static __device__ __forceinline__ v4f mma16(v8h a, v8h b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ v16f mma32(v8h a, v8h b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <> struct Frag<float> {
  typedef v4f type;
  static __device__ __forceinline__ v4f mma16(v4f a, v4f b, v4f c) {
#pragma unroll
    for (int e = 0; e < 4; e++) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ v16f mma32(v4f a, v4f b, v16f c) {
#pragma unroll
    for (int e = 0; e < 4; e++) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
  }
};
// A row's maximum is not followed at every step: weights may exceed 1, and rescaling the sums, which costs a product for each of the
// output's columns, is left out for nearly every block after the first ones.  Few rows of queries: the maximum is taken over when it has grown by
// more than LAG (as a power of two).  Many: when the block's weights add up to more than OVER, which costs no maximum of the block.
// fp16 weights are multiplied by 2^7, so that those down to 2^-21 of the largest are normal numbers; the lag of 2^8 makes 2^15 of the largest,
// and a sum below OVER none larger than that: half of what fp16 holds.  The factor leaves with the division by the sum.
template <typename T> constexpr float LIFT = sizeof(T) == 2 && !__is_same(T, bf16_t) ? 7.f : 0.f;
constexpr float LAG = 8.f;
constexpr float OVER = 32768.f;
// acc + the sum of a fragment's elements
__device__ __forceinline__ float sum_of(v8bf x, float acc) {
  typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int j = 0; j < 8; j += 2) acc = __builtin_amdgcn_fdot2_f32_bf16((v2bf){x[j], x[j + 1]}, (v2bf){(__bf16)1.f, (__bf16)1.f}, acc, false);
  return acc;
}
__device__ __forceinline__ float sum_of(v8h x, float acc) {
#pragma unroll
  for (int j = 0; j < 8; j += 2) acc = __builtin_amdgcn_fdot2((v2h){x[j], x[j + 1]}, (v2h){(_Float16)1.f, (_Float16)1.f}, acc, false);
  return acc;
}
__device__ __forceinline__ float sum_of(v4f x, float acc) { return acc + ((x[0] + x[1]) + (x[2] + x[3])); }

alignas(16) __device__ const uint32_t kv_chunk[4][4] = {{0, 0, 0, 0}, {0x7FC00000, 0x7FC00000, 0x7FC00000, 0x7FC00000},
                                                        {0x7FC07FC0, 0x7FC07FC0, 0x7FC07FC0, 0x7FC07FC0}, {0x7E007E00, 0x7E007E00, 0x7E007E00, 0x7E007E00}};
// A scale of 0: queries of zeros, and NaN where they were not finite
template <typename T, typename F> __device__ __forceinline__ F times_zero(F q) {
#pragma unroll
  for (int j = 0; j < 16 / (int)sizeof(T); j++) q[j] = (T)((float)q[j] * 0.f);
  return q;
}
template <typename T> constexpr uint32_t SIGNS = sizeof(T) == 4 ? 0x80000000u : 0x80008000u;
template <typename T> constexpr int NAN_CHUNK = sizeof(T) == 4 ? 1 : __is_same(T, bf16_t) ? 2 : 3;

// What lies at an address of LDS.  The reads of a block differ from one base by constants (kv_address.h): `base` is hidden from the compiler so that it derives each address where it is used instead of
// keeping sixteen of them.
template <typename F> __device__ __forceinline__ F at_lds(uint32_t a) { return *(const __attribute__((address_space(3))) F*)(uintptr_t)a; }
__device__ __forceinline__ v4s at_lds_turned(uint32_t a) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(uintptr_t)a); }
__device__ __forceinline__ uint32_t hidden(uint32_t base) {
  asm volatile("" : "+v"(base));
  return base;
}

// Rows of the cache on their way into LDS.  A lane keeps where its row of a block lies; the pages' numbers came through LDS themselves
// (`ids`, asked for two blocks ahead), because a load into a register would make the compiler wait for everything in flight.
__device__ __forceinline__ void ask_page(const KvCache& c, const int* pages, int row, int end, uint32_t lds) { lds_load4(pages + kv_asked(c, row, end), lds); }
// Rows r0 .. of a block, 64 / CH of them (r0 a multiple of that), chunk by chunk: lane l writes the l-th 16 bytes behind lds.  Their
// offsets lie in lanes `first` and on.  A lane's chunk: bytes behind the head's first row, or what stands for a chunk that is none.
struct Chunk { long long off; const char* fill; };
template <typename T, int CH> __device__ __forceinline__ Chunk chunk_of(const KvCache& c, int lane, long long mine, int first, int r0) {
  const int chunk = kv_asks_chunk<CH>(lane, r0);
  const long long at = (long long)__shfl((unsigned long long)mine, first + kv_asks_row<CH>(lane), 64);
  const bool behind = chunk * 16 >= c.d * (int)sizeof(T);
  return {at + chunk * 16, at < 0 || behind ? (const char*)kv_chunk[at == KV_ROW_NONE && !behind ? NAN_CHUNK<T> : 0] : nullptr};
}
template <bool ONCE> __device__ __forceinline__ void ask_chunk(const char* from, const Chunk& x, uint32_t lds) {
  const uint8_t* const at = (const uint8_t*)(x.fill ? x.fill : from + x.off);
  if (ONCE) slab_load16_nt(at, lds);
  else slab_load16(at, lds);
}

// Nothing but arithmetic outside of the matrix cores may be moved across
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0x6); }

// Values that some query of the tile does not see may be infinities or NaN, and 0 * NaN is one.  They leave the product, and come back
// through another one, of which kinds a query sees: up to 32 rows count 1 each for infinity, 64 for -infinity, 4096 for NaN.
template <typename T, typename F> __device__ __forceinline__ bool not_finite(F v) {
  bool bad = false;
#pragma unroll
  for (int j = 0; j < 16 / (int)sizeof(T); j++) bad |= !(fabsf((float)v[j]) < INFINITY);
  return bad;
}
template <typename T, typename F> __device__ __forceinline__ F take_kinds(F* v) {
  F kinds;
#pragma unroll
  for (int j = 0; j < 16 / (int)sizeof(T); j++) {
    const float x = (float)(*v)[j];
    const uint32_t fine = fabsf(x) < INFINITY ? ~0u : 0u, up = x == INFINITY ? 0x3F800000u : 0u, down = x == -INFINITY ? 0x42800000u : 0u, no = x != x ? 0x45800000u : 0u;
    kinds[j] = (T)__uint_as_float(up | down | no);            // 1, 64, 4096
    (*v)[j] = (T)__uint_as_float(__float_as_uint(x) & fine);
  }
  return kinds;
}
// That is done in masked blocks.  In the others an infinite value times a weight that rounded to zero, or an infinite sum that is rescaled by
// zero, leaves NaN where infinity belongs, for the weight is positive in the definition: a tile with a NaN is done once more with all its
// blocks masked, and sums are rescaled so there, and where parts of them meet, that infinities stay.  To look for a NaN and to have all
// waves know takes 0.5 us of a call of 9 us, 1.5 us of the 44 us of the trees below, nothing to 0.5 % of the long ones.
template <typename V> __device__ __forceinline__ V rescaled(V x, float by) { return __builtin_elementwise_abs(x) == INFINITY ? x : x * by; }
template <typename V> __device__ __forceinline__ bool has_nan(const V& x) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(V) / 4); i++) bad |= x[i] != x[i];
  return bad;
}
// Whether one of the waves said so in LDS, as every lane's value
template <int NW> __device__ __forceinline__ bool any_of(const int* said) {
  int any = 0;
#pragma unroll
  for (int w = 0; w < NW; w++) any |= said[w];
  return __builtin_amdgcn_readfirstlane(any);
}
// 1 where a bit is set, else 0
template <typename T> __device__ __forceinline__ T one_bit(uint32_t seen, int n) { return (T)__uint_as_float((seen >> n & 1u) * 0x3F800000u); }
__device__ __forceinline__ float of_kinds(float count) {
  const int n = (int)count;
  const uint32_t up = (n & 63) ? 0x7F800000u : 0u, down = (n & 4032) ? 0xFF800000u : 0u, no = n >= 4096 ? 0x7FC00000u : 0u;
  return __uint_as_float(up) + __uint_as_float(down) + __uint_as_float(no);        // inf - inf: NaN
}

// ---------------------------------------------------------------- up to 16 RT rows of queries
// For query row r:  O_r = sum_j 2^(s_rj - m) V_j / sum_j 2^(s_rj - m),  s_rj = scale log2(e) q_r . k_j over the rows j that r sees, in one
// pass over K and V with m the running maximum.  Bound by memory: 2 d bytes-an-element for 4 d operations a query row.
//
// A wave takes blocks of KVB rows of the cache in turn with the others of its workgroup, into two stages of LDS of its own, so nothing waits for
// another wave until the waves' sums meet at the end.  The stages of
// a compute unit hold 128 KB, half of it on its way, which is what the latency of memory takes at 7 TB/s; one workgroup of MANY waves holds all,
// two of NW waves each half (cut_of).  Rows are read once a tile, so the reads are marked as non-temporal: 173 us instead of 194 for the 64 tokens below.
// RT = 2 serves 17 to 32 rows with one pass instead of two (16 sequences, 8 tokens of 4 heads, 4096 rows: 58 us, 63 in tiles of 16, 65 of 128).
//
// Measured, bf16, 8 heads of 128 columns for 32 of queries: 64 tokens over 1024 to 16384 rows, 1.07 GB, 172 us (6.2 TB/s); one token over 131072
// rows, 537 MB, 88 us (6.1 TB/s); fp32, 12 heads of 64 columns, one token over 200 rows 9.6 us, most of it the launch and the reads of the lists, the
// page's number and its rows, which wait for one another.
template <typename T, int D, int RT, int NW>
__global__ __launch_bounds__(NW * 64) void kv_few_k(AttendArgs a) {
  typedef typename Frag<T>::type F;
  typedef KvFew<sizeof(T), D, RT, NW> L;
  constexpr int EB = sizeof(T), CH = L::CH, KT = L::KT, KVB = L::KVB, ROWS = L::ROWS, HALF = L::HALF, ASKS = L::ASKS, DT = L::DT;
  extern __shared__ __align__(1024) char lds[];
  __shared__ float stat[NW][ROWS][2];
  __shared__ int lost[NW];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, h4 = lane >> 4;
  Finder<L::UNIT, true> f;
  f.look(args_again(), ROWS);
  const int wg = f.plan.wgs ? kv_wg_of(blockIdx.x, f.plan.wgs) : 0;
  if (wg < 0) return;
  f.begin(args_again(), ROWS, wg);
  uint32_t at = f.plan.wgs ? kv_from(f.plan, wg) : blockIdx.x;
  const uint32_t stop = f.plan.wgs ? kv_from(f.plan, wg + 1) : at + 1;
  for (bool first = true, again = false; at < stop; first = false) {
  Item it;
  const uint32_t take = f.next(args_again(), ROWS, wg, at, stop, &it);
  if (!take) return;
  at += take;
  const int begin = it.begin, end = it.end, h = it.h;
  if (!first) __syncthreads();                      // the stages held the last tile's sums

  // the tile's queries: lane l16 of row tile r holds chunks h4, h4 + 4, ... of row 16 r + l16; zeros where there is none, from memory that is there
  const int group = a.group;
  int token[RT];
  F q[RT][CH / 4];
  {
    const AttendArgs k = args_again();
    const uint32_t flip = k.sign < 0.f ? SIGNS<T> : 0u;
#pragma unroll
    for (int r = 0; r < RT; r++) {
      const long long row = (long long)it.tile * ROWS + 16 * r + l16;
      const bool there = row < (long long)it.s.n * group;
      token[r] = there ? kv_token(row, group) : -1;
      const T* const x = (const T*)(k.q.at + kv_query_at(it.s.t0, there ? kv_query(row, token[r], group) : KvQuery{0, 0}, h, group, k.q.token, k.q.head));
#pragma unroll
      for (int s = 0; s < CH / 4; s++) {
        const int e0 = (h4 + 4 * s) * (16 / EB);
        q[r][s] = __builtin_bit_cast(F, (load16(x + (e0 < k.c.d ? e0 : 0)) & (there && e0 < k.c.d ? ~0u : 0u)) ^ flip);
        if (k.sign == 0.f) q[r][s] = times_zero<T>(q[r][s]);
      }
    }
  }

  const int* const pages = a.b.pages + it.b * a.b.ld;
  const long long head = h * a.c.head;
  const uint32_t stage0 = __builtin_amdgcn_readfirstlane(lds_addr_of(lds + L::stages(wave)));
  const int* const ids = (const int*)(lds + L::ids(wave));
  const uint32_t ids0 = __builtin_amdgcn_readfirstlane(lds_addr_of(ids));
  const int blocks = end > begin ? (end - begin + KVB - 1) / KVB : 0, turns = blocks > wave ? (blocks - wave + NW - 1) / NW : 0;
  auto first_row = [&](int n) { return begin + (wave + n * NW) * KVB; };
  auto ask_ids = [&](int n) INLINE { ask_page(a.c, pages, first_row(n) + (lane & (KVB - 1)), end, ids0 + L::ids_of(n)); };
  auto ask_block = [&](int n) INLINE {
    const long long at = kv_row_or_behind(a.c, first_row(n) + (lane & (KVB - 1)), end, ids[L::ids_of(n) / 4 + lane]);
    const uint32_t to = stage0 + L::stage(n);
#pragma unroll
    for (int j = 0; j < ASKS; j++) {
      const Chunk x = chunk_of<T, CH>(a.c, lane, at, j * (64 / CH), j * (64 / CH));
      ask_chunk<true>(a.c.keys + head, x, to + j * 1024);
      ask_chunk<true>(a.c.values + head, x, to + HALF + j * 1024);
    }
  };
  // blocks that every query of the tile sees whole come first
  const int sure = again ? 0 : min(end, it.s.base + (a.tree ? 0 : (int)((long long)it.tile * ROWS / group) + 1));
  v4f o[RT][DT] = {};
  float m[RT], l[RT];
#pragma unroll
  for (int r = 0; r < RT; r++) m[r] = -INFINITY, l[r] = 0.f;

  if (turns) {
    ask_ids(0);
    ask_ids(1);
    ask_ids(2);
    wait_vm_lds<0>();
    ask_block(0);
  }
  auto block = [&](int n, auto is_masked) INLINE {
    constexpr bool masked = decltype(is_masked)::value;
    const int k0 = first_row(n);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // the stage's last reads
    if (n + 1 < turns) {
      ask_ids(n + 3);                                            // a place in the list is asked for even behind the last block
      ask_block(n + 1);
      wait_vm_lds<2 * ASKS + 1>();
    } else {
      wait_vm_lds<0>();
    }
    const uint32_t stage = stage0 + L::stage(n);
    const uint32_t ks = hidden(stage + L::key0(l16, h4));
    v4f s[RT][KT];
#pragma unroll
    for (int t = 0; t < KT; t++) {
#pragma unroll
      for (int r = 0; r < RT; r++) s[r][t] = (v4f){0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < CH / 4; c++) {
        const F k = at_lds<F>(L::key(ks, t, c));
#pragma unroll
        for (int r = 0; r < RT; r++) s[r][t] = Frag<T>::mma16(k, q[r][c], s[r][t]);
      }
    }
    uint32_t seen[RT];
    float p[RT][KT][4];
#pragma unroll
    for (int r = 0; r < RT; r++) {
      if (masked) seen[r] = (uint32_t)(seen_bits(args_again(), it.s, token[r], k0, end) >> (4 * h4));
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < KT; t++)
#pragma unroll
        for (int i = 0; i < 4; i++) {
          float x = s[r][t][i] * a.scale;
          if (masked) x = seen_score(seen[r], 16 * t + i, x);
          p[r][t][i] = x;
          top = fmaxf(top, x);
        }
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const bool more = top > m[r] + LAG;                        // of this row alone: its neighbours' scores change nothing in it
      if (__any(more)) {
        const float f = more ? __builtin_amdgcn_exp2f(m[r] - top) : 1.f;
        if (more) m[r] = top;
        l[r] *= f;
#pragma unroll
        for (int d = 0; d < DT; d++)
          if (masked && sure == 0) o[r][d] = rescaled(o[r][d], f);
          else o[r][d] *= f;
      }
      const float from = (m[r] == -INFINITY ? 0.f : m[r]) - LIFT<T>;
#pragma unroll
      for (int t = 0; t < KT; t++)
#pragma unroll
        for (int i = 0; i < 4; i++) {
          p[r][t][i] = __builtin_amdgcn_exp2f(p[r][t][i] - from);
          if (EB == 4) l[r] += p[r][t][i];
        }
    }
    const uint32_t vs = hidden(stage + L::value0(l16, h4));
    if constexpr (EB == 2) {
      F w[RT];
#pragma unroll
      for (int r = 0; r < RT; r++) {
#pragma unroll
        for (int j = 0; j < 8; j++) w[r][j] = (T)p[r][j / 4][j % 4];
        l[r] = sum_of(w[r], l[r]);                               // of the weights as they multiply the values
      }
#pragma unroll
      for (int d = 0; d < DT; d++) {
        union { F f; v4s half[2]; } v;
#pragma unroll
        for (int t = 0; t < 2; t++) v.half[t] = at_lds_turned(L::value_16_bit(vs, t, d));
        if (masked && __any(not_finite<T>(v.f))) {
          const F kinds = take_kinds<T>(&v.f);
#pragma unroll
          for (int r = 0; r < RT; r++) {
            F one;
#pragma unroll
            for (int j = 0; j < 8; j++) one[j] = one_bit<T>(seen[r], 16 * (j / 4) + j % 4);
            const v4f n = Frag<T>::mma16(kinds, one, (v4f){0, 0, 0, 0});
#pragma unroll
            for (int i = 0; i < 4; i++) o[r][d][i] += of_kinds(n[i]);
          }
        }
#pragma unroll
        for (int r = 0; r < RT; r++) o[r][d] = Frag<T>::mma16(v.f, w[r], o[r][d]);
      }
    } else {
#pragma unroll
      for (int d = 0; d < DT; d++) {
        F v;
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = at_lds<float>(L::value_fp32(vs, i, d));
        if (masked && __any(not_finite<T>(v))) {
          const F kinds = take_kinds<T>(&v);
#pragma unroll
          for (int r = 0; r < RT; r++) {
            F one;
#pragma unroll
            for (int i = 0; i < 4; i++) one[i] = one_bit<float>(seen[r], i);
            const v4f n = Frag<T>::mma16(kinds, one, (v4f){0, 0, 0, 0});
#pragma unroll
            for (int i = 0; i < 4; i++) o[r][d][i] += of_kinds(n[i]);
          }
        }
#pragma unroll
        for (int r = 0; r < RT; r++) o[r][d] = Frag<T>::mma16(v, (F){p[r][0][0], p[r][0][1], p[r][0][2], p[r][0][3]}, o[r][d]);
      }
    }
  };
  int n = 0;
  for (; n < turns && first_row(n) + KVB <= sure; n++) block(n, std::false_type());
  for (; n < turns; n++) block(n, std::true_type());

  // the waves' sums: [row][d] in the wave's stages, chunks of four swizzled by the row
  bool bad = false;
#pragma unroll
  for (int r = 0; r < RT; r++) {
    l[r] += __shfl_xor(l[r], 16, 64);
    l[r] += __shfl_xor(l[r], 32, 64);
    const int row = 16 * r + l16;
    if (h4 == 0) stat[wave][row][0] = m[r], stat[wave][row][1] = l[r];
#pragma unroll
    for (int d = 0; d < DT; d++) {
      *(v4f*)(lds + L::sum(wave, row, 4 * d + h4)) = o[r][d];
      bad |= has_nan(o[r][d]);
    }
  }
  lost[wave] = __any(bad);
  __syncthreads();
  again = !again && any_of<NW>(lost);
  if (again) {
    at -= take;
    continue;
  }
  const AttendArgs k = args_again();
  for (int e = threadIdx.x; e < ROWS * (D / 4); e += NW * 64) {
    const int row = e / (D / 4), c = e % (D / 4);
    const long long of = (long long)it.tile * ROWS + row;
    if (of >= (long long)it.s.n * group || c * 4 >= k.c.d) continue;
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < NW; w++) top = fmaxf(top, stat[w][row][0]);
    v4f y = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < NW; w++) {
      const float f = __builtin_amdgcn_exp2f(stat[w][row][0] - (top == -INFINITY ? 0.f : top));
      sum += f * stat[w][row][1];
      y += rescaled(*(const v4f*)(lds + L::sum(w, row, c)), f);
    }
    if (it.slot >= 0) {
      *(v4f*)(k.part + kv_part_at(it.slot, ROWS, row, k.c.d) + c * 4) = y;
      float* const st = k.part + kv_stat_at(k.slots, it.slot, ROWS, row, k.c.d);
      if (c == 0) st[0] = top, st[1] = sum;
    } else {
      Pack<T, 4> z;
#pragma unroll
      for (int j = 0; j < 4; j++) z.v[j] = from_float<T>(sum == 0.f ? 0.f : y[j] / sum);
      *(Pack<T, 4>*)((T*)(const_cast<char*>(k.out.at) + kv_query_at(it.s.t0, kv_query(of, kv_token(of, group), group), h, group, k.out.token, k.out.head)) + c * 4) = z;
    }
  }
  }
}

// ---------------------------------------------------------------- many rows of queries
// The same sums.  Four waves of 32 rows each share blocks of KVB rows of the cache, in two stages of LDS: a block's products run while the next one
// arrives.  4 d operations for each row of queries against 2 d elements for all 128 of them: bound by instructions, not memory.  32x32 products
// rather than 16x16, for they read half of the LDS for the same work.  K and V are read from LDS AHEAD = 4 products before they are used, held
// there by in_order(): left to the compiler each product waits for its own read (the prompt below, on one card: 552 us with one read ahead, 519
// with two, 517 with four; more do not fit the registers).  KVB is 64 where two stages of it fit twice into LDS (32: 553 us), 32 for rows of more than 256 bytes.
//
// Measured, bf16, 8 heads of 128 columns for 32 of queries: a prompt of 8192 tokens 517 to 558 us, by card and state (0.99 to 1.06 PFLOP/s; the
// matrix cores are busy for about half of it, the exponentials, masks and roundings beside them take the other half of the issue slots);
// 8 trees of 64 tokens over up to 8000 rows 44 us; 512 tokens of a prompt 19 us.
template <typename T, int D> constexpr int TILE_WAVES = D * sizeof(T) <= 128 ? 3 : D * sizeof(T) <= 256 ? 2 : 1;       // of a SIMD
template <typename T, int D, int KVB>
__global__ __launch_bounds__(256, (TILE_WAVES<T, D>)) void kv_tile_k(AttendArgs a) {
  typedef typename Frag<T>::type F;
  typedef KvWide<sizeof(T), D> L;
  constexpr int EB = sizeof(T), CH = L::CH, KT = L::KT, NW = L::NW, ROWS = L::ROWS, N = L::N, HALF = L::HALF, MINE = L::MINE, ASKS = L::ASKS, DT = L::DT;
  static_assert(KVB == L::KVB, "what the addresses are for");
  extern __shared__ __align__(1024) char lds[];
  __shared__ int lost[2][NW];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, h2 = lane >> 5;
  Finder<KVB, false> f;
  f.look(args_again(), ROWS);
  const int wg = f.plan.wgs ? kv_wg_of(blockIdx.x, f.plan.wgs) : 0;
  if (wg < 0) return;
  f.begin(args_again(), ROWS, wg);
  uint32_t at = f.plan.wgs ? kv_from(f.plan, wg) : blockIdx.x;
  const uint32_t stop = f.plan.wgs ? kv_from(f.plan, wg + 1) : at + 1;
  int pass = 0;
  for (bool again = false; at < stop; pass ^= 1) {
    Item it;
    const uint32_t take = f.next(args_again(), ROWS, wg, at, stop, &it);
    if (!take) return;
    at += take;
    const int begin = it.begin, end = it.end, h = it.h;

    const int group = a.group;
    // the wave's queries: lane l32 holds chunks h2, h2 + 2, ... of its row; zeros where there is none, from memory that is there
    const long long row0 = (long long)it.tile * ROWS + wave * 32, row = row0 + l32;
    const bool there = row < (long long)it.s.n * group;
    const int token = there ? kv_token(row, group) : -1;
    F q[CH / 2];
    {
      const AttendArgs k = args_again();
      const uint32_t flip = k.sign < 0.f ? SIGNS<T> : 0u;
      const T* const x = (const T*)(k.q.at + kv_query_at(it.s.t0, there ? kv_query(row, token, group) : KvQuery{0, 0}, h, group, k.q.token, k.q.head));
#pragma unroll
      for (int c = 0; c < CH / 2; c++) {
        const int e0 = (h2 + 2 * c) * N;
        q[c] = __builtin_bit_cast(F, (load16(x + (e0 < k.c.d ? e0 : 0)) & (there && e0 < k.c.d ? ~0u : 0u)) ^ flip);
        if (k.sign == 0.f) q[c] = times_zero<T>(q[c]);
      }
    }
    // what the wave's rows see at least (unmasked) and at most: blocks behind the latter are left out
    const int last = min(it.s.n - 1, (int)((row0 + 31) / group));
    const int sure = again ? 0 : min(end, it.s.base + (a.tree ? 0 : (int)(row0 / group) + 1));
    const int wave_end = row0 >= (long long)it.s.n * group ? 0 : a.tree ? end : min(end, it.s.base + last + 1);

    const int* const pages = a.b.pages + it.b * a.b.ld;
    const long long head = h * a.c.head;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_addr_of(lds));
    const int* const ids = (const int*)(lds + L::ids(wave));
    const uint32_t ids0 = __builtin_amdgcn_readfirstlane(lds_addr_of(ids));
    const int blocks = end > begin ? (end - begin + KVB - 1) / KVB : 0;
    const bool simple = L::simple(a.c);
    auto row_of = [&](int n) INLINE { return begin + n * KVB + wave * MINE; };
    auto ask_ids = [&](int n) INLINE { ask_page(a.c, pages, row_of(n) + (lane & (MINE - 1)), end, ids0 + L::ids_of(n)); };
    // Rows in one page by an offset from the wave's place, anything else row by row, which takes a hundred instructions instead of a dozen.
    auto ask_block = [&](int n, bool whole) INLINE {
      const uint32_t to = lds0 + L::stage(n) + L::share(wave);
      const int page = __builtin_amdgcn_readfirstlane(ids[L::ids_of(n) / 4]);
      if (whole && kv_is_page(a.c, page)) {
        const char* k = a.c.keys + (head + kv_row_of_page(a.c, row_of(n), page));
        const long long apart = a.c.values - a.c.keys;
#pragma unroll
        for (int j = 0; j < ASKS; j++) {
          const uint32_t off = L::simple_offset(lane, wave * MINE + j * (64 / CH), (uint32_t)a.c.slot);
          slab_load16s((const uint8_t*)k, off, to + j * 1024);
          slab_load16s((const uint8_t*)k + apart, off, to + HALF + j * 1024);
          k += 64 / CH * a.c.slot;
        }
      } else {
        const int l = hidden(lane);                 // nothing of this is worth a register beside the blocks that do without it
        const AttendArgs k = args_again();
        const long long mine = kv_row_or_behind(k.c, row_of(n) + (l & (MINE - 1)), end, ids[L::ids_of(n) / 4 + l]);
#pragma unroll
        for (int j = 0; j < ASKS; j++) {
          const Chunk x = chunk_of<T, CH>(k.c, l, mine, j * (64 / CH), wave * MINE + j * (64 / CH));
          ask_chunk<false>(k.c.keys + head, x, to + j * 1024);
          ask_chunk<false>(k.c.values + head, x, to + HALF + j * 1024);
        }
      }
    };
    const uint32_t k_at = L::key0(l32, h2), v_at = L::value0(lane);
    v16f o[DT] = {};
    float m = -INFINITY, l = 0.f;
    auto block = [&](int n, auto is_masked) INLINE {
      constexpr bool masked = decltype(is_masked)::value;
      const int k0 = begin + n * KVB;
      wait_vm_barrier<0>();
      if (n + 1 < blocks) {
        ask_block(n + 1, simple && L::simple_block(k0 + KVB, end));
        ask_ids(n + 2);
      }
      if (masked && k0 >= wave_end) return;
      const uint32_t ks = hidden(lds0 + L::stage(n) + k_at);
      // products and the reads AHEAD of them in a fixed order: left alone, the compiler waits for every read in front of its product
      constexpr int QK = KT * CH / 2, STEPS = L::STEPS, PV = KT * STEPS * DT, AHEAD = 4;
      v16f s[KT];
      F k[AHEAD];
      auto key = [&](int i) INLINE { return at_lds<F>(L::key(ks, i / (CH / 2), i % (CH / 2))); };
#pragma unroll
      for (int i = 0; i < AHEAD; i++) k[i] = key(i);
#pragma unroll
      for (int i = 0; i < QK; i++) {
        const v16f zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
        in_order();
        s[i / (CH / 2)] = Frag<T>::mma32(k[i % AHEAD], q[i % (CH / 2)], i % (CH / 2) ? s[i / (CH / 2)] : zero);
        if (i + AHEAD < QK) k[i % AHEAD] = key(i + AHEAD);
      }
      uint32_t seen[KT];
      if (masked) {
        const unsigned long long bits = seen_bits(args_again(), it.s, token, k0, end) >> (4 * h2);
#pragma unroll
        for (int t = 0; t < KT; t++) {
          seen[t] = (uint32_t)(bits >> (32 * t));
#pragma unroll
          for (int i = 0; i < 16; i++) s[t][i] = seen_score(seen[t], 8 * (i / 4) + i % 4, s[t][i]);
        }
      }
      // Weights against the maximum so far.  As long as their sum stays below OVER, which no sum does before the first maximum is taken, no
      // weight is too large and the block's own maximum is not needed.
      F w[KT * STEPS];
      float sum;
      auto weights = [&](float from) INLINE {
        sum = 0.f;
#pragma unroll
        for (int e = 0; e < KT * 16; e++) w[e / N][e % N] = (T)__builtin_amdgcn_exp2f(__fmaf_rn(s[e / 16][e % 16], a.scale, from));
#pragma unroll
        for (int i = 0; i < KT * STEPS; i++) sum = sum_of(w[i], sum);
      };
      weights(LIFT<T> - m);
      if (__any(!(sum <= OVER))) {
        // of this row alone: its neighbours' scores change nothing in it
        const float other = __shfl_xor(sum, 32, 64);
        const bool more = !(sum <= OVER) || !(other <= OVER);
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < KT * 16; e++) top = fmaxf(top, s[e / 16][e % 16]);
        top = fmaxf(top, __shfl_xor(top, 32, 64)) * a.scale;
        const float to = more && top > m ? top : m, by = to == m ? 1.f : __builtin_amdgcn_exp2f(m - to);
        m = to;
        l *= by;
#pragma unroll
        for (int d = 0; d < DT; d++)
          if (masked && sure == 0) o[d] = rescaled(o[d], by);
          else o[d] *= by;
        weights(LIFT<T> - (m == -INFINITY ? 0.f : m));       // nothing seen so far, or only scores of -inf: zeros
      }
      l += sum;
      const uint32_t vs = hidden(lds0 + L::stage(n) + v_at);
      F v[AHEAD];
      auto value = [&](int i) INLINE {
        const int d = i % DT, row = i / DT * 2 * N;
        F x;
        if constexpr (EB == 2) {
          union { F f; v4s half[2]; } y;
#pragma unroll
          for (int j = 0; j < 2; j++) y.half[j] = at_lds_turned(L::value_16_bit(vs, row, j, d));
          x = y.f;
        } else {
#pragma unroll
          for (int j = 0; j < 4; j++) x[j] = at_lds<float>(L::value_fp32(vs, row, j, d));
        }
        return x;
      };
#pragma unroll
      for (int i = 0; i < AHEAD; i++) v[i] = value(i);
#pragma unroll
      for (int i = 0; i < PV; i++) {
        const int d = i % DT, t = i / DT / STEPS, u = i / DT % STEPS;
        if (masked && __any(not_finite<T>(v[i % AHEAD]))) {
          const F kinds = take_kinds<T>(&v[i % AHEAD]);
          F one;
#pragma unroll
          for (int j = 0; j < N; j++) one[j] = one_bit<T>(seen[t], 2 * N * u + 8 * (j / 4) + j % 4);
          const v16f count = Frag<T>::mma32(kinds, one, (v16f){0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0});
#pragma unroll
          for (int e = 0; e < 16; e++) o[d][e] += of_kinds(count[e]);
        }
        in_order();
        o[d] = Frag<T>::mma32(v[i % AHEAD], w[i / DT], o[d]);
        if (i + AHEAD < PV) v[i % AHEAD] = value(i + AHEAD);
      }
    };
    if (blocks > 0) {
      ask_ids(0);
      wait_vm_lds<0>();
      ask_block(0, simple && L::simple_block(begin, end));
      ask_ids(1);
    }
    // blocks that every query of the wave sees whole come first
    int n = 0;
    for (; n < blocks && begin + n * KVB + KVB <= sure; n++) block(n, std::false_type());
    for (; n < blocks; n++) block(n, std::true_type());
    bool bad = false;
#pragma unroll
    for (int d = 0; d < DT; d++) bad |= has_nan(o[d]);
    lost[pass][wave] = __any(bad);                  // read while others say the next one
    l += __shfl_xor(l, 32, 64);
    if (there && it.slot >= 0) {
      const AttendArgs k = args_again();
      const int in = wave * 32 + l32;
      float* const part = k.part + kv_part_at(it.slot, ROWS, in, k.c.d);
      if (h2 == 0) {
        float* const st = k.part + kv_stat_at(k.slots, it.slot, ROWS, in, k.c.d);
        st[0] = m, st[1] = l;
      }
#pragma unroll
      for (int d = 0; d < DT; d++)
#pragma unroll
        for (int p = 0; p < 4; p++) {
          const int e = 32 * d + 8 * p + 4 * h2;
          if (e < k.c.d) *(v4f*)(part + e) = (v4f){o[d][4 * p], o[d][4 * p + 1], o[d][4 * p + 2], o[d][4 * p + 3]};
        }
    }
    __syncthreads();                                // the stages are free, and all waves go over the tile again or none; results may lie where queries did
    again = !again && any_of<NW>(lost[pass]);
    if (again) {
      at -= take;
      continue;
    }
    if (there && it.slot < 0) {
      const AttendArgs k = args_again();
      T* const out = (T*)(const_cast<char*>(k.out.at) + kv_query_at(it.s.t0, kv_query(row, token, group), h, group, k.out.token, k.out.head));
      const float by = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
      for (int d = 0; d < DT; d++)
#pragma unroll
        for (int p = 0; p < 4; p++) {
          const int e = 32 * d + 8 * p + 4 * h2;
          if (e >= k.c.d) continue;
          Pack<T, 4> z;
#pragma unroll
          for (int j = 0; j < 4; j++) z.v[j] = from_float<T>(l == 0.f ? 0.f : o[d][4 * p + j] * by);
          *(Pack<T, 4>*)(out + e) = z;
        }
    }
  }
}

// The parts of a tile become its rows: with m the largest of the parts' maxima,  O = sum_p 2^(m_p - m) O_p / sum_p 2^(m_p - m) l_p,  in the parts'
// order, so that a call's result does not depend on which workgroup ended first.  A launch of its own, 4 us of one token over 131072 rows, bound by
// the latency of the list and of a part behind it, so parts are read four at a time.  The last workgroup of a tile to end could do
// the same in the same order without that launch, if it saw the parts of the others through the L2s of eight XCDs; not built or measured.
// Of the blockIdx.x-th Left, rows blockIdx.y * per and on, `few` at a time: for each of them the parts are
// shared out over the threads that are left beside four elements each, and joined in LDS.
template <typename T>
__global__ __launch_bounds__(256) void kv_join_k(AttendArgs a, int rows, int per, int few) {
  __shared__ v4f sums[256];
  __shared__ float stat[256][2];
  const int first = blockIdx.y * per, count = *count_of(a, rows);
  const KvLeft t = left_of(a, rows)[blockIdx.x];      // behind the count: whatever the memory held
  if ((int)blockIdx.x >= count || t.pieces <= 1 || first >= t.rows) return;
  const int pieces = t.pieces, there = t.rows, tile = t.tile, h = t.h, w0 = t.w0;
  const int quads = a.c.d / 4, share = 256 / (few * quads), e = threadIdx.x % (few * quads), part = threadIdx.x / (few * quads), c = e % quads;
  for (int r0 = first; r0 < first + per && r0 < there; r0 += few) {
    const int r = r0 + e / quads;
    const bool mine = part < share && r < there;
    float m, l;
    v4f y;
    auto add_parts = [&](auto infinities) INLINE {  // they stay only where that is asked for: it takes as many instructions again
      constexpr int FLY = 4;                          // parts on their way at a time
      m = -INFINITY, l = 0.f;
      y = (v4f){0, 0, 0, 0};
      for (int p = part; mine && p < pieces; p += FLY * share) {
        v4f x[FLY];
        float top[FLY], sum[FLY];
#pragma unroll
        for (int k = 0; k < FLY; k++) {
          const int at = min(p + k * share, pieces - 1);
          const int slot = kv_slot_of(w0, at);
          const float* const st = a.part + kv_stat_at(a.slots, slot, rows, r, a.c.d);
          x[k] = *(const v4f*)(a.part + kv_part_at(slot, rows, r, a.c.d) + c * 4);
          top[k] = p + k * share < pieces ? st[0] : -INFINITY;
          sum[k] = st[1];
        }
        float most = m;
#pragma unroll
        for (int k = 0; k < FLY; k++) most = fmaxf(most, top[k]);
        const float safe = most == -INFINITY ? 0.f : most, by = __builtin_amdgcn_exp2f(m - safe);
        y = infinities ? rescaled(y, by) : y * by;
        l *= by;
        m = most;
#pragma unroll
        for (int k = 0; k < FLY; k++) {
          const float f = __builtin_amdgcn_exp2f(top[k] - safe);
          const bool there = p + k * share < pieces;  // not again what stands in for a part behind the last
          const v4f more = infinities ? rescaled(x[k], f) : x[k] * f;
          l += there ? sum[k] * f : 0.f;
#pragma unroll
          for (int j = 0; j < 4; j++) y[j] += there ? more[j] : 0.f;
        }
      }
    };
    add_parts(std::false_type());
    if (has_nan(y)) add_parts(std::true_type());
    if (r0 > first) __syncthreads();
    sums[threadIdx.x] = y;
    stat[threadIdx.x][0] = m, stat[threadIdx.x][1] = l;
    __syncthreads();
    if (!mine || part) continue;
    float top = m;
    for (int p = 1; p < share; p++) top = fmaxf(top, stat[p * few * quads + e][0]);
    const float safe = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    y = (v4f){0, 0, 0, 0};
    for (int p = 0; p < share; p++) {
      const float f = __builtin_amdgcn_exp2f(stat[p * few * quads + e][0] - safe);
      sum += f * stat[p * few * quads + e][1];
      y += rescaled(sums[p * few * quads + e], f);
    }
    const long long row = (long long)tile * rows + r;
    const KvQuery of = kv_query(row, kv_token(row, a.group), a.group);
    Pack<T, 4> z;
#pragma unroll
    for (int j = 0; j < 4; j++) z.v[j] = from_float<T>(sum == 0.f ? 0.f : y[j] / sum);
    *(Pack<T, 4>*)((T*)(const_cast<char*>(a.out.at) + kv_query_at(t.t0, of, h, a.group, a.out.token, a.out.head)) + c * 4) = z;
  }
}

namespace {
// What the host can see of a call, in the order of the arguments
int attend_args(const pahq_kv_cache* cache, const pahq_kv_batch* batch, int q_heads, AttendArgs* a, KvRange* held, KvRange* lists) {
  if (const int rc = kv_cache_args(cache, &a->c, held)) return rc;
  if (const int rc = kv_batch_args(batch, cache->page_size, &a->b, lists)) return rc;
  if (q_heads < 1 || q_heads % a->c.heads) return PAHQ_EINVAL;
  a->group = q_heads / a->c.heads;
  if (q_heads > 65535 || (long long)batch->tokens * a->group >= KV_MAX_LENGTH || batch->tokens > PAHQ_ROTARY_MAX_TOKENS) return PAHQ_ETOOBIG;
  return PAHQ_OK;
}

KvCut cut_of(const AttendArgs& a, int eb) { return kv_cut(a.b.tokens, a.b.batch, a.group, a.c.heads, a.b.most, a.c.d, eb); }
long long tiles_of(const AttendArgs& a, const KvCut& k) { return kv_call_tiles(a.b.tokens, a.b.batch, a.group, a.c.heads, k.rows); }
size_t part_bytes(const AttendArgs& a, const KvCut& k) { return kv_part_bytes(k.slots, k.rows, a.c.d); }

template <void (*K)(AttendArgs), int THREADS, int LDS>
int launch(hipStream_t st, unsigned grid, const AttendArgs& a) {
  if (LDS > 65536) {
    // more LDS than a launch gets by default: an attribute of the kernel on one device, set once for each
    static std::atomic<bool> set[64];
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return PAHQ_EHIP;
    if (!set[dev].load(std::memory_order_acquire)) {
      if (hipFuncSetAttribute((const void*)K, hipFuncAttributeMaxDynamicSharedMemorySize, LDS) != hipSuccess) return PAHQ_EHIP;
      set[dev].store(true, std::memory_order_release);
    }
  }
  hipLaunchKernelGGL(K, dim3(grid), dim3(THREADS), LDS, st, a);
  return hipGetLastError() == hipSuccess ? PAHQ_OK : PAHQ_EHIP;
}
template <typename T, int D>
int attend_as(hipStream_t st, const AttendArgs& a, const KvCut& k) {
  constexpr int EB = sizeof(T), NW = KvWaves<EB, D>::NW, MANY = KvWaves<EB, D>::MANY;
  const long long tiles = tiles_of(a, k);
  const unsigned grid = (unsigned)std::max<long long>(tiles, k.slots);
  int rc = PAHQ_EHIP;
  if (k.rows == 16) rc = k.waves ? launch<kv_few_k<T, D, 1, MANY>, MANY * 64, KvFew<EB, D, 1, MANY>::LDS>(st, grid, a)
                                 : launch<kv_few_k<T, D, 1, NW>, NW * 64, KvFew<EB, D, 1, NW>::LDS>(st, grid, a);
  if constexpr (D * EB <= 512) {
    if (k.rows == 32) rc = k.waves ? launch<kv_few_k<T, D, 2, MANY>, MANY * 64, KvFew<EB, D, 2, MANY>::LDS>(st, grid, a)
                                   : launch<kv_few_k<T, D, 2, NW>, NW * 64, KvFew<EB, D, 2, NW>::LDS>(st, grid, a);
    if (k.rows == 128) rc = launch<kv_tile_k<T, D, KvWide<EB, D>::KVB>, 256, KvWide<EB, D>::LDS>(st, grid, a);
  }
  if (rc || !k.slots) return rc;
  const KvJoin j = kv_join(tiles, k.slots, k.rows, a.c.d);
  hipLaunchKernelGGL(kv_join_k<T>, dim3(j.left, k.rows / j.per), dim3(256), 0, st, a, k.rows, j.per, j.few);
  return hipGetLastError() == hipSuccess ? PAHQ_OK : PAHQ_EHIP;
}
template <typename T>
int attend_as(hipStream_t st, const AttendArgs& a, const KvCut& k) {
  return a.c.d <= 64 ? attend_as<T, 64>(st, a, k) : a.c.d <= 128 ? attend_as<T, 128>(st, a, k) : attend_as<T, 256>(st, a, k);
}
}  // namespace

}  // namespace pahq

using namespace pahq;

extern "C" int pahq_kv_attention_workspace(const pahq_kv_cache* cache, const pahq_kv_batch* batch, int32_t q_heads, size_t* bytes) {
  AttendArgs a = {};
  KvRange held[2], lists[3];
  if (!bytes) return PAHQ_EINVAL;
  if (const int rc = attend_args(cache, batch, q_heads, &a, held, lists)) return rc;
  *bytes = 0;
  if (a.b.batch == 0 || a.b.tokens == 0) return PAHQ_OK;
  const KvCut cut = cut_of(a, dtype_bytes(cache->dtype));
  if (tiles_of(a, cut) >= KV_MOST_ITEMS) return PAHQ_ETOOBIG;
  *bytes = part_bytes(a, cut);
  return PAHQ_OK;
}

extern "C" int pahq_kv_attention(void* hip_stream, const pahq_kv_cache* cache, const pahq_kv_batch* batch, const pahq_kv_rows* q, int32_t q_heads,
                                 const uint64_t* tree, int32_t words, float scale, const pahq_kv_rows* out, void* workspace, size_t workspace_bytes) {
  AttendArgs a = {};
  KvRange held[2], lists[3], qr, outr;
  if (const int rc = attend_args(cache, batch, q_heads, &a, held, lists)) return rc;
  const float factor = (float)(std::fabs((double)scale) * 1.4426950408889634);        // of the scores, for exp2
  if (words < (tree ? 1 : 0) || (uintptr_t)tree % 8 || !std::isfinite(factor)) return PAHQ_EINVAL;
  if (batch->batch == 0 || batch->tokens == 0) return PAHQ_OK;
  const int eb = dtype_bytes(cache->dtype), tokens = batch->tokens;
  if (!kv_rows_args(q, tokens, q_heads, a.c.d, eb, false, &a.q, &qr) || !kv_rows_args(out, tokens, q_heads, a.c.d, eb, true, &a.out, &outr)) return PAHQ_EINVAL;
  const KvCut cut = cut_of(a, eb);
  if (tiles_of(a, cut) >= KV_MOST_ITEMS) return PAHQ_ETOOBIG;      // workgroups of a launch, whose threads are counted in 32 bits
  const size_t need = part_bytes(a, cut);
  if (need && (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < need)) return PAHQ_EINVAL;
  const KvRange masks = {tree, (size_t)tokens * words * 8}, space = {need ? workspace : nullptr, need};
  const KvRange read[] = {held[0], held[1], lists[0], lists[1], lists[2], masks, space, qr};
  if (kv_meets(&outr, 1, read, 7) || kv_meets(&space, 1, read, 6) || kv_meets(&space, 1, &qr, 1)) return PAHQ_EINVAL;
  const bool in_place = q->at == out->at && q->token == out->token && q->head == out->head;
  if (!in_place && !kv_rows_apart(a.out, outr, q_heads, a.q, qr, q_heads, (size_t)a.c.d * eb)) return PAHQ_EINVAL;
  a.tree = (const unsigned long long*)tree;
  a.words = words;
  a.scale = factor > 0.f ? factor : 1.f;
  a.sign = scale < 0.f ? -1.f : factor > 0.f ? 1.f : 0.f;
  a.part = (float*)workspace;
  a.slots = cut.slots;
  a.least = cut.least;
  a.over = cut.over;
  a.enough = cut.enough;
  a.brief = cut.brief;
  a.by_pair = tiles_of(a, cut) <= cut.slots;
  hipStream_t st = (hipStream_t)hip_stream;
  switch (cache->dtype) {
    case PAHQ_F32: return attend_as<float>(st, a, cut);
    case PAHQ_BF16: return attend_as<bf16_t>(st, a, cut);
    default: return attend_as<f16_t>(st, a, cut);
  }
}
