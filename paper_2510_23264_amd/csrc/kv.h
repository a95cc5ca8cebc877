// What the operators on a paged cache of keys and values share: their operands as kernels take them, the checks of what the host can
// see, and where a sequence's rows lie.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>
#include "../../include/pahq.h"
#include "device_tensor.h"
#include "kv_address.h"

namespace pahq {

struct KvBatch {
  const int *starts, *lengths, *pages;
  long long ld;
  int batch, width, tokens, most;                   // most: rows a list of pages has room for
};
struct KvRows {
  const char* at;
  long long token, head;                            // strides in bytes
};

// ---------------------------------------------------------------- host
// A range of memory, and whether rows of `row` bytes at the strides have a place each (sorted by stride, each behind the extent of the
// ones before); false where no memory is as large.
struct KvRange { const void* at; size_t bytes; };
inline bool kv_distinct(const long long* n, const long long* stride, int dims, long long row) {
  int order[4];
  for (int i = 0; i < dims; i++) {
    int k = i;
    for (; k > 0 && stride[order[k - 1]] > stride[i]; k--) order[k] = order[k - 1];
    order[k] = i;
  }
  long long extent = row;
  for (int i = 0; i < dims; i++) {
    const long long s = stride[order[i]], c = n[order[i]];
    if (c <= 1) continue;
    long long more;
    if (s < extent || __builtin_mul_overflow(s, c - 1, &more) || __builtin_add_overflow(extent, more, &extent) || extent > 1ll << 56) return false;
  }
  return true;
}
inline bool kv_meets(const KvRange* a, int na, const KvRange* b, int nb) {
  for (int i = 0; i < na; i++)
    for (int j = 0; j < nb; j++)
      if (a[i].at && b[j].at && overlap(a[i].at, a[i].bytes, b[j].at, b[j].bytes)) return true;
  return false;
}

// The cache as kernels take it, and its memory as one range; PAHQ_OK or what is wrong
inline int kv_cache_args(const pahq_kv_cache* c, KvCache* a, KvRange* memory) {
  if (!c) return PAHQ_EINVAL;
  const int eb = dtype_bytes(c->dtype);
  if (!eb || c->pages < 1 || c->page_size < 1 || c->heads < 1 || c->d_head < 8 || c->d_head % 8 || c->d_head > PAHQ_KV_MAX_HEAD) return PAHQ_EINVAL;
  if (!c->keys || !c->values || (uintptr_t)c->keys % 16 || (uintptr_t)c->values % 16) return PAHQ_EINVAL;
  if (c->heads > 65535) return PAHQ_ETOOBIG;
  const long long strides[3] = {c->page_stride, c->head_stride, c->slot_stride}, n[3] = {c->pages, c->heads, c->page_size};
  long long s[4], count[4] = {n[0], n[1], n[2], 2};
  for (int i = 0; i < 3; i++) {
    if (strides[i] < 0 || strides[i] > 1ll << 52 || (strides[i] * eb) % 16) return PAHQ_EINVAL;
    s[i] = strides[i] * eb;
  }
  const intptr_t between = (intptr_t)((uintptr_t)c->values - (uintptr_t)c->keys);
  s[3] = between < 0 ? -between : between;
  const long long row = (long long)c->d_head * eb;
  if (!kv_distinct(n, s, 3, row)) return PAHQ_EINVAL;
  size_t bytes = row;
  for (int i = 0; i < 3; i++) bytes += (size_t)(n[i] - 1) * s[i];
  // apart, or side by side in one tensor
  if (overlap(c->keys, bytes, c->values, bytes) && !kv_distinct(count, s, 4, row)) return PAHQ_EINVAL;
  *a = KvCache{(char*)c->keys, (char*)c->values, s[0], s[1], s[2], c->pages, c->page_size, c->heads, c->d_head, 0, 0};
  kv_divider((uint32_t)c->page_size, &a->magic, &a->shift);
  memory[0] = {c->keys, bytes};
  memory[1] = {c->values, bytes};
  return PAHQ_OK;
}
inline int kv_batch_args(const pahq_kv_batch* b, int page_size, KvBatch* a, KvRange* memory) {
  if (!b || b->batch < 0 || b->width < 0 || b->tokens < 0) return PAHQ_EINVAL;
  *a = KvBatch{};
  memory[0] = memory[1] = memory[2] = {nullptr, 0};
  if (b->batch == 0) return PAHQ_OK;
  if (!b->starts || !b->lengths || (uintptr_t)b->starts % 4 || (uintptr_t)b->lengths % 4 || (uintptr_t)b->pages % 4) return PAHQ_EINVAL;
  if (b->batch > PAHQ_KV_MAX_BATCH) return PAHQ_ETOOBIG;
  size_t bytes = 0;
  if (b->width && (!b->pages || b->ld_pages < b->width || !extent(b->batch, b->ld_pages, b->width, 4, &bytes))) return PAHQ_EINVAL;
  const long long room = (long long)b->width * page_size;
  *a = KvBatch{b->starts, b->lengths, b->pages, b->ld_pages, b->batch, b->width, b->tokens, room < KV_MAX_LENGTH ? (int)room : KV_MAX_LENGTH};
  memory[0] = {b->starts, (size_t)(b->batch + 1) * 4};
  memory[1] = {b->lengths, (size_t)b->batch * 4};
  memory[2] = {b->width ? b->pages : nullptr, bytes};
  return PAHQ_OK;
}
// Rows [tokens][heads][d] of `eb` bytes an element; distinct: no two in one place
inline bool kv_rows_args(const pahq_kv_rows* r, int tokens, int heads, int d, int eb, bool distinct, KvRows* a, KvRange* memory) {
  if (!r || !r->at || (uintptr_t)r->at % eb || r->token < 0 || r->head < 0) return false;
  size_t bytes;
  if (!extent(tokens, r->token, heads, r->head, d, eb, &bytes)) return false;
  const long long n[2] = {tokens, heads}, s[2] = {r->token * eb, r->head * eb};
  if (distinct && !kv_distinct(n, s, 2, (long long)d * eb)) return false;
  *a = KvRows{(const char*)r->at, r->token * eb, r->head * eb};
  *memory = {r->at, bytes};
  return true;
}
// Written rows beside read ones: the same rows, other columns of the same rows, or apart
inline bool kv_rows_apart(const KvRows& out, const KvRange& om, int out_heads, const KvRows& in, const KvRange& im, int in_heads, size_t row) {
  if (!overlap(om.at, om.bytes, im.at, im.bytes)) return true;
  return out.token == in.token && side_by_side(out.at, (size_t)(out_heads - 1) * out.head + row, in.at, (size_t)(in_heads - 1) * in.head + row, (size_t)out.token);
}

// ---------------------------------------------------------------- device
__device__ __forceinline__ int kv_start(const KvBatch& q, int b) { return kv_clipped_start(q.starts[b], q.tokens); }
__device__ __forceinline__ KvSequence kv_sequence(const KvBatch& q, int b) {
  return kv_clipped(q.starts[b], q.starts[b + 1], q.lengths[b], q.tokens, q.most);
}
// Where a sequence has outgrown its list of pages its clipped rows are other ones than those it means: nothing is written there
__device__ __forceinline__ bool kv_has_room(const KvBatch& q, int b) { return q.lengths[b] <= q.most; }
// The sequence that token t belongs to: the last b in [0, batch] with start(b) <= t, -1 for none (and `batch` for tokens behind the last).
// Of starts that do not grow any one comes out; the caller checks that t lies in its sequence.
template <typename F> __device__ __forceinline__ int kv_owner(int batch, int t, F start) {
  int lo = -1, hi = batch + 1;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start(mid) <= t) lo = mid;
    else hi = mid;
  }
  return lo;
}
// Bytes from the cache's start to row j < q.most of sequence b in head 0, KV_ROW_NONE where its page is none of the cache's
__device__ __forceinline__ long long kv_row(const KvCache& c, const int* pages, int j) { return kv_row_in(c, j, pages[kv_in_list(c, j)]); }

}  // namespace pahq
