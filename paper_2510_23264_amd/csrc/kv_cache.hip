// Filling and tidying a paged cache of keys and values (the layout and the definitions are in include/pahq.h).
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <algorithm>
#include "../../include/pahq.h"
#include "kv.h"
#include "rotary_turn.h"

namespace pahq {

struct AppendArgs {
  KvCache c;
  KvBatch b;
  KvRows k, v, q, out;
  const long long* positions;
  const unsigned long long* table;
  float magnitude;
  int rot, q_heads, nt;                             // nt: tokens of a workgroup
};

// Keys and queries: pair i of a token at position p becomes (f cos - g sin, f sin + g cos) at p times the table's i-th frequency, in fp32, rounded
// once.  Bound by memory: each element is read and written once, the cosines and sines are made once for a token and not for each of its heads.
// A workgroup takes nt neighbouring tokens: their places and their cosines and sines into LDS, then the heads: of keys and queries an
// item is V pairs (the last one of a head fewer) or V elements behind them, of values V elements: 16 bytes a read and write.
// Measured: 8192 tokens, bf16, 8 heads of 128 columns for 32 of queries, 201 MB, 47 us (4.3 TB/s, a copy reaches 5.1); 4 tokens 5.1 us, which is
// the launch and the reads of the lists that wait for one another.
template <typename T, bool HALF>
__global__ __launch_bounds__(256) void kv_append_k(AppendArgs a) {
  constexpr int V = 16 / sizeof(T), MOST = 32;
  extern __shared__ float2 turn[];                  // [nt][rot / 2]
  __shared__ long long place[MOST];
  __shared__ int at_row[MOST];
  const int half = a.rot / 2, t0 = blockIdx.x * a.nt, nt = min(a.nt, a.b.tokens - t0);
  if ((int)threadIdx.x < nt) {
    const int t = t0 + threadIdx.x, b = kv_owner(a.b.batch, t, [&](int i) { return kv_start(a.b, i); });
    long long p = -2;                               // no sequence's: nothing is written, not the query either
    if (b >= 0 && b < a.b.batch) {
      const KvSequence s = kv_sequence(a.b, b);
      if (t < s.t0 + s.n) {
        const int row = s.base + (t - s.t0);
        p = row >= 0 && kv_has_room(a.b, b) ? kv_row(a.c, a.b.pages + b * a.b.ld, row) : -1;
        at_row[threadIdx.x] = row;
      }
    }
    place[threadIdx.x] = p;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < nt * half; e += 256) {
    const int t = e / half, i = e - t * half;
    if (place[t] == -2) continue;
    turn[e] = rotary_turn(a.positions ? a.positions[t0 + t] : at_row[t], a.table[i], a.magnitude, 1.f);
  }
  __syncthreads();
  const int pairs = (half + V - 1) / V, turned = pairs + (a.c.d - a.rot + V - 1) / V, copied = a.c.d / V;
  const int q_items = a.q_heads * turned, k_items = a.c.heads * turned, items = q_items + k_items + a.c.heads * copied;
  for (int t = 0; t < nt; t++) {
    const long long p = place[t];
    if (p == -2) continue;
    for (int e = threadIdx.x; e < items; e += 256) {
      if (e >= q_items && p < 0) break;
      if (e >= q_items + k_items) {
        const int r = e - q_items - k_items, h = r / copied, i = r - h * copied;
        const Pack<T, V> x = *(const Pack<T, V>*)(a.v.at + (t0 + t) * a.v.token + h * a.v.head + i * 16);
        *(Pack<T, V>*)(a.c.values + p + h * a.c.head + i * 16) = x;
        continue;
      }
      const bool query = e < q_items;
      const int r = query ? e : e - q_items, h = r / turned, i = r - h * turned;
      const T* const x = (const T*)(query ? a.q.at + (t0 + t) * a.q.token + h * a.q.head : a.k.at + (t0 + t) * a.k.token + h * a.k.head);
      T* const y = (T*)(query ? const_cast<char*>(a.out.at) + (t0 + t) * a.out.token + h * a.out.head : a.c.keys + p + h * a.c.head);
      if (i >= pairs) {
        const int from = a.rot + (i - pairs) * V;
        if (from + V <= a.c.d) *(Pack<T, V>*)(y + from) = *(const Pack<T, V>*)(x + from);
        else
          for (int j = from; j < a.c.d; j++) y[j] = x[j];
        continue;
      }
      const float2* const cs = turn + t * half + i * V;
      if (i * V + V <= half) {
        const int ia = HALF ? i * V : 2 * i * V, ib = HALF ? half + i * V : 2 * i * V + V;
        Pack<T, V> u = *(const Pack<T, V>*)(x + ia), w = *(const Pack<T, V>*)(x + ib);
#pragma unroll
        for (int j = 0; j < V; j++) {
          T& m = HALF ? u.v[j] : (2 * j < V ? u.v[2 * j % V] : w.v[2 * j % V]);
          T& n = HALF ? w.v[j] : (2 * j < V ? u.v[(2 * j + 1) % V] : w.v[(2 * j + 1) % V]);
          const float f = as_float(m), g = as_float(n);
          m = from_float<T>(f * cs[j].x - g * cs[j].y);
          n = from_float<T>(f * cs[j].y + g * cs[j].x);
        }
        *(Pack<T, V>*)(y + ia) = u;
        *(Pack<T, V>*)(y + ib) = w;
      } else {
        for (int j = 0; i * V + j < half; j++) {
          const int ia = HALF ? i * V + j : 2 * (i * V + j), ib = HALF ? ia + half : ia + 1;
          const float f = as_float(x[ia]), g = as_float(x[ib]);
          y[ia] = from_float<T>(f * cs[j].x - g * cs[j].y);
          y[ib] = from_float<T>(f * cs[j].y + g * cs[j].x);
        }
      }
    }
  }
}

// A workgroup takes a head of a sequence, as many path nodes at a time as its threads hold 16 bytes of: it reads their rows, waits and
// writes.  Sources grow and lie at or behind their targets, so no later read finds a row that an earlier step wrote.
// A copy of little; measured: 192 sequences, up to 8 of 64 nodes, fp16, 12 heads of 64 columns 5 us, at most 9 MB: the launch and the reads of lists, paths
// and pages' numbers, which wait for one another.
__global__ __launch_bounds__(256) void kv_keep_k(KvCache c, KvBatch q, const int* paths, int depth, int row_bytes, int* new_lengths) {
  __shared__ int stay;
  const int b = blockIdx.x, h = blockIdx.y;
  const KvSequence s = kv_sequence(q, b);
  const int* const path = paths + (long long)b * depth;
  if (threadIdx.x < 64) {
    int n = 0;
    for (int i0 = 0; i0 < depth; i0 += 64) {
      const int i = i0 + threadIdx.x;
      const bool ok = i < depth && path[i] > (i ? path[i - 1] : -1) && path[i] < s.n;
      const unsigned long long bad = ~__ballot(ok);
      n += bad ? __builtin_ctzll(bad) : 64;
      if (bad) break;
    }
    if (threadIdx.x == 0) {
      stay = n;
      if (h == 0) new_lengths[b] = s.base + n;
    }
  }
  __syncthreads();
  const int chunks = row_bytes / 16, step = 256 / chunks, mine = threadIdx.x / chunks, at = (threadIdx.x - mine * chunks) * 16, n = kv_has_room(q, b) ? stay : 0;
  const int* const pages = q.pages + b * q.ld;
  for (int i0 = 0; i0 < n; i0 += step) {
    const int i = i0 + mine;
    long long to = -1;
    uint4 k, v;
    if (mine < step && i < n) {
      const long long from = path[i] == i || s.base + path[i] < 0 ? -1 : kv_row(c, pages, s.base + path[i]);
      if (from >= 0) {
        to = s.base + i < 0 ? -1 : kv_row(c, pages, s.base + i);
        k = *(const uint4*)(c.keys + from + h * c.head + at);
        v = *(const uint4*)(c.values + from + h * c.head + at);
      }
    }
    __syncthreads();
    if (to >= 0) {
      *(uint4*)(c.keys + to + h * c.head + at) = k;
      *(uint4*)(c.values + to + h * c.head + at) = v;
    }
  }
}

namespace {
template <typename T>
int append_as(hipStream_t st, AppendArgs a, int layout) {
  // tokens of a workgroup: as many as give every thread a sine, fewer where the chip would not be full (four workgroups for each compute unit)
  a.nt = std::max(1, std::min(std::min(a.rot ? 512 / a.rot : 32, 32), a.b.tokens / 1024));
  const dim3 grid((a.b.tokens + a.nt - 1) / a.nt);
  const size_t lds = (size_t)a.nt * (a.rot / 2) * sizeof(float2);
  if (layout == PAHQ_ROTARY_HALF) hipLaunchKernelGGL((kv_append_k<T, true>), grid, dim3(256), lds, st, a);
  else hipLaunchKernelGGL((kv_append_k<T, false>), grid, dim3(256), lds, st, a);
  return hipGetLastError() == hipSuccess ? PAHQ_OK : PAHQ_EHIP;
}
}  // namespace

}  // namespace pahq

using namespace pahq;

extern "C" int pahq_kv_append(void* hip_stream, const pahq_kv_cache* cache, const pahq_kv_batch* batch, const pahq_kv_rows* k, const pahq_kv_rows* v,
                              const int64_t* positions, const uint64_t* table, int32_t rot_dim, int32_t layout, float magnitude, const pahq_kv_rows* q,
                              int32_t q_heads, const pahq_kv_rows* out) {
  AppendArgs a = {};
  KvRange held[2], lists[3], kr, vr, qr = {}, outr = {};
  if (const int rc = kv_cache_args(cache, &a.c, held)) return rc;
  if (const int rc = kv_batch_args(batch, cache->page_size, &a.b, lists)) return rc;
  const int eb = dtype_bytes(cache->dtype), d = a.c.d;
  if (!q != !out || (q && q_heads < 1) || (layout != PAHQ_ROTARY_HALF && layout != PAHQ_ROTARY_INTERLEAVED)) return PAHQ_EINVAL;
  if (table && (rot_dim < 2 || (rot_dim & 1) || rot_dim > d)) return PAHQ_EINVAL;
  if (batch->batch == 0 || batch->tokens == 0) return PAHQ_OK;
  if ((q && q_heads > 65535) || batch->tokens > PAHQ_ROTARY_MAX_TOKENS) return PAHQ_ETOOBIG;
  if (!kv_rows_args(k, a.b.tokens, a.c.heads, d, eb, false, &a.k, &kr) || !kv_rows_args(v, a.b.tokens, a.c.heads, d, eb, false, &a.v, &vr)) return PAHQ_EINVAL;
  if (q && (!kv_rows_args(q, a.b.tokens, q_heads, d, eb, false, &a.q, &qr) || !kv_rows_args(out, a.b.tokens, q_heads, d, eb, true, &a.out, &outr)))
    return PAHQ_EINVAL;
  if ((uintptr_t)positions % 8 || (uintptr_t)table % 8) return PAHQ_EINVAL;
  const KvRange read[] = {kr, vr, qr, outr, lists[0], lists[1], lists[2], {positions, (size_t)a.b.tokens * 8}, {table, (size_t)rot_dim * 4}};
  if (kv_meets(held, 2, read, table ? 9 : 8) || kv_meets(&outr, 1, read + 4, table ? 5 : 4)) return PAHQ_EINVAL;
  if (q) {
    const bool in_place = q->at == out->at && q->token == out->token && q->head == out->head;
    const size_t row = (size_t)d * eb;
    if ((!in_place && !kv_rows_apart(a.out, outr, q_heads, a.q, qr, q_heads, row)) || !kv_rows_apart(a.out, outr, q_heads, a.k, kr, a.c.heads, row) ||
        !kv_rows_apart(a.out, outr, q_heads, a.v, vr, a.c.heads, row))
      return PAHQ_EINVAL;
    a.q_heads = q_heads;
  }
  a.positions = (const long long*)positions;
  a.table = (const unsigned long long*)table;
  a.rot = table ? rot_dim : 0;
  a.magnitude = magnitude;
  hipStream_t st = (hipStream_t)hip_stream;
  switch (cache->dtype) {
    case PAHQ_F32: return append_as<float>(st, a, layout);
    case PAHQ_BF16: return append_as<bf16_t>(st, a, layout);
    default: return append_as<f16_t>(st, a, layout);
  }
}

extern "C" int pahq_kv_keep(void* hip_stream, const pahq_kv_cache* cache, const pahq_kv_batch* batch, const int32_t* paths, int32_t depth, int32_t* new_lengths) {
  KvCache c;
  KvBatch q;
  KvRange held[2], lists[3];
  if (const int rc = kv_cache_args(cache, &c, held)) return rc;
  if (const int rc = kv_batch_args(batch, cache->page_size, &q, lists)) return rc;
  if (depth < 0) return PAHQ_EINVAL;
  if (q.batch == 0) return PAHQ_OK;
  if ((depth && !paths) || !new_lengths || (uintptr_t)paths % 4 || (uintptr_t)new_lengths % 4) return PAHQ_EINVAL;
  const KvRange written[3] = {held[0], held[1], {new_lengths, (size_t)q.batch * 4}};
  const KvRange read[4] = {lists[0], lists[1], lists[2], {depth ? paths : nullptr, (size_t)q.batch * depth * 4}};
  if (kv_meets(written, 3, read, 4) || kv_meets(held, 2, written + 2, 1)) return PAHQ_EINVAL;
  hipLaunchKernelGGL(kv_keep_k, dim3(q.batch, c.heads), dim3(256), 0, (hipStream_t)hip_stream, c, q, paths, depth, c.d * dtype_bytes(cache->dtype), new_lengths);
  return hipGetLastError() == hipSuccess ? PAHQ_OK : PAHQ_EHIP;
}

extern "C" int pahq_tree_bits(const int32_t* parents, int32_t n, uint64_t* bits) {
  if (n < 0 || (n && (!parents || !bits))) return PAHQ_EINVAL;
  for (int i = 0; i < n; i++)
    if (parents[i] < -1 || parents[i] >= i) return PAHQ_EINVAL;
  const size_t words = ((size_t)n + 63) / 64;
  for (int i = 0; i < n; i++) {
    uint64_t* const row = bits + i * words;
    for (size_t w = 0; w < words; w++) row[w] = parents[i] < 0 ? 0 : bits[parents[i] * words + w];
    row[i / 64] |= 1ull << (i % 64);
  }
  return PAHQ_OK;
}
