// Attention of new tokens over a paged cache (the definition is in include/pahq.h).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <algorithm>
#include "../../include/pahq.h"
#include "device_util.h"
#include "kv.h"

namespace pahq {

struct AttendArgs {
  KvCache c;
  KvBatch b;
  KvRows q, out;
  const unsigned long long* tree;
  int words, group;                                 // group: query heads of a cache head
  float scale;                                      // times log2 e
};

// A workgroup takes a query head of a token, a wave every fourth row it sees, each with a running maximum and sum; the
// four meet in LDS.
template <typename T>
__global__ __launch_bounds__(256) void kv_attend_k(AttendArgs a) {
  __shared__ float part[4][PAHQ_KV_MAX_HEAD + 2];
  const int t = blockIdx.x, h = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d = a.c.d;
  const int b = kv_owner(a.b.batch, t, [&](int i) { return kv_start(a.b, i); });
  if (b < 0 || b >= a.b.batch) return;
  const KvSequence s = kv_sequence(a.b, b);
  if (t >= s.t0 + s.n) return;
  const T* const q = (const T*)(a.q.at + t * a.q.token + h * a.q.head);
  const long long head = (long long)(h / a.group) * a.c.head;
  float x[4], o[4] = {0, 0, 0, 0}, m = -INFINITY, l = 0.f;
  for (int e = 0; e < 4; e++) x[e] = lane * 4 + e < d ? as_float(q[lane * 4 + e]) : 0.f;
  for (int j = wave; j < s.length; j += 4) {
    const int ahead = j - s.base;
    if (ahead >= 0) {
      if (!a.tree && ahead > t - s.t0) break;
      if (a.tree && (ahead >= 64ll * a.words || !(a.tree[(long long)t * a.words + ahead / 64] >> (ahead & 63) & 1))) continue;
    }
    const long long row = kv_row(a.c, a.b.pages + b * a.b.ld, j);
    float y = 0.f, v[4] = {0, 0, 0, 0};
    for (int e = 0; e < 4; e++)
      if (lane * 4 + e < d) {
        y += row < 0 ? NAN : x[e] * as_float(((const T*)(a.c.keys + row + head))[lane * 4 + e]);
        v[e] = row < 0 ? NAN : as_float(((const T*)(a.c.values + row + head))[lane * 4 + e]);
      }
    y = wave_sum(y) * a.scale;
    const float top = fmaxf(m, y);
    if (top == -INFINITY && y == y) continue;       // nothing so far weighs anything
    const float keep = exp2f(m - top), p = exp2f(y - top);
    m = top;
    l = l * keep + p;
    for (int e = 0; e < 4; e++) o[e] = o[e] * keep + p * v[e];
  }
  for (int e = 0; e < 4; e++) part[wave][lane * 4 + e] = o[e];
  if (lane == 0) part[wave][PAHQ_KV_MAX_HEAD] = m, part[wave][PAHQ_KV_MAX_HEAD + 1] = l;
  __syncthreads();
  float top = -INFINITY, sum = 0.f, y = 0.f;
  for (int w = 0; w < 4; w++) top = fmaxf(top, part[w][PAHQ_KV_MAX_HEAD]);
  if (top == -INFINITY) top = 0.f;
  for (int w = 0; w < 4; w++) {
    const float f = exp2f(part[w][PAHQ_KV_MAX_HEAD] - top);
    sum += f * part[w][PAHQ_KV_MAX_HEAD + 1];
    y += f * part[w][threadIdx.x];
  }
  if ((int)threadIdx.x < d) ((T*)(a.out.at + t * a.out.token + h * a.out.head))[threadIdx.x] = from_float<T>(sum == 0.f ? 0.f : y / sum);
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
}  // namespace

}  // namespace pahq

using namespace pahq;

extern "C" int pahq_kv_attention_workspace(const pahq_kv_cache* cache, const pahq_kv_batch* batch, int32_t q_heads, size_t* bytes) {
  AttendArgs a = {};
  KvRange held[2], lists[3];
  if (!bytes) return PAHQ_EINVAL;
  if (const int rc = attend_args(cache, batch, q_heads, &a, held, lists)) return rc;
  *bytes = 0;
  return PAHQ_OK;
}

extern "C" int pahq_kv_attention(void* hip_stream, const pahq_kv_cache* cache, const pahq_kv_batch* batch, const pahq_kv_rows* q, int32_t q_heads,
                                 const uint64_t* tree, int32_t words, float scale, const pahq_kv_rows* out, void* workspace, size_t workspace_bytes) {
  AttendArgs a = {};
  KvRange held[2], lists[3], qr, outr;
  if (const int rc = attend_args(cache, batch, q_heads, &a, held, lists)) return rc;
  if (words < (tree ? 1 : 0) || (uintptr_t)tree % 8) return PAHQ_EINVAL;
  if (batch->batch == 0 || batch->tokens == 0) return PAHQ_OK;
  const int eb = dtype_bytes(cache->dtype), tokens = batch->tokens;
  if (!kv_rows_args(q, tokens, q_heads, a.c.d, eb, false, &a.q, &qr) || !kv_rows_args(out, tokens, q_heads, a.c.d, eb, true, &a.out, &outr)) return PAHQ_EINVAL;
  const KvRange masks = {tree, (size_t)tokens * words * 8}, space = {workspace, workspace_bytes};
  const KvRange read[] = {held[0], held[1], lists[0], lists[1], lists[2], masks, space, qr};
  if (kv_meets(&outr, 1, read, 7) || (workspace_bytes && kv_meets(&space, 1, read, 6)) || (workspace_bytes && kv_meets(&space, 1, &qr, 1))) return PAHQ_EINVAL;
  const bool in_place = q->at == out->at && q->token == out->token && q->head == out->head;
  if (!in_place && !kv_rows_apart(a.out, outr, q_heads, a.q, qr, q_heads, (size_t)a.c.d * eb)) return PAHQ_EINVAL;
  a.tree = (const unsigned long long*)tree;
  a.words = words;
  a.scale = (float)(scale * 1.4426950408889634);
  const dim3 grid(tokens, q_heads);
  hipStream_t st = (hipStream_t)hip_stream;
  switch (cache->dtype) {
    case PAHQ_F32: hipLaunchKernelGGL(kv_attend_k<float>, grid, dim3(256), 0, st, a); break;
    case PAHQ_BF16: hipLaunchKernelGGL(kv_attend_k<bf16_t>, grid, dim3(256), 0, st, a); break;
    default: hipLaunchKernelGGL(kv_attend_k<f16_t>, grid, dim3(256), 0, st, a);
  }
  return hipGetLastError() == hipSuccess ? PAHQ_OK : PAHQ_EHIP;
}
