// Rotary positions as an operator on device tensors: pairs of elements of every head turn by an angle that grows with the
// token's position (the layouts, the stretched frequencies and the definition are in include/pahq.h).
//
// The angle.  A frequency is kept as the fraction of a turn it advances in one position, in 64 binary digits, so position *
// frequency modulo one turn is one 64-bit integer product, exact at every position; binary32 angles are off by more
// than a hundredth of a radian from position 2^18 on.  The quarter turns come off as the product's two top digits, so
// that what is left, at most an eighth of a turn, loses no more than 2^-25 of that when it becomes a float.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <algorithm>
#include "../../include/pahq.h"
#include "device_tensor.h"

namespace pahq {

struct RotaryArgs {
  long long x_token, x_head, o_token, o_head;       // strides in elements
  const long long* positions;
  const unsigned long long* table;
  int tokens, heads, d, rot;
  int nt, nh;                                       // tokens and heads of a workgroup
  int items;                                        // of a head: groups of V pairs, then of V elements behind the rotated part
  unsigned by_items, by_nh;                         // ceil(2^32 / .): quotients of the small numbers of a workgroup
  float magnitude, direction;
};

// n / d where n * d < 2^32, from ceil(2^32 / d), which does not fit a word for d = 1
__device__ __forceinline__ int quotient(int n, int d, unsigned by_d) { return d == 1 ? n : (int)__umulhi((unsigned)n, by_d); }

// A workgroup takes nt neighbouring tokens and nh heads of each: first the tokens' cosines and sines into LDS, shared by the
// heads, then the heads, V elements of a pair's two sides a thread (V = 1: any alignment and any number of pairs).
// Bound by memory where V elements are 16 bytes: x is read and written once, 8192 tokens of 40 x 128 in bfloat16 34 us at a floor of 33.  V
// divides the pairs and what lies behind them, so other widths go by smaller pieces: 20 of 80 elements, 20000 x 8 in bfloat16, by 4
// bytes, 34 us where the bytes would take 10 (both with x in HBM).
template <typename T, int V, bool HALF>
__global__ __launch_bounds__(256) void rotary_k(const T* x, T* out, RotaryArgs q) {
  extern __shared__ float2 turn[];                  // [nt][rot / 2]
  const int half = q.rot / 2, t0 = blockIdx.x * q.nt, nt = min(q.nt, q.tokens - t0), h0 = blockIdx.y * q.nh, nh = min(q.nh, q.heads - h0);
  for (int e = threadIdx.x; e < nt * half; e += 256) {
    const int t = e / half, i = e - t * half;
    const unsigned long long phase = (unsigned long long)q.positions[t0 + t] * q.table[i] + (1ull << 61);
    const int quarter = (int)(phase >> 62);
    const int left = (int)(((long long)(phase << 2) >> 32) ^ 0x80000000ll);       // in 2^-34 turns, from -1/8 on
    float s, c;
    sincospif((float)left * 1.1641532182693481e-10f, &s, &c);                     // 2^-33: half turns
    const float cq = quarter & 1 ? s : c, sq = quarter & 1 ? c : s;
    turn[e] = make_float2((quarter == 1 || quarter == 2 ? -cq : cq) * q.magnitude, (quarter >= 2 ? -sq : sq) * q.magnitude * q.direction);
  }
  __syncthreads();
  const int pairs = half / V;
  for (int e = threadIdx.x; e < nt * q.nh * q.items; e += 256) {
    const int r = quotient(e, q.items, q.by_items), i = e - r * q.items, t = quotient(r, q.nh, q.by_nh), h = r - t * q.nh;
    if (h >= nh) continue;
    const T* p = x + (t0 + t) * q.x_token + (h0 + h) * q.x_head;
    T* o = out + (t0 + t) * q.o_token + (h0 + h) * q.o_head;
    if (i >= pairs) {
      const int at = q.rot + (i - pairs) * V;
      *(Pack<T, V>*)(o + at) = *(const Pack<T, V>*)(p + at);
      continue;
    }
    const float2* cs = turn + t * half + i * V;
    const int ia = HALF ? i * V : 2 * i * V, ib = HALF ? half + i * V : 2 * i * V + V;
    Pack<T, V> a = *(const Pack<T, V>*)(p + ia), b = *(const Pack<T, V>*)(p + ib);
#pragma unroll
    for (int j = 0; j < V; j++) {
      // half: a holds the first sides of V pairs and b their second sides; interleaved: the 2 V elements of V pairs in turn
      T& u = HALF ? a.v[j] : (2 * j < V ? a.v[2 * j % V] : b.v[2 * j % V]);
      T& w = HALF ? b.v[j] : V == 1 ? b.v[0] : (2 * j < V ? a.v[(2 * j + 1) % V] : b.v[(2 * j + 1) % V]);
      const float f = as_float(u), g = as_float(w);
      u = from_float<T>(f * cs[j].x - g * cs[j].y);
      w = from_float<T>(f * cs[j].y + g * cs[j].x);
    }
    *(Pack<T, V>*)(o + ia) = a;
    *(Pack<T, V>*)(o + ib) = b;
  }
}

namespace {
unsigned reciprocal(int d) { return (unsigned)(((1ull << 32) + d - 1) / d); }

template <typename T, int V, bool HALF>
int launch_rotary(hipStream_t st, const T* x, T* out, RotaryArgs q, bool copy) {
  const int half = q.rot / 2;
  q.items = half / V + (copy ? (q.d - q.rot) / V : 0);
  // Tokens: as many as give every thread a sine, fewer where the chip would not be full; then the heads are split as well,
  // down to a pass of the threads each.  nt nh items <= 2^19 and nh <= 8192 keep the
  // quotients exact.
  q.nt = std::max(1, std::min(std::min(256 / half, 32), q.tokens / 1024));
  const int groups = (q.tokens + q.nt - 1) / q.nt, most = std::min(8192, std::max(1, (1 << 19) / (q.nt * q.items)));
  const int least = std::max(1, 256 / (q.nt * q.items)), split = std::max(1, 1024 / groups);
  q.nh = std::min(std::min(most, q.heads), std::max(least, (q.heads + split - 1) / split));
  q.by_items = reciprocal(q.items);
  q.by_nh = reciprocal(q.nh);
  hipLaunchKernelGGL((rotary_k<T, V, HALF>), dim3(groups, (q.heads + q.nh - 1) / q.nh), dim3(256), (size_t)q.nt * half * sizeof(float2), st, x, out, q);
  return hipGetLastError() == hipSuccess ? PAHQ_OK : PAHQ_EHIP;
}
template <typename T, bool HALF>
int rotary_as(hipStream_t st, const T* x, T* out, const RotaryArgs& q, bool copy) {
  // the most elements an access takes that divide the pairs and what lies behind them
  const int both = (q.rot / 2) | (q.d - q.rot);
  if (sizeof(T) == 2 && both % 8 == 0) return launch_rotary<T, 16 / sizeof(T), HALF>(st, x, out, q, copy);
  if (both % 4 == 0) return launch_rotary<T, 4, HALF>(st, x, out, q, copy);
  if (both % 2 == 0) return launch_rotary<T, 2, HALF>(st, x, out, q, copy);
  return launch_rotary<T, 1, HALF>(st, x, out, q, copy);
}
template <typename T>
int rotary_as(hipStream_t st, const T* x, T* out, const RotaryArgs& q, int layout, bool copy) {
  return layout == PAHQ_ROTARY_HALF ? rotary_as<T, true>(st, x, out, q, copy) : rotary_as<T, false>(st, x, out, q, copy);
}
// [tokens][heads][d] in either order of the first two, no two elements in one place; the strides' products fit (extent was asked)
bool strides_ok(long long tokens, long long heads, long long d, long long st, long long sh) {
  const bool rows = (heads == 1 || sh >= d) && (tokens == 1 || st >= (heads - 1) * sh + d);
  const bool planes = (tokens == 1 || st >= d) && (heads == 1 || sh >= (tokens - 1) * st + d);
  return rows || planes;
}
}  // namespace

}  // namespace pahq

using namespace pahq;

extern "C" int pahq_rotary_table(int32_t rot_dim, double theta, int32_t scaling, double factor, double original, double turns_lo, double turns_hi,
                                 uint64_t* table) {
  if (rot_dim < 2 || (rot_dim & 1) || rot_dim > PAHQ_ROTARY_MAX_DIM || !table) return PAHQ_EINVAL;
  if (!(theta > 0.0) || !isfinite(theta) || scaling < PAHQ_ROTARY_PLAIN || scaling > PAHQ_ROTARY_BANDS) return PAHQ_EINVAL;
  if (scaling != PAHQ_ROTARY_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return PAHQ_EINVAL;
  if (scaling == PAHQ_ROTARY_BASE && rot_dim < 4) return PAHQ_EINVAL;
  if (scaling == PAHQ_ROTARY_BANDS && (!(original > 0.0) || !isfinite(original) || !(turns_lo >= 0.0) || !(turns_hi > turns_lo) || !isfinite(turns_hi))) return PAHQ_EINVAL;
  const long double tau = 6.283185307179586476925286766559005768L;
  long double base = theta;
  if (scaling == PAHQ_ROTARY_BASE) base *= powl(factor, (long double)rot_dim / (rot_dim - 2));
  for (int i = 0; i < rot_dim / 2; i++) {
    long double f = powl(base, -2.0L * i / rot_dim) / tau;             // turns a position
    if (scaling == PAHQ_ROTARY_LINEAR) f /= factor;
    if (scaling == PAHQ_ROTARY_BANDS) {
      const long double g = fminl(1.0L, fmaxl(0.0L, (f * original - turns_lo) / (turns_hi - turns_lo)));
      f *= g + (1.0L - g) / factor;
    }
    if (!isfinite(f)) return PAHQ_EINVAL;
    // whole turns drop out; 2^64 itself (a fraction that rounds up to one) is no turn
    const long double scaled = roundl((f - floorl(f)) * 18446744073709551616.0L);
    table[i] = scaled >= 18446744073709551616.0L ? 0ull : (uint64_t)scaled;
  }
  return PAHQ_OK;
}

extern "C" int pahq_rotary(void* hip_stream, const void* x, int32_t dtype, int32_t tokens, int32_t heads, int32_t d_head, int64_t x_token, int64_t x_head,
                           const int64_t* positions, const uint64_t* table, int32_t rot_dim, int32_t layout, float magnitude, int32_t inverse, void* out,
                           int64_t out_token, int64_t out_head) {
  const int eb = dtype_bytes(dtype);
  if (tokens < 0 || heads < 0 || d_head < 1 || !eb || rot_dim < 2 || (rot_dim & 1) || rot_dim > d_head || rot_dim > PAHQ_ROTARY_MAX_DIM) return PAHQ_EINVAL;
  if ((layout != PAHQ_ROTARY_HALF && layout != PAHQ_ROTARY_INTERLEAVED) || (inverse != 0 && inverse != 1)) return PAHQ_EINVAL;
  if (tokens == 0 || heads == 0) return PAHQ_OK;
  if (!x || !out || !positions || !table || (uintptr_t)x % eb || (uintptr_t)out % eb || (uintptr_t)positions % 8 || (uintptr_t)table % 8) return PAHQ_EINVAL;
  // workgroups are counted in 16 bits along the heads, threads in 32 along the tokens
  if (heads > 65535 || d_head > PAHQ_ROTARY_MAX_HEAD || tokens > PAHQ_ROTARY_MAX_TOKENS) return PAHQ_ETOOBIG;
  size_t xb, ob;                                                        // x is only read: its rows may share memory
  if (x_token < 0 || x_head < 0 || out_token < 0 || out_head < 0 || !extent(tokens, x_token, heads, x_head, d_head, eb, &xb) ||
      !extent(tokens, out_token, heads, out_head, d_head, eb, &ob) || !strides_ok(tokens, heads, d_head, out_token, out_head))
    return PAHQ_EINVAL;
  const bool in_place = x == out && x_token == out_token && x_head == out_head;
  const size_t xw = (size_t)((heads - 1ll) * x_head + d_head) * eb, ow = (size_t)((heads - 1ll) * out_head + d_head) * eb;      // of a token
  if (!in_place && overlap(x, xb, out, ob) && !side_by_side(x, xw, out, ow, x_token == out_token ? (size_t)x_token * eb : 0))
    return PAHQ_EINVAL;
  if (overlap(out, ob, positions, (size_t)tokens * 8) || overlap(out, ob, table, (size_t)rot_dim * 4)) return PAHQ_EINVAL;
  hipStream_t st = (hipStream_t)hip_stream;
  const RotaryArgs q = {x_token, x_head, out_token, out_head, (const long long*)positions, (const unsigned long long*)table, tokens, heads, d_head, rot_dim,
                        0, 0, 0, 0, 0, magnitude, inverse ? -1.f : 1.f};
  switch (dtype) {
    case PAHQ_F32: return rotary_as(st, (const float*)x, (float*)out, q, layout, !in_place);
    case PAHQ_BF16: return rotary_as(st, (const bf16_t*)x, (bf16_t*)out, q, layout, !in_place);
    default: return rotary_as(st, (const f16_t*)x, (f16_t*)out, q, layout, !in_place);
  }
}
