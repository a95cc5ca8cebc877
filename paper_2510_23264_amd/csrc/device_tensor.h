// What the operators on device tensors share: element types, loads and stores of eight neighbouring elements at any
// alignment of the element, and the host's check of memory that two operands share.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>
#include <type_traits>
#include "../../include/pahq.h"

namespace pahq {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

inline int dtype_bytes(int dtype) { return dtype == PAHQ_F32 ? 4 : dtype == PAHQ_BF16 || dtype == PAHQ_F16 ? 2 : 0; }
inline bool overlap(const void* p, size_t pn, const void* q, size_t qn) {
  const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
  return a < b + qn && b < a + pn;
}
// Bytes from the first to the last element of [outer][inner][row], strides in elements; false where no memory is as large (or the
// count passes 64 bits).
inline bool extent(long long outer, long long outer_stride, long long inner, long long inner_stride, long long row, int eb, size_t* bytes) {
  long long a, b;
  if (__builtin_mul_overflow(outer - 1, outer_stride, &a) || __builtin_mul_overflow(inner - 1, inner_stride, &b) || __builtin_add_overflow(a, b, &a) ||
      __builtin_add_overflow(a, row, &a) || a > 1ll << 53)
    return false;
  *bytes = (size_t)a * eb;
  return true;
}
inline bool extent(long long rows, long long stride, long long row, int eb, size_t* bytes) { return extent(rows, stride, 1, 0, row, eb, bytes); }

// Two matrices of rows of pn and qn bytes whose rows lie `stride` bytes apart in both (0: not the same), as columns of one: no row
// of one touches a row of the other.
inline bool side_by_side(const void* p, size_t pn, const void* q, size_t qn, size_t stride) {
  if (stride == 0) return false;
  const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
  const size_t d = b >= a ? (b - a) % stride : (stride - (a - b) % stride) % stride;      // where q's row starts in p's row
  return d >= pn && d + qn <= stride;
}

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(bf16_t x) { return (float)x; }
__device__ __forceinline__ float as_float(f16_t x) { return (float)x; }
// round to nearest, ties to even
template <typename T> __device__ __forceinline__ T from_float(float x) { return (T)x; }

// N elements of an array that is aligned to its element only: one load or store of N * sizeof(T) bytes where the hardware
// has one (global memory takes any alignment).
template <typename T, int N> struct __attribute__((packed, aligned(sizeof(T)))) Pack { T v[N]; };

// elements [0, 8) of p that exist (left of them), the rest zero
template <typename T>
__device__ __forceinline__ void load8(const T* p, int left, float* v) {
  constexpr int N = 16 / sizeof(T);
  if (left >= 8) {
#pragma unroll
    for (int h = 0; h < 8 / N; h++) {
      const Pack<T, N> q = *(const Pack<T, N>*)(p + h * N);
#pragma unroll
      for (int j = 0; j < N; j++) v[h * N + j] = as_float(q.v[j]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; j++) v[j] = j < left ? as_float(p[j]) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int left, const float* v) {
  constexpr int N = 16 / sizeof(T);
  if (left >= 8) {
#pragma unroll
    for (int h = 0; h < 8 / N; h++) {
      Pack<T, N> q;
#pragma unroll
      for (int j = 0; j < N; j++) q.v[j] = from_float<T>(v[h * N + j]);
      *(Pack<T, N>*)(p + h * N) = q;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; j++)
      if (j < left) p[j] = from_float<T>(v[j]);
  }
}

// Sixteen bytes of elements as four registers (an array of 16-bit elements takes one each), at any alignment of the element.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_at_2 __attribute__((ext_vector_type(4), aligned(2)));
template <typename T> __device__ __forceinline__ u32x4 load16(const T* p) { return *(const u32x4_at_2*)p; }
// A store that does not stay in the caches (non-temporal)
template <typename T> __device__ __forceinline__ void store16_nt(T* p, u32x4 v) { __builtin_nontemporal_store((u32x4_at_2)v, (u32x4_at_2*)p); }
template <typename T> __device__ __forceinline__ float element(u32x4 v, int i) {
  if (sizeof(T) == 4) return __uint_as_float(v[i]);
  const uint16_t h = (uint16_t)(v[i / 2] >> (i % 2 * 16));
  return as_float(__builtin_bit_cast(T, (std::conditional_t<sizeof(T) == 2, uint16_t, uint32_t>)h));
}
template <typename T> __device__ __forceinline__ u32x4 pack16(const float* f) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    if (sizeof(T) == 4) v[i] = __float_as_uint(f[i]);
    else {
      typedef T T2 __attribute__((ext_vector_type(2)));
      typedef std::conditional_t<sizeof(T) == 2, uint32_t, uint64_t> W;
      v[i] = (uint32_t)__builtin_bit_cast(W, (T2){from_float<T>(f[2 * i % (16 / sizeof(T))]), from_float<T>(f[(2 * i + 1) % (16 / sizeof(T))])});
    }
  }
  return v;
}

}  // namespace pahq
