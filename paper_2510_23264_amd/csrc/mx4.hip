// Rows in 4 microscaled bits as operators on device tensors: E2M1 codes with one power-of-two scale per 32
// elements (the layout and the definition are in include/pahq.h), and the product of two such matrices on the
// matrix instruction that takes them as they are (V_MFMA_SCALE_F32_16X16X128_F8F6F4).
//
// Why the instruction may be used directly, where the E4M3 products of the engine go through fp16: the products of
// two E2M1 values are multiples of 1/4 up to 36, and the instruction's sums of 128 of them, under scales up to 2^12
// apart and with an accumulator up to 10^4 times as large, came out within 2^-22 of sum |a w|: what binary32
// additions in any order leave.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <atomic>
#include "../../include/pahq.h"
#include "mma_util.h"
#include "device_tensor.h"

namespace pahq {

// ---------------------------------------------------------------- quantiser
// Eight neighbouring elements a lane, so that four lanes hold a block and its maximum takes two exchanges.  The
// maximum is taken over the bit patterns without sign, which order finite values, infinity and NaN in this order.
__device__ __forceinline__ uint32_t mx4_scale_of(uint32_t top) {
  if (top >= 0x7F800000u) return 255u;                      // not finite: the scale's NaN
  if (top == 0u) return 127u;
  const int e = (int)(top >> 23) - 2;                       // subnormals have exponent field 0: the smallest scale
  return e > 0 ? (uint32_t)e : 0u;
}
// 2^-s as a float: a product with it is exact, and what falls below the normal range rounds to code 0 anyway
__device__ __forceinline__ float mx4_inverse(uint32_t scale) { return __uint_as_float((254u - scale) << 23); }

// Codes of eight scaled values, the first in the low nibble.  The conversion rounds to nearest, ties to the even code,
// and saturates at 6 (checked on gfx950 at every border and between).
__device__ __forceinline__ uint32_t mx4_encode8(const float* v, float inv) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0] * inv, v[1] * inv, 1.0f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2] * inv, v[3] * inv, 1.0f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4] * inv, v[5] * inv, 1.0f, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6] * inv, v[7] * inv, 1.0f, 3);
  return w;
}

// A workgroup takes 8 groups of 256 elements at a time, half a wave each.
template <typename T>
__global__ __launch_bounds__(256) void mx4_rows_quant_k(const T* x, long long ld, int rows, int cols, int groups, uint32_t* codes, uint8_t* scales) {
  const int l = threadIdx.x & 31;
  const uint32_t units = (uint32_t)rows * (uint32_t)groups;
  const uint32_t u = blockIdx.x * 8u + (threadIdx.x >> 5);
  if (u >= units) return;                                    // whole halves of a wave: exchanges stay inside four lanes
  const uint32_t row = u / (uint32_t)groups, g = u - row * (uint32_t)groups;
  const int c0 = (int)g * 256 + l * 8;
  float v[8];
  load8(x + (long long)row * ld + c0, cols - c0, v);
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; j++) top = max(top, __float_as_uint(v[j]) & 0x7FFFFFFFu);
  top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
  const uint32_t s = mx4_scale_of(top);
  codes[(long long)u * 32 + l] = s == 255u ? 0u : mx4_encode8(v, mx4_inverse(s));
  if ((l & 3) == 0) scales[(long long)u * 8 + (l >> 2)] = (uint8_t)s;
}

// x [cols][rows] (the masters' layout [k][n]): one thread holds a block of 32 down a column, neighbouring threads
// neighbouring columns.  Workgroup: 64 columns, 128 elements of each.
template <typename T>
__global__ __launch_bounds__(256) void mx4_cols_quant_k(const T* x, long long ld, int rows, int cols, int blocks, uint8_t* codes, uint8_t* scales) {
  const int row = blockIdx.x * 64 + (threadIdx.x & 63), b = blockIdx.y * 4 + (threadIdx.x >> 6);
  if (row >= rows) return;
  float v[32];
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 32; j++) {
    const int k = b * 32 + j;
    v[j] = k < cols ? as_float(x[(long long)k * ld + row]) : 0.f;
    top = max(top, __float_as_uint(v[j]) & 0x7FFFFFFFu);
  }
  const uint32_t s = mx4_scale_of(top);
  uint4 w = make_uint4(0, 0, 0, 0);
  if (s != 255u) {
    const float inv = mx4_inverse(s);
    w = make_uint4(mx4_encode8(v, inv), mx4_encode8(v + 8, inv), mx4_encode8(v + 16, inv), mx4_encode8(v + 24, inv));
  }
  *(uint4*)(codes + ((long long)row * blocks + b) * 16) = w;
  scales[(long long)row * blocks + b] = (uint8_t)s;
}

// ---------------------------------------------------------------- values
// code * 2^s: one mantissa bit, so exact in binary32 and bfloat16 down to the smallest scale (2^-128 is subnormal in
// both); fp16 rounds once, and goes to infinity or zero where its range ends.
__device__ __forceinline__ float mx4_scale_value(uint32_t s) {
  return __uint_as_float(s == 0u ? 0x00400000u : s == 255u ? 0x7FC00000u : s << 23);
}
template <typename T>
__global__ __launch_bounds__(256) void mx4_values_k(const uint32_t* codes, const uint8_t* scales, int rows, int cols, int groups, T* out, long long ld) {
  const int l = threadIdx.x & 31;
  const uint32_t u = blockIdx.x * 8u + (threadIdx.x >> 5);
  if (u >= (uint32_t)rows * (uint32_t)groups) return;
  const uint32_t row = u / (uint32_t)groups, g = u - row * (uint32_t)groups;
  const int c0 = (int)g * 256 + l * 8;
  if (c0 >= cols) return;
  const uint32_t w = codes[(long long)u * 32 + l];
  const float s = mx4_scale_value(scales[(long long)u * 8 + (l >> 2)]);
  typedef float v2f __attribute__((ext_vector_type(2)));
  const v2f p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
  const v2f p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
  const float v[8] = {p0[0] * s, p0[1] * s, p1[0] * s, p1[1] * s, p2[0] * s, p2[1] * s, p3[0] * s, p3[1] * s};
  store8(out + (long long)row * ld + c0, cols - c0, v);
}

// ---------------------------------------------------------------- product
typedef float v16f __attribute__((ext_vector_type(16)));
template <int N> struct Int { static constexpr int value = N; };

// Tile of a workgroup: the eight XCDs take neighbouring ranges of the tiles, which run down bands of eight rows of tiles, so
// that what an XCD works on at a time shares operands in its L2.  tm >= mt: no tile (the ranges are rounded up).
__device__ __forceinline__ void tile_of(int wg, int mt, int nt, int& tm, int& tn) {
  const int t = xcd_tile(wg, mt * nt);
  if (t >= mt * nt) { tm = mt; tn = 0; return; }
  const int band = t / (8 * nt), in = t - band * 8 * nt, high = min(8, mt - band * 8);
  tn = in / high;
  tm = band * 8 + in - tn * high;
}

// Few rows: 16 * MT rows x 16 columns a workgroup, the sum over k split over its waves (slab s of 256 elements to wave s
// mod WAVES) and joined in LDS in the order of the waves, so results do not depend on timing.  Operands come straight from
// global memory: a lane reads two neighbouring blocks of its row with their scales, which are one halfword, and the four
// lanes of a row take 128 contiguous bytes.  Which 32 elements of the slab a lane's block is does not matter to the sum as
// long as both operands agree.  Rows and columns past the end read the last one and are not stored.
template <typename T, int MT, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void mx4_gemm_few_k(const uint8_t* a, const uint8_t* as, const uint8_t* w, const uint8_t* ws, int m, int n,
                                                            int slabs, const float* bias, const T* res, long long ld_res, T* out, long long ld) {
  __shared__ float part[WAVES][MT * 16][17];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * (16 * MT);
  const long long row_bytes = (long long)slabs * 128;
  const long long wr = min(n0 + r, n - 1);
  const uint8_t* wp = w + wr * row_bytes + g * 32;
  const uint8_t* wsp = ws + wr * slabs * 8 + g * 2;
  const uint8_t* ap[MT];
  const uint8_t* asp[MT];
#pragma unroll
  for (int t = 0; t < MT; t++) {
    const long long ar = min(m0 + t * 16 + r, m - 1);
    ap[t] = a + ar * row_bytes + g * 32;
    asp[t] = as + ar * slabs * 8 + g * 2;
  }
  v4f acc[MT];
#pragma unroll
  for (int t = 0; t < MT; t++) acc[t] = (v4f){0.f, 0.f, 0.f, 0.f};
  for (int s = wave; s < slabs; s += WAVES) {
    const int4 w0 = *(const int4*)(wp + (long long)s * 128), w1 = *(const int4*)(wp + (long long)s * 128 + 16);
    const int wsc = *(const uint16_t*)(wsp + (long long)s * 8);
    const v8i b0 = {w0.x, w0.y, w0.z, w0.w, 0, 0, 0, 0}, b1 = {w1.x, w1.y, w1.z, w1.w, 0, 0, 0, 0};
#pragma unroll
    for (int t = 0; t < MT; t++) {
      const int4 a0 = *(const int4*)(ap[t] + (long long)s * 128), a1 = *(const int4*)(ap[t] + (long long)s * 128 + 16);
      const int asc = *(const uint16_t*)(asp[t] + (long long)s * 8);
      const v8i c0 = {a0.x, a0.y, a0.z, a0.w, 0, 0, 0, 0}, c1 = {a1.x, a1.y, a1.z, a1.w, 0, 0, 0, 0};
      acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(c0, b0, acc[t], 4, 4, 0, asc, 0, wsc);
      acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(c1, b1, acc[t], 4, 4, 1, asc, 1, wsc);
    }
  }
#pragma unroll
  for (int t = 0; t < MT; t++)
#pragma unroll
    for (int i = 0; i < 4; i++) part[wave][t * 16 + g * 4 + i][r] = acc[t][i];
  __syncthreads();
  for (int e = threadIdx.x; e < MT * 256; e += WAVES * 64) {
    const int row = m0 + (e >> 4), col = n0 + (e & 15);
    if (row >= m || col >= n) continue;
    float y = 0.f;
#pragma unroll
    for (int v = 0; v < WAVES; v++) y += part[v][e >> 4][e & 15];
    if (bias) y += bias[col];
    if (res) y += as_float(res[(long long)row * ld_res + col]);
    out[(long long)row * ld + col] = from_float<T>(y);
  }
}

// Tiles through LDS.  AF x WF products of 32 x 32 (V_MFMA_SCALE_F32_32X32X64_F8F6F4) a wave, WM x WN waves; slabs of 256
// elements of k (128 bytes of codes a row) in two stages, requested one slab ahead straight into LDS.  In a slab a lane takes
// four neighbouring blocks of its row, one a step, so the bytes of one word of scales serve its four steps through the
// instruction's byte selector.  Row AF j + f of a wave's A rows (WF j + f of its W rows) is MFMA row j of fragment f:
// a lane then holds WF neighbouring columns of a result row, and one LDS read brings the scales of all fragments.
// LDS holds fragment f's rows next to each other (any order can be loaded) with the 16-byte chunks of a row XOR-swizzled
// by half the row's place, so that 16 lanes cover all 64 banks.  Scales are 8 bytes of a row a slab: fetched by slabs they
// would cost a cache line of 128 bytes each, so a thread fetches those of one row for four slabs at a time.
template <int AF, int WF, int WM, int WN>
struct Mx4Tile {
  static constexpr int BM = AF * 32 * WM, BN = WF * 32 * WN, THREADS = WM * WN * 64, ROWS = BM + BN;
  static constexpr int STAGE = ROWS * 128, SCALES = ROWS * 32;
  static constexpr int LDS = 2 * STAGE + SCALES;
  static_assert(ROWS == THREADS, "a thread fetches the scales of one row");
};
template <typename T, int AF, int WF, int WM, int WN>
__global__ __launch_bounds__(WM * WN * 64) void mx4_gemm_tile_k(const uint8_t* a, const uint8_t* as, const uint8_t* w, const uint8_t* ws, int m, int n,
                                                              int slabs, int mt, int nt, const float* bias, const T* res, long long ld_res, T* out,
                                                              long long ld) {
  typedef Mx4Tile<AF, WF, WM, WN> C;
  extern __shared__ __align__(16) uint8_t lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), j = lane & 31, g = lane >> 5;
  const int wm = wave / WN, wn = wave % WN;
  int tm, tn;
  tile_of(blockIdx.x, mt, nt, tm, tn);
  if (tm >= mt) return;
  const int m0 = tm * C::BM, n0 = tn * C::BN;
  const long long row_bytes = (long long)slabs * 128;
  // this lane's eight chunks of a stage: place (slot, position) of LDS, and where in the tile's rows the bytes come from
  constexpr int L = 8;
  uint32_t off[L];
#pragma unroll
  for (int i = 0; i < L; i++) {
    const int slot = (i * (C::THREADS / 64) + wave) * 8 + (lane >> 3), c = (lane & 7) ^ ((slot >> 1) & 7);
    int row;
    if (slot < C::BM) row = min((slot / (AF * 32)) * (AF * 32) + (slot & 31) * AF + (slot / 32) % AF, m - 1 - m0);
    else {
      const int q = slot - C::BM;
      row = min((q / (WF * 32)) * (WF * 32) + (q & 31) * WF + (q / 32) % WF, n - 1 - n0);
    }
    off[i] = (uint32_t)(row * row_bytes + c * 16);
  }
  const uint8_t* ab = a + m0 * row_bytes;
  const uint8_t* wb = w + n0 * row_bytes;
  const uint32_t stage0 = lds_addr_of(lds);
  const auto request = [&](int s) {
    const uint32_t base = stage0 + (s & 1) * C::STAGE + wave * 1024;
#pragma unroll
    for (int i = 0; i < L; i++)
      slab_load16s((i * (C::THREADS / 64) * 8 < C::BM ? ab : wb) + (long long)s * 128, off[i], base + i * C::THREADS * 16);
  };
  static_assert(C::BM % (C::THREADS / 8) == 0, "a request belongs to one operand");
  // scales of row tid of the tile, four slabs: words [slab][half of the slab][row] in LDS
  const uint8_t* sp = tid < C::BM ? as + (long long)(m0 + min(tid, m - 1 - m0)) * slabs * 8 : ws + (long long)(n0 + min(tid - C::BM, n - 1 - n0)) * slabs * 8;
  uint2 sc[4];
  const auto fetch_scales = [&](int s) {
#pragma unroll
    for (int i = 0; i < 4; i++) sc[i] = s + i < slabs ? *(const uint2*)(sp + (long long)(s + i) * 8) : make_uint2(0, 0);
  };
  uint32_t* const scl = (uint32_t*)(lds + 2 * C::STAGE);
  v16f acc[AF][WF];
#pragma unroll
  for (int x = 0; x < AF; x++)
#pragma unroll
    for (int y = 0; y < WF; y++)
#pragma unroll
      for (int i = 0; i < 16; i++) acc[x][y][i] = 0.f;

  fetch_scales(0);
  request(0);
  for (int s = 0; s < slabs; s++) {
    wait_vm_barrier<0>();              // slab s is there for every wave, and none reads the stage of slab s - 1 any more
    if ((s & 3) == 0) {
#pragma unroll
      for (int i = 0; i < 4; i++) {
        scl[(i * 2 + 0) * C::ROWS + tid] = sc[i].x;
        scl[(i * 2 + 1) * C::ROWS + tid] = sc[i].y;
      }
      wait_vm_barrier<63>();
      if (s + 4 < slabs) fetch_scales(s + 4);
    }
    if (s + 1 < slabs) request(s + 1);
    const uint8_t* const sa = lds + (s & 1) * C::STAGE + wm * (AF * 32) * 128;
    const uint8_t* const sw = lds + (s & 1) * C::STAGE + (C::BM + wn * (WF * 32)) * 128;
    const uint32_t* const sc_s = scl + ((s & 3) * 2 + g) * C::ROWS;
    int asc[AF], wsc[WF];
#pragma unroll
    for (int x = 0; x < AF; x++) asc[x] = (int)sc_s[wm * (AF * 32) + j * AF + x];
#pragma unroll
    for (int y = 0; y < WF; y++) wsc[y] = (int)sc_s[C::BM + wn * (WF * 32) + j * WF + y];
    const auto step = [&](auto sel) {
      constexpr int S = decltype(sel)::value;
      v8i af[AF], wf[WF];
      const int at = j * 128 + (((4 * g + S) ^ ((j >> 1) & 7)) * 16);       // 32 rows a fragment: the swizzle is the lane's own
#pragma unroll
      for (int x = 0; x < AF; x++) {
        const int4 v = *(const int4*)(sa + x * 32 * 128 + at);
        af[x] = (v8i){v.x, v.y, v.z, v.w, 0, 0, 0, 0};
      }
#pragma unroll
      for (int y = 0; y < WF; y++) {
        const int4 v = *(const int4*)(sw + y * 32 * 128 + at);
        wf[y] = (v8i){v.x, v.y, v.z, v.w, 0, 0, 0, 0};
      }
#pragma unroll
      for (int x = 0; x < AF; x++)
#pragma unroll
        for (int y = 0; y < WF; y++)
          acc[x][y] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(af[x], wf[y], acc[x][y], 4, 4, S, asc[x], S, wsc[y]);
    };
    step(Int<0>());
    step(Int<1>());
    step(Int<2>());
    step(Int<3>());
  }
  const int col = n0 + wn * (WF * 32) + j * WF;
  if (col >= n) return;
  const bool whole = col + WF <= n;
  float b[WF];
#pragma unroll
  for (int y = 0; y < WF; y++) b[y] = bias && col + y < n ? bias[col + y] : 0.f;
#pragma unroll
  for (int x = 0; x < AF; x++)
#pragma unroll
    for (int i = 0; i < 16; i++) {
      const int row = m0 + wm * (AF * 32) + (8 * (i / 4) + 4 * g + i % 4) * AF + x;
      if (row >= m) continue;
      T* const o = out + (long long)row * ld + col;
      const T* const r = res + (long long)row * ld_res + col;
      if (whole) {
        Pack<T, WF> v, q;
        if (res) q = *(const Pack<T, WF>*)r;
#pragma unroll
        for (int y = 0; y < WF; y++) {
          float f = acc[x][y][i] + b[y];
          if (res) f += as_float(q.v[y]);
          v.v[y] = from_float<T>(f);
        }
        *(Pack<T, WF>*)o = v;
      } else {
#pragma unroll
        for (int y = 0; y < WF; y++)
          if (col + y < n) o[y] = from_float<T>(acc[x][y][i] + b[y] + (res ? as_float(r[y]) : 0.f));
      }
    }
}

namespace {
template <typename T>
int quantize_as(hipStream_t st, const T* x, int rows, int cols, long long ld, int by, uint8_t* codes, uint8_t* scales) {
  const int groups = (cols + 255) / 256;
  if (by == PAHQ_MX4_BY_ROWS) {
    const unsigned wg = (unsigned)(((long long)rows * groups + 7) / 8);
    hipLaunchKernelGGL(mx4_rows_quant_k<T>, dim3(wg), dim3(256), 0, st, x, ld, rows, cols, groups, (uint32_t*)codes, scales);
  } else {
    hipLaunchKernelGGL(mx4_cols_quant_k<T>, dim3((rows + 63) / 64, groups * 2), dim3(256), 0, st, x, ld, rows, cols, groups * 8, codes, scales);
  }
  return hipGetLastError() == hipSuccess ? PAHQ_OK : PAHQ_EHIP;
}
template <typename T>
int values_as(hipStream_t st, const uint8_t* codes, const uint8_t* scales, int rows, int cols, T* out, long long ld) {
  const int groups = (cols + 255) / 256;
  const unsigned wg = (unsigned)(((long long)rows * groups + 7) / 8);
  hipLaunchKernelGGL(mx4_values_k<T>, dim3(wg), dim3(256), 0, st, (const uint32_t*)codes, scales, rows, cols, groups, out, ld);
  return hipGetLastError() == hipSuccess ? PAHQ_OK : PAHQ_EHIP;
}
template <typename T, int AF, int WF, int WM, int WN>
int launch_tile(hipStream_t st, const uint8_t* a, const uint8_t* as, const uint8_t* w, const uint8_t* ws, int m, int n, int slabs, const float* bias,
                const T* res, long long ld_res, T* out, long long ld) {
  typedef Mx4Tile<AF, WF, WM, WN> C;
  const int mt = (m + C::BM - 1) / C::BM, nt = (n + C::BN - 1) / C::BN;
  const void* fn = (const void*)mx4_gemm_tile_k<T, AF, WF, WM, WN>;
  // more LDS than a launch gets by default: an attribute of the kernel on one device, set once for each
  static std::atomic<bool> set[64];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return PAHQ_EHIP;
  if (!set[dev].load(std::memory_order_acquire)) {
    if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS) != hipSuccess) return PAHQ_EHIP;
    set[dev].store(true, std::memory_order_release);
  }
  hipLaunchKernelGGL((mx4_gemm_tile_k<T, AF, WF, WM, WN>), dim3((mt * nt + 7) / 8 * 8), dim3(C::THREADS), C::LDS, st, a, as, w, ws, m, n, slabs, mt, nt,
                     bias, res, ld_res, out, ld);
  return hipGetLastError() == hipSuccess ? PAHQ_OK : PAHQ_EHIP;
}
template <typename T>
int gemm_as(hipStream_t st, const uint8_t* a, const uint8_t* as, const uint8_t* w, const uint8_t* ws, int m, int n, int slabs, const float* bias,
            const T* res, long long ld_res, T* out, long long ld) {
#define TILE(AF_, WF_, WM_, WN_) return launch_tile<T, AF_, WF_, WM_, WN_>(st, a, as, w, ws, m, n, slabs, bias, res, ld_res, out, ld)
  if (m > 64 && slabs < (1 << 16)) {
    if ((long long)((m + 255) / 256) * ((n + 255) / 256) >= 256) TILE(2, 4, 4, 2);
    TILE(2, 2, 2, 2);
  }
#undef TILE
  const unsigned nt = (unsigned)((n + 15) / 16);
#define FEW(MT_, WAVES_) hipLaunchKernelGGL((mx4_gemm_few_k<T, MT_, WAVES_>), dim3(nt, (m + 16 * MT_ - 1) / (16 * MT_)), dim3(WAVES_ * 64), 0, st, a, as, w, \
                                            ws, m, n, slabs, bias, res, ld_res, out, ld)
  if (m <= 16) FEW(1, 8);
  else if (m <= 32) FEW(2, 8);
  else FEW(4, 4);
#undef FEW
  return hipGetLastError() == hipSuccess ? PAHQ_OK : PAHQ_EHIP;
}
// rows of codes are 16-byte loads, rows of scales 8-byte ones
bool held_aligned(const void* codes, const void* scales) { return ((uintptr_t)codes & 15) == 0 && ((uintptr_t)scales & 7) == 0; }
size_t code_bytes(long long rows, long long cols) { return (size_t)(rows * ((cols + 255) / 256) * 128); }
// most groups of 256 elements of one matrix: workgroups are counted in 32 bits (5e11 elements do not fit the card)
bool too_big(long long rows, long long cols) { return rows * ((cols + 255) / 256) >= (1ll << 31); }
}  // namespace

}  // namespace pahq

using namespace pahq;

extern "C" int pahq_mx4_bytes(int32_t rows, int32_t cols, size_t* codes, size_t* scales) {
  if (rows < 0 || cols < 1 || !codes || !scales) return PAHQ_EINVAL;
  *codes = code_bytes(rows, cols);
  *scales = *codes / 16;
  return PAHQ_OK;
}

extern "C" int pahq_mx4_quantize(void* hip_stream, const void* x, int32_t dtype, int32_t rows, int32_t cols, int64_t ld, int32_t by, uint8_t* codes,
                                 uint8_t* scales) {
  if (rows < 0 || cols < 1 || !dtype_bytes(dtype) || (by != PAHQ_MX4_BY_ROWS && by != PAHQ_MX4_BY_COLUMNS)) return PAHQ_EINVAL;
  if (rows == 0) return PAHQ_OK;
  const bool down = by == PAHQ_MX4_BY_COLUMNS;
  if (!x || !codes || !scales || ld < (down ? rows : cols)) return PAHQ_EINVAL;
  if (!held_aligned(codes, scales) || (uintptr_t)x % dtype_bytes(dtype)) return PAHQ_EINVAL;
  // grid.y counts 128 elements down the columns
  if (too_big(rows, cols) || (down && cols > 65535 * 128)) return PAHQ_ETOOBIG;
  const size_t xb = (size_t)((down ? (cols - 1ll) * ld + rows : (rows - 1ll) * ld + cols) * dtype_bytes(dtype)), cb = code_bytes(rows, cols);
  if (overlap(x, xb, codes, cb) || overlap(x, xb, scales, cb / 16) || overlap(codes, cb, scales, cb / 16)) return PAHQ_EINVAL;
  hipStream_t st = (hipStream_t)hip_stream;
  switch (dtype) {
    case PAHQ_F32: return quantize_as(st, (const float*)x, rows, cols, ld, by, codes, scales);
    case PAHQ_BF16: return quantize_as(st, (const bf16_t*)x, rows, cols, ld, by, codes, scales);
    default: return quantize_as(st, (const f16_t*)x, rows, cols, ld, by, codes, scales);
  }
}

extern "C" int pahq_mx4_dequantize(void* hip_stream, const uint8_t* codes, const uint8_t* scales, int32_t rows, int32_t cols, void* out, int32_t dtype,
                                   int64_t ld) {
  if (rows < 0 || cols < 1 || !dtype_bytes(dtype)) return PAHQ_EINVAL;
  if (rows == 0) return PAHQ_OK;
  if (!out || !codes || !scales || ld < cols || !held_aligned(codes, scales) || (uintptr_t)out % dtype_bytes(dtype)) return PAHQ_EINVAL;
  if (too_big(rows, cols)) return PAHQ_ETOOBIG;
  const size_t ob = (size_t)(((rows - 1ll) * ld + cols) * dtype_bytes(dtype)), cb = code_bytes(rows, cols);
  if (overlap(out, ob, codes, cb) || overlap(out, ob, scales, cb / 16)) return PAHQ_EINVAL;
  hipStream_t st = (hipStream_t)hip_stream;
  switch (dtype) {
    case PAHQ_F32: return values_as(st, codes, scales, rows, cols, (float*)out, ld);
    case PAHQ_BF16: return values_as(st, codes, scales, rows, cols, (bf16_t*)out, ld);
    default: return values_as(st, codes, scales, rows, cols, (f16_t*)out, ld);
  }
}

extern "C" int pahq_mx4_gemm(void* hip_stream, const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* w_codes, const uint8_t* w_scales, int32_t m,
                             int32_t n, int32_t k, const float* bias, const void* residual, int64_t ld_residual, void* out, int32_t dtype, int64_t ld_out) {
  const int eb = dtype_bytes(dtype);
  if (m < 0 || n < 0 || k < 1 || !eb) return PAHQ_EINVAL;
  if (m == 0 || n == 0) return PAHQ_OK;
  if (!a_codes || !a_scales || !w_codes || !w_scales || !out || ld_out < n || (residual && ld_residual < n)) return PAHQ_EINVAL;
  if (!held_aligned(a_codes, a_scales) || !held_aligned(w_codes, w_scales)) return PAHQ_EINVAL;
  if ((uintptr_t)out % eb || (uintptr_t)residual % eb || (uintptr_t)bias % 4) return PAHQ_EINVAL;
  // rows of the grid are counted in 16 bits, columns and groups in 32
  if (too_big(m, k) || too_big(n, k) || m > 65535 * 16) return PAHQ_ETOOBIG;
  const size_t ob = (size_t)(((m - 1ll) * ld_out + n) * eb), ab = code_bytes(m, k), wb = code_bytes(n, k);
  if (overlap(out, ob, a_codes, ab) || overlap(out, ob, a_scales, ab / 16) || overlap(out, ob, w_codes, wb) || overlap(out, ob, w_scales, wb / 16) ||
      (bias && overlap(out, ob, bias, (size_t)n * 4)))
    return PAHQ_EINVAL;
  // the residual may be the result's own rows: every element is read by the thread that writes it
  if (residual && !(residual == out && ld_residual == ld_out) && overlap(out, ob, residual, (size_t)(((m - 1ll) * ld_residual + n) * eb))) return PAHQ_EINVAL;
  hipStream_t st = (hipStream_t)hip_stream;
  const int slabs = (k + 255) / 256;
  switch (dtype) {
    case PAHQ_F32:
      return gemm_as(st, a_codes, a_scales, w_codes, w_scales, m, n, slabs, bias, (const float*)residual, ld_residual, (float*)out, ld_out);
    case PAHQ_BF16:
      return gemm_as(st, a_codes, a_scales, w_codes, w_scales, m, n, slabs, bias, (const bf16_t*)residual, ld_residual, (bf16_t*)out, ld_out);
    default:
      return gemm_as(st, a_codes, a_scales, w_codes, w_scales, m, n, slabs, bias, (const f16_t*)residual, ld_residual, (f16_t*)out, ld_out);
  }
}
