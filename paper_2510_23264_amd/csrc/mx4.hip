// Rows in 4 microscaled bits as operators on device tensors: E2M1 codes with one power-of-two scale per 32
// elements (the layout and the definition are in include/pahq.h), and the product of two such matrices on the
// matrix instructions that take them as they are (V_MFMA_SCALE_F32_16X16X128_F8F6F4 and V_MFMA_SCALE_F32_32X32X64_F8F6F4).
//
// Why the instructions may be used directly, where the E4M3 products of the engine go through fp16: a block of 32 products under
// one pair of scales, multiples of 1/4 of up to 36 each, is summed exactly, and blocks are added like binary32 numbers, each addition
// rounded to nearest, subnormal numbers included.  Measured through both instructions: nothing lost where all partial sums
// are binary32 numbers (one product 2^16 times as large as 224 others, a slab 2^8 times as large as those behind it); otherwise within
// one unit of 2^-24 of sum |a w| a block (at most 6 units over 256 elements, 18 over 4096, with scales up to 2^34 apart) and
// without a bias (all products positive, scales 2^24 apart: 0.01 units in the mean).
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <algorithm>
#include <atomic>
#include "../../include/pahq.h"
#include "mma_util.h"
#include "device_tensor.h"
#include "mx4_rules.h"

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

// x [cols][rows] (the masters' layout [k][n]): one thread holds blocks of 32 down the columns of one word of a row, neighbouring
// threads neighbouring words.  Workgroup: 64 words, 256 elements down, a block a wave; the codes go through LDS so that a row's
// 128 bytes leave together.  Back to back into the same memory, as 16 bytes from each thread and so: in bfloat16 4096 x 4096 16.8 and
// 14.9 us, 4096 x 11008 44.4 and 31.7; in fp32 14.5 and 12.9, 32.8 and 32.0.  All workgroups of a round load first and then store: with x
// from HBM these take 28 and 59, 31 and 74 us (profiles/operators_counters.txt), the same values by rows 15 and 35, 25 and 64.
template <typename T>
__global__ __launch_bounds__(512) void mx4_cols_quant_k(const T* x, long long ld, int rows, int cols, int groups, uint8_t* codes, uint8_t* scales) {
  constexpr int N = 4 / sizeof(T), ROWS = 64 * N;
  __shared__ uint4 held[ROWS * 8];                      // [row][block], blocks XOR-swizzled by the row
  __shared__ __align__(8) uint8_t held_scales[ROWS * 8];
  const int lane = threadIdx.x & 63, b = threadIdx.x >> 6, row0 = blockIdx.x * ROWS, row = row0 + lane * N, here = min(N, rows - row);
  {
    const int k0 = blockIdx.y * 256 + b * 32;
    float v[N][32];
    uint32_t top[N] = {};
#pragma unroll
    for (int j = 0; j < 32; j++) {
      const T* const p = x + (long long)(k0 + j) * ld + row;
      Pack<T, N> q = {};
      if (k0 + j < cols) {
        if (here == N) q = *(const Pack<T, N>*)p;
        else if (here > 0) q.v[0] = p[0];
      }
#pragma unroll
      for (int c = 0; c < N; c++) {
        v[c][j] = as_float(q.v[c]);
        top[c] = max(top[c], __float_as_uint(v[c][j]) & 0x7FFFFFFFu);
      }
    }
#pragma unroll
    for (int c = 0; c < N; c++) {
      const int r = lane * N + c;
      const uint32_t s = mx4_scale_of(top[c]);
      uint4 w = make_uint4(0, 0, 0, 0);
      if (s != 255u) {
        const float inv = mx4_inverse(s);
        w = make_uint4(mx4_encode8(v[c], inv), mx4_encode8(v[c] + 8, inv), mx4_encode8(v[c] + 16, inv), mx4_encode8(v[c] + 24, inv));
      }
      held[r * 8 + (b ^ (r & 7))] = w;
      held_scales[r * 8 + b] = (uint8_t)s;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < ROWS / 64; i++) {
    const int r = i * 64 + (threadIdx.x >> 3), c = threadIdx.x & 7;
    if (row0 + r < rows) *(uint4*)(codes + ((long long)(row0 + r) * groups + blockIdx.y) * 128 + c * 16) = held[r * 8 + (c ^ (r & 7))];
  }
  if (threadIdx.x < ROWS && row0 + threadIdx.x < rows)
    *(uint2*)(scales + ((long long)(row0 + threadIdx.x) * groups + blockIdx.y) * 8) = *(const uint2*)(held_scales + threadIdx.x * 8);
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

// The instruction's operand type is wide enough for 8-bit elements; 4-bit ones are its first half.
__device__ __forceinline__ v8i four_bits(int4 v) { return (v8i){v.x, v.y, v.z, v.w, 0, 0, 0, 0}; }

// Few rows: up to 16 rows x 16 columns a workgroup, the sum over k split over its eight waves (slab s of 256 elements to wave s
// mod 8) and joined in LDS in the order of the waves, so results do not depend on timing.  Operands come straight from global
// memory: a lane reads two neighbouring blocks of its row with their scales, which are one halfword, and the four lanes of a row
// take 128 contiguous bytes.  Which 32 elements of the slab a lane's block is does not matter to the sum as long as both
// operands agree.  Rows and columns past the end read the last one and are not stored.  Bound by waits for memory one after the other: a
// wave has one slab in flight, so k = 4096 is two waits and k = 11008 six, and behind the join bias and residual are two more.  In a trace
// with the weights in HBM 1 x 4096 x 4096 with both takes 5.9 us (1.7 for the bytes at the rate of a large copy, 2.3 an empty
// launch), 1 x 4096 x 11008 10.6 (4.7), 1 x 1024 x 16000 9.0 (1.7), where 64 workgroups read alone.
template <typename T>
__global__ __launch_bounds__(512) void mx4_gemm_few_k(const uint8_t* a, const uint8_t* as, const uint8_t* w, const uint8_t* ws, int m, int n, int slabs,
                                                      const float* bias, const T* res, long long ld_res, T* out, long long ld) {
  constexpr int WAVES = 8;
  __shared__ float part[WAVES][16][17];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4, n0 = blockIdx.x * 16;
  const long long row_bytes = (long long)slabs * 128, wr = min(n0 + r, n - 1), ar = min(r, m - 1);
  const uint8_t* wp = w + wr * row_bytes + g * 32;
  const uint8_t* wsp = ws + wr * slabs * 8 + g * 2;
  const uint8_t* ap = a + ar * row_bytes + g * 32;
  const uint8_t* asp = as + ar * slabs * 8 + g * 2;
  v4f acc = {0.f, 0.f, 0.f, 0.f};
  for (int s = wave; s < slabs; s += WAVES) {
    const int4 w0 = *(const int4*)(wp + s * 128ll), w1 = *(const int4*)(wp + s * 128ll + 16);
    const int4 a0 = *(const int4*)(ap + s * 128ll), a1 = *(const int4*)(ap + s * 128ll + 16);
    const int wsc = *(const uint16_t*)(wsp + s * 8ll), asc = *(const uint16_t*)(asp + s * 8ll);
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(four_bits(a0), four_bits(w0), acc, 4, 4, 0, asc, 0, wsc);
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(four_bits(a1), four_bits(w1), acc, 4, 4, 1, asc, 1, wsc);
  }
#pragma unroll
  for (int i = 0; i < 4; i++) part[wave][g * 4 + i][r] = acc[i];
  __syncthreads();
  const int row = threadIdx.x >> 4, col = n0 + (threadIdx.x & 15);
  if (row >= m || col >= n) return;             // (of the 512 threads 256 have an element)
  float y = 0.f;
#pragma unroll
  for (int v = 0; v < WAVES; v++) y += part[v][row][threadIdx.x & 15];
  if (bias) y += bias[col];
  if (res) y += as_float(res[row * ld_res + col]);
  out[row * ld + col] = from_float<T>(y);
}

// Tiles through LDS.  AF x WF products of 32 x 32 (V_MFMA_SCALE_F32_32X32X64_F8F6F4) a wave, a group of WM x WN waves a tile, KW
// groups a workgroup that share the sum over k.  Slabs of 256 elements of k (128 bytes of codes a row) come in two stages,
// straight into LDS, each group's its own.  In a slab a lane takes four neighbouring blocks of its row, one a step, so the bytes
// of one word of scales serve its four steps through the instruction's byte selector.  LDS holds a row's 16-byte chunks
// XOR-swizzled by half the row's number, so that 16 lanes cover all 64 banks.  Scales are 8 bytes of a row a slab; they come by
// pairs of slabs, 16 bytes a request.
// Every read of a fragment (a step ahead) and every request (up to two slabs ahead) stands between two products: the wait for the
// next slab and the barrier are in front of a slab's last step, when all its fragments are in registers and its stage is free.
// A workgroup of one group walks the tiles of its XCD's range; the first slabs of the next tile are requested before the results
// of this one are stored.
template <int AF, int WF, int WM, int WN, int KW>
struct Mx4Tile {
  static constexpr int BM = AF * 32 * WM, BN = WF * 32 * WN, WAVES = WM * WN, THREADS = KW * WAVES * 64, ROWS = BM + BN;
  static constexpr int STAGE = ROWS * 128, GROUP = 2 * (STAGE + ROWS * 16);          // two slabs, two pairs' scales
  static constexpr int STRIDE = WF * 32 + 8;                                         // floats, of a row of a group's results
  static constexpr int OUT = KW > 1 ? KW * AF * 32 * STRIDE * 4 : GROUP + WAVES * 2048;
  static constexpr int LDS = KW * GROUP > OUT ? KW * GROUP : OUT;
  static constexpr int PER_CU = 160 * 1024 / LDS, PER_SIMD = (PER_CU * KW * WAVES + 3) / 4;     // workgroups and waves that the LDS leaves room for
  static constexpr int L = ROWS / (8 * WAVES), SL = ROWS / (64 * WAVES);             // requests of a wave: a slab's codes, a pair's scales
  static_assert(ROWS % (64 * WAVES) == 0 && LDS <= 160 * 1024 && (KW == 1 || WAVES == 1), "whole requests");
  static_assert(BM % (8 * WAVES) == 0 && BM % 64 == (WAVES == 1 && SL == 1 ? 32 : 0), "a request of codes belongs to one operand");
};
template <typename T, int AF, int WF, int WM, int WN, int KW>
__global__ __launch_bounds__(KW * WM * WN * 64, (Mx4Tile<AF, WF, WM, WN, KW>::PER_SIMD)) void mx4_gemm_tile_k(const uint8_t* a, const uint8_t* as, const uint8_t* w,
                                                                                          const uint8_t* ws, int m, int n, int slabs, int mt, int nt,
                                                                                          const float* bias, const T* res, long long ld_res, T* out,
                                                                                          long long ld) {
  typedef Mx4Tile<AF, WF, WM, WN, KW> C;
  constexpr int L = C::L, SL = C::SL, FRAGMENTS = AF + WF;
  // a slab's requests: FIRST of them in the step that frees its stage, the others in the next
  constexpr int FIRST = L * 5 / 8;
  extern __shared__ __align__(16) uint8_t lds[];
  const int lane = threadIdx.x & 63, j = lane & 31, g = lane >> 5, any_wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = any_wave / C::WAVES, wave = any_wave % C::WAVES, wm = wave / WN, wn = wave % WN;
  // tiles of this workgroup's XCD: neighbouring ones run down bands of eight rows of tiles, so that what an XCD works on at a
  // time shares operands in its L2
  const int total = mt * nt, chunk = (total + 7) >> 3, tile_end = min(total, ((int)blockIdx.x & 7) * chunk + chunk), stride = gridDim.x >> 3;
  int tile = ((int)blockIdx.x & 7) * chunk + ((int)blockIdx.x >> 3);
  if (tile >= tile_end) return;
  // this group's slabs of k: s0 .. s0 + count - 1
  const int share = (slabs + KW - 1) / KW, s0 = group * share, count = min(share, slabs - s0);
  const uint32_t row_bytes = (uint32_t)slabs * 128u;

  // Where this lane's chunks of a stage come from, in the rows of the tile that is loaded (rows past the end: the last one, not
  // stored), and its rows' scales.
  int m0, n0;
  uint32_t off[L];
  const uint8_t *ab, *wb, *sp[SL];
  const auto scales_of = [&](int place) {
    return place < C::BM ? as + (long long)min(m0 + place, m - 1) * slabs * 8 : ws + (long long)min(n0 + place - C::BM, n - 1) * slabs * 8;
  };
  const auto place_tile = [&]() {
    const int band = tile / (8 * nt), in = tile - band * 8 * nt, high = min(8, mt - band * 8);
    m0 = (band * 8 + in % high) * C::BM;
    n0 = in / high * C::BN;
#pragma unroll
    for (int i = 0; i < L; i++) {
      const int place = (i * C::WAVES + wave) * 8, c = (lane & 7) ^ (lane >> 4) ^ ((place >> 1) & 4);
      const int row = place + (lane >> 3) - (i * C::WAVES * 8 < C::BM ? 0 : C::BM);
      off[i] = (uint32_t)min(row, i * C::WAVES * 8 < C::BM ? m - 1 - m0 : n - 1 - n0) * row_bytes + c * 16;
    }
    ab = a + (long long)m0 * row_bytes + s0 * 128ll;
    wb = w + (long long)n0 * row_bytes + s0 * 128ll;
#pragma unroll
    for (int i = 0; i < SL; i++) sp[i] = scales_of((i * C::WAVES + wave) * 64 + lane);
  };
  uint8_t* const mine = lds + group * C::GROUP;
  const uint32_t stage0 = lds_addr_of(mine) + wave * 1024, scales0 = stage0 + 2 * C::STAGE;
  // a pair of slabs behind the last full one starts a slab early, so that nothing behind the row is read
  const auto pair_start = [&](int s) { return max(0, min(s0 + (s & ~1), slabs - 2)); };
  const auto request_scales = [&](int s) {
#pragma unroll
    for (int i = 0; i < SL; i++) slab_load16(sp[i] + pair_start(s) * 8ll, scales0 + (s >> 1 & 1) * (C::ROWS * 16) + i * C::WAVES * 1024);
  };
  const auto request = [&](int s, int i) {
    slab_load16s((i * C::WAVES * 8 < C::BM ? ab : wb) + s * 128ll, off[i], stage0 + (s & 1) * C::STAGE + i * C::WAVES * 1024);
  };
  const auto request_first = [&]() {
    if (count <= 0) return;
    if (slabs == 1) {
#pragma unroll 1
      for (int i = 0; i < 4 * SL; i++)          // a row has 8 bytes alone: words 0 1 0 1 of 16 rows
        lds_load4(scales_of((i / 4 * C::WAVES + wave) * 64 + i % 4 * 16 + (lane >> 2)) + (lane & 1) * 4, scales0 + i / 4 * C::WAVES * 1024 + i % 4 * 256);
    } else {
      request_scales(0);
    }
#pragma unroll
    for (int i = 0; i < L; i++) request(0, i);
    if (count > 1) {
#pragma unroll
      for (int i = 0; i < FIRST; i++) request(1, i);
    }
  };

  // fragments and scales of this wave
  const uint8_t* const fa = mine + (wm * (AF * 32) + j) * 128;
  const uint8_t* const fw = mine + (C::BM + wn * (WF * 32) + j) * 128;
  const uint8_t* const fs = mine + 2 * C::STAGE + g * 4 + j * 16;
  int4 af[2][AF], wf[2][WF];
  int asc[2][AF], wsc[2][WF];
  const auto read = [&](int s, int S, int to, int i) {           // fragment i of a step: first those of A
    const int at = (s & 1) * C::STAGE + (((4 * g + S) ^ ((j >> 1) & 7)) * 16);
    if (i < AF) af[to][i] = *(const int4*)(fa + at + i * 32 * 128);
    else wf[to][i - AF] = *(const int4*)(fw + at + (i - AF) * 32 * 128);
  };
  const auto read_scales = [&](int s, int to) {
    const uint8_t* const p = fs + (s >> 1 & 1) * (C::ROWS * 16) + ((s0 + s - pair_start(s)) & 1) * 8;
#pragma unroll
    for (int x = 0; x < AF; x++) asc[to][x] = *(const int*)(p + (wm * (AF * 32) + x * 32) * 16);
#pragma unroll
    for (int y = 0; y < WF; y++) wsc[to][y] = *(const int*)(p + (C::BM + wn * (WF * 32) + y * 32) * 16);
  };
  v16f acc[AF][WF];
  // The products of a step; behind each of them stands its share of `pieces` other instructions.
  const auto multiply = [&](auto sel, int from, int pieces, auto piece) {
    constexpr int S = decltype(sel)::value, N = AF * WF;
#pragma unroll
    for (int i = 0; i < N; i++) {
      const int x = i % AF, y = i / AF;
      acc[x][y] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(four_bits(af[from][x]), four_bits(wf[from][y]), acc[x][y], 4, 4, S, asc[0][x], S, wsc[0][y]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int p = i * pieces / N; p < (i + 1) * pieces / N; p++) {
        piece(p);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  const auto arrive = [&](auto left) {
    constexpr int N = decltype(left)::value;
    if (C::WAVES > 1) wait_vm_barrier<N>();
    else wait_vm_lds<N>();
  };
  // One slab.  NEXT: slab s + 1 is there, the rest of it to be requested; MORE: slab s + 2 too (2: with scales).  Behind the
  // last slab the stage read is an old one that nothing uses.  No branch stands inside: around one the compiler moves the
  // products away from what they hide.  A slab of the 256 x 256 tile: products alone 2190 clocks, with everything 2620; 3280
  // where reads and requests stood in front of a step's products.
  const auto slab = [&](int s, auto next, auto more) {
    constexpr int NEXT = decltype(next)::value, MORE = decltype(more)::value;
    multiply(Int<0>(), 0, FRAGMENTS + (NEXT ? L - FIRST : 0), [&](int p) {
      constexpr int N = NEXT ? L - FIRST : 0;           // requests first: they have the longest way
      if (p < N) request(s + 1, FIRST + p);
      else read(s, 1, 1, p - N);
    });
    multiply(Int<1>(), 1, FRAGMENTS, [&](int p) { read(s, 2, 0, p); });
    multiply(Int<2>(), 0, FRAGMENTS, [&](int p) { read(s, 3, 1, p); });
    arrive(Int<0>());
    multiply(Int<3>(), 1, 1 + FRAGMENTS + (MORE ? FIRST : 0) + (MORE == 2 ? 1 : 0), [&](int p) {
      if (p == 0) read_scales(s + 1, 1);
      else if (p <= FRAGMENTS) read(s + 1, 0, 0, p - 1);
      else if (p <= FRAGMENTS + FIRST) request(s + 2, p - FRAGMENTS - 1);
      else request_scales(s + 2);
    });
#pragma unroll
    for (int x = 0; x < AF; x++) asc[0][x] = asc[1][x];
#pragma unroll
    for (int y = 0; y < WF; y++) wsc[0][y] = wsc[1][y];
  };

  // The results go through LDS, so that a store writes whole lines: V columns a lane.  Non-temporal: what the results would push
  // out of the caches, operands and residual, is worth more there (8192 x 11008 x 4096 248 -> 220 us, 2048 x 8192 x 1024 with a
  // residual in fp32 40 -> 30; without LDS, 8 bytes a lane, 211 and 30, but 50 x 50257 x 768 in fp32 13.5 instead of 10.8).  Where
  // the results are read next nothing is left of it: with mx4_quantize behind them 286 and 285 us, 2048 x 4096 x 1024 18 and 19.
  constexpr int V = 16 / sizeof(T), ACROSS = WF * 32 / V;
  const auto finish = [&](float* f, const float* b, u32x4 u, T* o, const T* r, int left) {
    if (left >= V) {
#pragma unroll
      for (int v = 0; v < V; v++) f[v] = res ? f[v] + b[v] + element<T>(u, v) : f[v] + b[v];
      store16_nt(o, pack16<T>(f));
    } else {
#pragma unroll
      for (int v = 0; v < V; v++)
        if (v < left) o[v] = from_float<T>(res ? f[v] + b[v] + as_float(r[v]) : f[v] + b[v]);
    }
  };

  // stores of a wave and tile (one group)
  constexpr int STORES = AF * 32 * ACROSS / 64;
  bool stores_under_way = false;
  place_tile();
  request_first();
  while (true) {
    // slab 0: behind it are FIRST requests of slab 1, and the last tile's stores where their number is known
    if (count > 1 && stores_under_way) arrive(Int<FIRST + STORES>());
    else if (count > 1) arrive(Int<FIRST>());
    else arrive(Int<0>());
    read_scales(0, 0);
#pragma unroll
    for (int i = 0; i < FRAGMENTS; i++) read(0, 0, 0, i);
#pragma unroll
    for (int x = 0; x < AF; x++)
#pragma unroll
      for (int y = 0; y < WF; y++)
#pragma unroll
        for (int i = 0; i < 16; i++) acc[x][y][i] = 0.f;
    int s = 0;
#pragma unroll 1
    for (; s + 3 < count; s += 2) {
      slab(s, Int<1>(), Int<2>());
      slab(s + 1, Int<1>(), Int<1>());
    }
    if (s + 2 < count) slab(s++, Int<1>(), Int<2>());
    if (s + 1 < count) slab(s++, Int<1>(), Int<0>());
    if (s < count) slab(s, Int<0>(), Int<0>());

    if constexpr (KW > 1) {
      // several groups: all rows, added in the order of the groups by all threads
      wait_vm_barrier<0>();
      constexpr int H = AF * 32, DOWN = C::THREADS / ACROSS, R = (H + DOWN - 1) / DOWN;
      const int t = threadIdx.x, cl = t % ACROSS * V, rl = t / ACROSS, col = n0 + cl, left = n - col;
      float* const sums = (float*)lds + rl * C::STRIDE + cl;
      float b[V];
#pragma unroll
      for (int v = 0; v < V; v++) b[v] = bias ? bias[min(col + v, n - 1)] : 0.f;
      T* const o = out + (long long)(m0 + rl) * ld + col;
      const T* const p = res + (long long)(m0 + rl) * ld_res + col;
      u32x4 u[R];
      if (res && left >= V) {
#pragma unroll
        for (int r = 0; r < R; r++)
          if (mx4_in_tile(rl + r * DOWN, H, m - m0)) u[r] = load16(p + (long long)(r * DOWN) * ld_res);
      }
      float* const put = (float*)lds + group * (H * C::STRIDE) + 4 * g * C::STRIDE + j;
#pragma unroll
      for (int x = 0; x < AF; x++)
#pragma unroll
        for (int y = 0; y < WF; y++)
#pragma unroll
          for (int i = 0; i < 16; i++) put[(x * 32 + 8 * (i / 4) + i % 4) * C::STRIDE + y * 32] = acc[x][y][i];
      __syncthreads();
#pragma unroll
      for (int r = 0; r < R; r++) {
        if (!mx4_in_tile(rl + r * DOWN, H, m - m0) || left <= 0) continue;
        float f[V];
#pragma unroll
        for (int v = 0; v < V; v++) f[v] = sums[r * DOWN * C::STRIDE + v];
#pragma unroll
        for (int q = 1; q < KW; q++)
#pragma unroll
          for (int v = 0; v < V; v++) f[v] += sums[(q * H + r * DOWN) * C::STRIDE + v];
        finish(f, b, u[r], o + (long long)(r * DOWN) * ld, p + (long long)(r * DOWN) * ld_res, left);
      }
      return;
    } else {
      // One group: PR rows of a fragment at a time through 2 KB of the wave's own, in units of a 16-byte store a lane.  The
      // residual is read RING units ahead.
      constexpr int PR = 16 / WF, Q = PR / 2, DOWN = 64 / ACROSS, PU = PR / DOWN, UNITS = AF * (32 / PR) * PU, RING = UNITS < 8 ? UNITS : 8;
      static_assert(UNITS == STORES && PU >= 1, "units");
      arrive(Int<0>());                 // nobody reads the stages any more
      const int cl = lane % ACROSS * V, rl = lane / ACROSS, col = n0 + wn * (WF * 32) + cl, left = n - col;
      stores_under_way = m0 + C::BM <= m && n0 + C::BN <= n;
      // a lane's row of unit q: its row of unit 0 and a distance that is the same for all lanes
      const int row0 = m0 + wm * (AF * 32) + (PU == 1 ? 4 * (rl / Q) + rl % Q : rl);
      const auto down = [](int q) { return q / PU / (32 / PR) * 32 + q / PU % (32 / PR) / (4 / Q) * 8 + q / PU % (4 / Q) * Q + q % PU * 4; };
      T* const o = out + (long long)row0 * ld + col;
      const T* const p = res + (long long)row0 * ld_res + col;
      const bool add = res && left >= V;
      u32x4 u[RING];
#pragma unroll
      for (int q = 0; q < RING; q++)
        if (add && row0 + down(q) < m) u[q] = load16(p + down(q) * ld_res);
      float b[V];
#pragma unroll
      for (int v = 0; v < V; v++) b[v] = bias ? bias[min(col + v, n - 1)] : 0.f;
      tile += stride;
      if (tile < tile_end) {
        place_tile();
        request_first();
      }
      float* const box = (float*)(lds + C::GROUP + wave * 2048);
#pragma unroll
      for (int pass = 0; pass < UNITS / PU; pass++) {
        const int x = pass / (32 / PR), i0 = pass % (32 / PR) / (4 / Q) * 4 + pass % (4 / Q) * Q;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int y = 0; y < WF; y++)
#pragma unroll
          for (int i = 0; i < Q; i++) box[(g * Q + i) * (WF * 32) + y * 32 + j] = acc[x][y][i0 + i];
#pragma unroll
        for (int z = 0; z < PU; z++) {
          const int q = pass * PU + z;
          float f[V];
#pragma unroll
          for (int v = 0; v < V; v++) f[v] = box[(z * DOWN + rl) * (WF * 32) + cl + v];
          if (row0 + down(q) < m && left > 0) finish(f, b, u[q % RING], o + down(q) * ld, p + down(q) * ld_res, left);
          if (q + RING < UNITS && add && row0 + down(q + RING) < m) u[q % RING] = load16(p + down(q + RING) * ld_res);
        }
      }
      if (tile >= tile_end) return;
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
    constexpr int per = 64 * 4 / (int)sizeof(T);
    hipLaunchKernelGGL(mx4_cols_quant_k<T>, dim3((unsigned)((rows + per - 1ll) / per), groups), dim3(512), 0, st, x, ld, rows, cols, groups, codes, scales);
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
template <typename T, int AF, int WF, int WM, int WN, int KW>
int launch_tile(hipStream_t st, const uint8_t* a, const uint8_t* as, const uint8_t* w, const uint8_t* ws, int m, int n, int slabs, const float* bias,
                const T* res, long long ld_res, T* out, long long ld) {
  typedef Mx4Tile<AF, WF, WM, WN, KW> C;
  const int mt = (m + C::BM - 1) / C::BM, nt = (n + C::BN - 1) / C::BN;
  const int tiles = (mt * nt + 7) / 8 * 8;
  if (KW > 1 && tiles >= 1ll << 24) return PAHQ_ETOOBIG;       // fewer than 2^32 threads; the estimate takes larger tiles long before
  const void* fn = (const void*)mx4_gemm_tile_k<T, AF, WF, WM, WN, KW>;
  // more LDS than a launch gets by default: an attribute of the kernel on one device, set once for each
  static std::atomic<bool> set[64];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return PAHQ_EHIP;
  if (!set[dev].load(std::memory_order_acquire)) {
    if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS) != hipSuccess) return PAHQ_EHIP;
    set[dev].store(true, std::memory_order_release);
  }
  hipLaunchKernelGGL((mx4_gemm_tile_k<T, AF, WF, WM, WN, KW>), dim3(KW > 1 ? tiles : std::min(tiles, 256 * C::PER_CU)), dim3(C::THREADS), C::LDS, st, a, as, w, ws, m, n, slabs, mt,
                     nt, bias, res, ld_res, out, ld);
  return hipGetLastError() == hipSuccess ? PAHQ_OK : PAHQ_EHIP;
}
template <typename T>
int gemm_as(hipStream_t st, const uint8_t* a, const uint8_t* as, const uint8_t* w, const uint8_t* ws, int m, int n, int slabs, const float* bias,
            const T* res, long long ld_res, T* out, long long ld) {
  if (mx4_few(m, n, slabs) && mx4_few_fits(n)) {
    hipLaunchKernelGGL(mx4_gemm_few_k<T>, dim3((unsigned)((n + 15) / 16)), dim3(512), 0, st, a, as, w, ws, m, n, slabs, bias, res, ld_res, out, ld);
    return hipGetLastError() == hipSuccess ? PAHQ_OK : PAHQ_EHIP;
  }
#define TILE(...) return launch_tile<T, __VA_ARGS__>(st, a, as, w, ws, m, n, slabs, bias, res, ld_res, out, ld)
  switch (mx4_form(m, n, slabs)) {
    case 0: TILE(1, 1, 1, 1, 4);
    case 1: TILE(2, 2, 1, 1, 4);
    case 2: TILE(2, 2, 1, 1, 2);
    case 3: TILE(2, 2, 2, 2, 1);
    default: TILE(2, 4, 4, 2, 1);
  }
#undef TILE
}
// rows of codes are 16-byte loads, rows of scales 8-byte ones
bool held_aligned(const void* codes, const void* scales) { return ((uintptr_t)codes & 15) == 0 && ((uintptr_t)scales & 7) == 0; }
size_t code_bytes(long long rows, long long cols) { return (size_t)(rows * ((cols + 255) / 256) * 128); }
// Most groups of 256 elements of one matrix: a launch has fewer than 2^32 threads, of them 32 for a group.
bool too_big(long long rows, long long cols) { return rows * ((cols + 255) / 256) > (1ll << 27) - 8; }
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
  // grid.y counts 256 elements down the columns
  if (too_big(rows, cols) || (down && cols > 65535 * 256)) return PAHQ_ETOOBIG;
  const size_t cb = code_bytes(rows, cols);
  size_t xb;
  if (!extent(down ? cols : rows, ld, down ? rows : cols, dtype_bytes(dtype), &xb)) return PAHQ_EINVAL;
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
  const size_t cb = code_bytes(rows, cols);
  size_t ob;
  if (!extent(rows, ld, cols, dtype_bytes(dtype), &ob)) return PAHQ_EINVAL;
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
  // a tile's rows are addressed by 32 bits, tiles counted by 31; 512 threads take 16 columns of few rows
  if (k > PAHQ_MX4_MAX_K || too_big(m, k) || too_big(n, k) || ((m + 31ll) / 32) * ((n + 31ll) / 32) >= (1ll << 31) - 8) return PAHQ_ETOOBIG;
  const size_t ab = code_bytes(m, k), wb = code_bytes(n, k);
  size_t ob, rb = 0;
  if (!extent(m, ld_out, n, eb, &ob) || (residual && !extent(m, ld_residual, n, eb, &rb))) return PAHQ_EINVAL;
  if (overlap(out, ob, a_codes, ab) || overlap(out, ob, a_scales, ab / 16) || overlap(out, ob, w_codes, wb) || overlap(out, ob, w_scales, wb / 16) ||
      (bias && overlap(out, ob, bias, (size_t)n * 4)))
    return PAHQ_EINVAL;
  // the residual may be the result's own rows: every element is read by the thread that writes it
  if (residual && !(residual == out && ld_residual == ld_out) && overlap(out, ob, residual, rb) &&
      !side_by_side(out, (size_t)n * eb, residual, (size_t)n * eb, ld_out == ld_residual ? (size_t)ld_out * eb : 0))
    return PAHQ_EINVAL;
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
