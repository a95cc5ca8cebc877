// Which kernel a product of rows in 4 microscaled bits takes.  No GPU type in it, so that CPU tests compile it.
#pragma once
#include <math.h>

namespace pahq {

// Up to 16 rows: one 16 x 16 product a wave from global memory, except for 5 rows and more whose results and sums are both long.
// Chosen with the weights in HBM, as a program of many layers finds them: 1 x 4096 x 4096 4.3 us (in tiles 6.2), 1 x 1024 x 16000
// 7.8 (14.7), 1 x 11008 x 4096 8.3 (8.7), but 16 x 11008 x 4096 10.9 (8.9) and 11 x 31513 x 9086 47 (34).  Over 70 sizes
// 1.002 of the better one's time in the mean and 1.11 at most; where the last call left the weights in the caches, 1.015 and 1.49.
inline bool mx4_few(long long m, long long n, int slabs) { return m <= 16 && (m <= 4 || n < 4000 || slabs < 10); }
// Whether a launch can count that: 512 threads for 16 columns, fewer than 2^32 in all.  Beyond, tiles take few rows too.
inline bool mx4_few_fits(long long n) { return (n + 15) / 16 * 512 < 1ll << 32; }

// Otherwise tiles of `tile` x `tile`, the sum over k shared by `groups` groups of waves.  The times in microseconds are fitted to
// 400 random sizes from 17 x 16 x 32 to 8192 x 50000 x 12000, all with bfloat16 results and without a residual, which the estimate
// therefore knows nothing of: one workgroup alone takes
// launch + start + slab * (its slabs of 256 elements of k); each further one of a compute unit `round` of that, where only one
// fits (whole) a whole round of the chip half of the time.  The form with the least estimate took 1.01 of the best one's time in
// the mean, 1.2 at most.  A last round of 256 x 256 tiles that leaves most of the chip without one stays as it is: as smaller
// tiles in a launch of their own it cost 250 us instead of 244 (8192 x 11008 x 4096).
struct Mx4Form { int tile, groups; float launch, start, slab, round; bool whole; };
constexpr int MX4_FORMS = 5;
constexpr Mx4Form mx4_forms[MX4_FORMS] = {
    {32, 4, 3.2f, 0.4f, 0.31f, 1.5f, false},      //  100 x 2304 x 768 4.4 us (64 x 64 in two groups 5.5)
    {64, 4, 3.6f, 1.2f, 0.54f, 2.4f, true},       //  256 x 4096 x 4096 8.1 (32 x 32 11.0)
    {64, 2, 2.8f, 1.9f, 0.61f, 0.8f, false},      //  800 x 2304 x 768 6.3 (32 x 32 10.2, 128 x 128 7.7)
    {128, 1, 1.1f, 4.5f, 0.85f, 0.6f, false},     // 2048 x 4096 x 4096 29 (64 x 64 42, 256 x 256 38)
    {256, 1, 4.0f, 8.9f, 1.53f, 1.27f, true},     // 8192 x 4096 x 11008 180 (128 x 128 222)
};
inline float mx4_estimate(const Mx4Form& f, long long m, long long n, int slabs) {
  const float r = (float)((m + f.tile - 1) / f.tile) * (float)((n + f.tile - 1) / f.tile) / 256;
  const float further = r <= 1 ? 0 : f.whole ? 0.5f * (ceilf(r) + r) - 1 : r - 1;
  return f.launch + (f.start + f.slab * ((slabs + f.groups - 1) / f.groups)) * (1 + f.round * further);
}
// Whether a workgroup that joins partial sums has row `at` of its tile of `high` rows, `left` of them in the matrix: its threads may
// reach past the tile, into rows of another workgroup's.
constexpr bool mx4_in_tile(int at, int high, int left) { return at < high && at < left; }
inline int mx4_form(long long m, long long n, int slabs) {
  int best = 0;
  float least = 0;
  for (int i = 0; i < MX4_FORMS; i++) {
    const float t = mx4_estimate(mx4_forms[i], m, n, slabs);
    if (i == 0 || t < least) { least = t; best = i; }
  }
  return best;
}

}  // namespace pahq
