// The turn of one pair at one position, shared by the operators that rotate.
#pragma once
#include <hip/hip_runtime.h>

namespace pahq {

// (cos, sin) times magnitude, the sine times direction (1, or -1 to turn back).  The product position * frequency is a phase in 2^-64
// turns, exact at every position; its two top digits are the quarter turns, and what is left, at most an eighth of a turn,
// loses no more than 2^-25 of that when it becomes a float.
__device__ __forceinline__ float2 rotary_turn(long long position, unsigned long long frequency, float magnitude, float direction) {
  const unsigned long long phase = (unsigned long long)position * frequency + (1ull << 61);
  const int quarter = (int)(phase >> 62);
  const int left = (int)(((long long)(phase << 2) >> 32) ^ 0x80000000ll);         // in 2^-34 turns, from -1/8 on
  float s, c;
  sincospif((float)left * 1.1641532182693481e-10f, &s, &c);                       // 2^-33: half turns
  const float cq = quarter & 1 ? s : c, sq = quarter & 1 ? c : s;
  return make_float2((quarter == 1 || quarter == 2 ? -cq : cq) * magnitude, (quarter >= 2 ? -sq : sq) * magnitude * direction);
}

}  // namespace pahq
