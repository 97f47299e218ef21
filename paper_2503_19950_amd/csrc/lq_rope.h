// Rotary positions: what the kernels that turn queries and keys share.
#pragma once
#include <hip/hip_runtime.h>

#include "lq_device.h"

namespace lq {

struct RopeArg {
  const double* freq;      // radians per position of every pair; null: nothing is turned
  const int* positions;    // null: a token's place
  int dims, interleaved;
  float factor;
};

// Cosine and sine of position * freq, times the factor.  The angle is taken in turns in fp64, where its whole turns go: a
// position of 2^31 leaves 2^-22 turns of 53 bits' rounding at freq = 1, one below 2^20 less than fp32 can tell.  The rest, at
// most half a turn, is rounded to fp32 once.
__device__ __forceinline__ float2 turn_of(double freq, int position, float factor) {
  double t = (double)position * (freq * 0.15915494309189533577);      // 1 / (2 pi)
  t -= rint(t);
  float s, c;
  sincospif(2.f * (float)t, &s, &c);
  return make_float2(c * factor, s * factor);
}

// A pair turned: fp32, each result rounded to T once.
template <bool BF16>
__device__ __forceinline__ void turn_pair(uint16_t& x0, uint16_t& x1, float2 cs) {
  const float a = t2f<BF16>(x0), b = t2f<BF16>(x1);
  x0 = f2t<BF16>(fmaf(a, cs.x, -(b * cs.y)));
  x1 = f2t<BF16>(fmaf(b, cs.x, a * cs.y));
}

}  // namespace lq
