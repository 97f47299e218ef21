// What a cache that keeps weights adds to those of four tokens.
#pragma once
#include <hip/hip_runtime.h>

namespace lq {

// w[0..3] += the sum over a kv head's query heads of 2^(z - m) / l, for tokens t .. t + 3 of n; a step sets the weight of the newest
// one.  stat(g): m and 1 / l of head g; z: its logits, 16 tokens by head.
template <bool STEP, typename Stat>
__device__ __forceinline__ void add_weights(float* w, int t, int n, int heads, Stat stat, const float* z) {
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int g = 0; g < heads; ++g) {
    const float2 s = stat(g);
    const f32x4 y = *reinterpret_cast<const f32x4*>(z + 16 * g);
    if (s.y > 0.f)                                     // (else nothing had weight)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] = fmaf(__builtin_amdgcn_exp2f(y[e] - s.x), s.y, sum[e]);
  }
  const int fresh = STEP ? n - 1 - t : 4;              // of the four, the one that is new
  if (t + 4 <= n) {
    f32x4 x = *reinterpret_cast<const f32x4*>(w);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (e == fresh ? 0.f : x[e]) + sum[e];
    *reinterpret_cast<f32x4*>(w) = x;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (t + e < n) w[e] = (e == fresh ? 0.f : w[e]) + sum[e];
  }
}

}  // namespace lq
