// Rotary positions of queries and keys.
//
// Bound by the bytes.  A lane has 16 bytes of a row, a row lies within a wavefront, and a workgroup has up to T tokens of all
// heads (or of a share of them, where tokens are few), head by head: consecutive tokens of a head are 8 KB in one stretch, and a
// lane's token and channels stay the same, so that its cosines and sines are in registers, computed once by the workgroup
// together.  The other halves of a lane's pairs come from the lane that has them; all of a row is read before any of it is
// written, so that a row may be written where it was read.
// 32768 tokens x 40 heads, d = 128, bf16 (671 MB): 128 us (4 and 8 heads under way a lane 2 and 8 more; without
// the stores' way past the caches 139); a copy of as much takes 132.
#include "lq_internal.h"
#include "lq_paged.h"
#include "lq_quant8.h"

namespace lq {

namespace {

constexpr int WAVES = 8;

struct RotateParams {
  const uint16_t *q, *k;
  uint16_t *q_out, *k_out;
  RopeArg rope;
  int L, Hq, Hkv, heads;                     // Hq, Hkv: 0 for a tensor that is not wanted; heads: of a workgroup
  int tokens;                                // of a workgroup
};

// How pairs lie: neighbours; halves that are whole pieces of 16 bytes; halves that are not.
enum Pairs { NEIGHBOURS, HALVES, ODD };

__device__ __forceinline__ uint32_t from_lane(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_ds_bpermute(4 * lane, (int)v); }
// Eight channels from `shift` channels (0 .. 7) into lo on, hi behind it.
__device__ __forceinline__ u32x4 eight_from(u32x4 lo, u32x4 hi, int shift) {
  u32x4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) {              // word e of (lo, hi) >> 16 * shift
    const int s = shift / 2;
    auto word = [&](int i) { return i < 4 ? lo[i] : i < 8 ? hi[i - 4] : 0u; };
    uint32_t a = 0, b = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w)
      if (w == s) {
        a = word(e + w);
        b = word(e + w + 1);
      }
    y[e] = shift & 1 ? a >> 16 | b << 16 : a;
  }
  return y;
}

template <bool BF16, int D, int PAIRS>
__global__ void __launch_bounds__(64 * WAVES) rotate_kernel(const RotateParams P) {
  constexpr int PIECES = D / 8, ROWS = 64 / PIECES;      // of a row; of a wavefront
  constexpr int AHEAD = 2, PITCH = D / 2 + 2;
  __shared__ __align__(16) float2 angles[WAVES * ROWS * PITCH];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b = blockIdx.z;
  const int dims = P.rope.dims, half = dims / 2, t0 = (int)blockIdx.x * P.tokens, here = P.L - t0 < P.tokens ? P.L - t0 : P.tokens;
  const int row = wave * ROWS + lane / PIECES, c0 = lane % PIECES * 8;
  const int at_once = WAVES * ROWS / P.tokens, t = row % P.tokens;       // heads
  const bool mine = lane < ROWS * PIECES && row < at_once * P.tokens && t < here;
  const int head0 = blockIdx.y * P.heads, head1 = head0 + P.heads < P.Hq + P.Hkv ? head0 + P.heads : P.Hq + P.Hkv;
  auto place = [&](int head, bool out) -> uint16_t* {
    const uint16_t* base = head < P.Hq ? (out ? P.q_out : P.q) : out ? P.k_out : P.k;
    const int64_t at = head < P.Hq ? (int64_t)b * P.Hq + head : (int64_t)b * P.Hkv + head - P.Hq;
    return const_cast<uint16_t*>(base) + (at * P.L + t0 + t) * D + c0;
  };
  u32x4 x[AHEAD];
  auto load = [&](int h) {
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      x[j] = u32x4{0, 0, 0, 0};
      if (mine && h + j * at_once < head1) x[j] = *reinterpret_cast<const u32x4*>(place(h + j * at_once, false));
    }
  };
  // A lane computes the angles of one pair for some of the tokens.  What it takes to compute them is loaded
  // first (loads arrive in order).
  constexpr int WIDE = D / 2 > 32 ? 64 : 32, EACH = WAVES * 64 / WIDE, MOST = (WAVES * ROWS + EACH - 1) / EACH;
  const int pair = threadIdx.x % WIDE, s0 = threadIdx.x / WIDE;
  double freq = 0.0;
  int position[MOST];
  if (pair < half) freq = P.rope.freq[pair];
#pragma unroll
  for (int i = 0; i < MOST; ++i) {
    const int s = s0 + i * EACH;
    position[i] = t0 + s;
    if (P.rope.positions && s < here) position[i] = P.rope.positions[(int64_t)b * P.L + t0 + s];
  }
  int h = head0 + row / P.tokens;
  load(h);
#pragma unroll
  for (int i = 0; i < MOST; ++i)
    if (s0 + i * EACH < here && pair < half) angles[(s0 + i * EACH) * PITCH + pair] = turn_of(freq, position[i], P.rope.factor);
  __syncthreads();
  // of the lane's pairs, four or eight: the sine's sign is that of the other half in the result
  float co[8], si[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int c = c0 + e;
    const bool first = PAIRS == NEIGHBOURS ? !(e & 1) : c < half;
    const float2 cs = angles[(mine && c < dims ? t * PITCH + (PAIRS == NEIGHBOURS ? c / 2 : first ? c : c - half) : 0)];
    co[e] = cs.x;
    si[e] = first ? -cs.y : cs.y;
  }
  // lanes that have the other halves
  const int q = half / 8, shift = half % 8, up = lane + q, down = lane - q - (shift ? 1 : 0);
  for (; h - row / P.tokens < head1; h += AHEAD * at_once) {             // (wavefronts stay together)
    u32x4 z[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      u32x4 y{0, 0, 0, 0}, y2{0, 0, 0, 0};                               // the other halves of first and of second ones
      if constexpr (PAIRS == HALVES) {
        const int who = c0 < half ? up : down;
#pragma unroll
        for (int w = 0; w < 4; ++w) y[w] = from_lane(x[j][w], who);
      }
      if constexpr (PAIRS == ODD) {
        u32x4 n[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          n[0][w] = from_lane(x[j][w], up);
          n[1][w] = from_lane(x[j][w], up + 1);
          n[2][w] = from_lane(x[j][w], down);
          n[3][w] = from_lane(x[j][w], down + 1);
        }
        y = eight_from(n[0], n[1], shift);
        y2 = shift ? eight_from(n[2], n[3], 8 - shift) : n[2];
      }
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t o = PAIRS == NEIGHBOURS ? x[j][w] >> 16 | x[j][w] << 16 : PAIRS == HALVES ? y[w]
                           : ((c0 + 2 * w < half ? y[w] : y2[w]) & 0xFFFFu) | ((c0 + 2 * w + 1 < half ? y[w] : y2[w]) & 0xFFFF0000u);
        const uint32_t lo = f2t<BF16>(fmaf(t2f<BF16>((uint16_t)x[j][w]), co[2 * w], t2f<BF16>((uint16_t)o) * si[2 * w]));
        const uint32_t hi = f2t<BF16>(fmaf(t2f<BF16>((uint16_t)(x[j][w] >> 16)), co[2 * w + 1], t2f<BF16>((uint16_t)(o >> 16)) * si[2 * w + 1]));
        z[j][w] = (c0 + 2 * w < dims ? lo : x[j][w] & 0xFFFFu) | (c0 + 2 * w + 1 < dims ? hi << 16 : x[j][w] & 0xFFFF0000u);
      }
    }
    const int at = h;
    load(h + AHEAD * at_once);
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
      if (mine && at + j * at_once < head1) __builtin_nontemporal_store(z[j], reinterpret_cast<u32x4*>(place(at + j * at_once, true)));
  }
}

}  // namespace

hipError_t launch_rotate(const RopeArg& rope, int B, int L, int Hq, int Hkv, int d, bool bf16, const void* q, void* q_out, const void* k,
                         void* k_out, hipStream_t st) {
  const int rows = WAVES * (64 / (d / 8)), tokens = L < rows ? L : rows, heads = (q ? Hq : 0) + (k ? Hkv : 0);
  const int chunks = (int)(((int64_t)L + tokens - 1) / tokens);
  // all heads share a workgroup's angles where there are workgroups enough
  int shares = 1;
  while (shares < heads && (int64_t)chunks * B * shares < 512) shares *= 2;
  shares = shares < heads ? shares : heads;
  const int per = (heads + shares - 1) / shares;
  const RotateParams p{(const uint16_t*)q, (const uint16_t*)k, (uint16_t*)q_out, (uint16_t*)k_out, rope, L, q ? Hq : 0, k ? Hkv : 0, per, tokens};
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(chunks, (heads + per - 1) / per, B), dim3(64 * WAVES), 0, st, p); };
  auto with = [&](auto t, auto pairs) {
    constexpr bool T = decltype(t)::value;
    constexpr int PAIRS = decltype(pairs)::value;
    if (d == 64) return go(rotate_kernel<T, 64, PAIRS>);
    if (d == 96) return go(rotate_kernel<T, 96, PAIRS>);
    go(rotate_kernel<T, 128, PAIRS>);
  };
  auto with_type = [&](auto t) {
    if (rope.interleaved) with(t, std::integral_constant<int, NEIGHBOURS>{});
    else if (rope.dims % 16 == 0) with(t, std::integral_constant<int, HALVES>{});
    else with(t, std::integral_constant<int, ODD>{});
  };
  if (bf16) with_type(std::true_type{}); else with_type(std::false_type{});
  return launch_status("rotate");
}

}  // namespace lq
