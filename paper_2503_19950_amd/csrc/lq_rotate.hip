// Rotary positions of queries and keys.
//
// Bound by the bytes: a workgroup takes up to 16 tokens, computes their cosines and sines once, into LDS, and turns these
// tokens' rows of all heads (or of a share of them, where tokens are few) with them.  A thread holds both halves of eight
// pairs, or four pairs of neighbours, so that a row may be written where it was read.
#include "lq_internal.h"
#include "lq_paged.h"
#include "lq_quant8.h"

namespace lq {

namespace {

constexpr int TOKENS = 16, PITCH = 66;       // tokens of a workgroup; pairs from one token's angles to the next (64 and padding)

struct RotateParams {
  const uint16_t *q, *k;
  uint16_t *q_out, *k_out;
  RopeArg rope;
  int L, Hq, Hkv, heads;                     // Hq, Hkv: 0 for a tensor that is not wanted; heads: of a workgroup
  int log_t;                                 // tokens of a workgroup
};

// VECTOR: the rotated channels and their halves are whole pieces of 16 bytes
template <bool BF16, int D, bool VECTOR>
__global__ void __launch_bounds__(256) rotate_kernel(const RotateParams P) {
  __shared__ __align__(16) float2 cs[TOKENS * PITCH];
  const int b = blockIdx.z, tokens = 1 << P.log_t, t0 = (int)blockIdx.x << P.log_t, here = P.L - t0 < tokens ? P.L - t0 : tokens;
  const int dims = P.rope.dims, pairs = dims / 2;
  for (int x = threadIdx.x; x < here * pairs; x += 256) {
    const int t = x / pairs, i = x - t * pairs;
    const int position = P.rope.positions ? P.rope.positions[(int64_t)b * P.L + t0 + t] : t0 + t;
    cs[t * PITCH + i] = turn_of(P.rope.freq[i], position, P.rope.factor);
  }
  __syncthreads();
  // a row is `turning` pieces that turn (VECTOR: 8 pairs or 4 pairs of neighbours, else a pair) and the pieces behind them
  const bool side = P.rope.interleaved;
  const int turning = VECTOR ? (side ? dims / 8 : dims / 16) : pairs, pieces = turning + (VECTOR ? (D - dims) / 8 : D - dims);
  const int rows_at_once = 256 / pieces, first = threadIdx.x / pieces, piece = threadIdx.x - first * pieces;
  if (first >= rows_at_once) return;
  const int head0 = blockIdx.y * P.heads, head1 = head0 + P.heads < P.Hq + P.Hkv ? head0 + P.heads : P.Hq + P.Hkv;
  const int rows = (head1 - head0) << P.log_t;
  const bool turns = piece < turning;
  const int c0 = !turns ? dims + (piece - turning) * (VECTOR ? 8 : 1) : side ? piece * (VECTOR ? 8 : 2) : piece * (VECTOR ? 8 : 1);
  const int c1 = VECTOR ? c0 + pairs : side ? c0 + 1 : c0 + pairs;        // the pairs' other halves (VECTOR and side: in the same piece)
  auto row_of = [&](int r, bool out) -> uint16_t* {
    const int head = head0 + (r >> P.log_t), t = t0 + (r & (tokens - 1));
    const uint16_t* base = head < P.Hq ? (out ? P.q_out : P.q) : out ? P.k_out : P.k;
    const int64_t at = head < P.Hq ? (int64_t)b * P.Hq + head : (int64_t)b * P.Hkv + head - P.Hq;
    return const_cast<uint16_t*>(base) + (at * P.L + t) * D;
  };
  constexpr int AHEAD = 4;                               // rows under way at a time
  for (int r0 = first; r0 < rows; r0 += AHEAD * rows_at_once) {
    u32x4 x[AHEAD], y[AHEAD];
    uint16_t x1[AHEAD], y1[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int r = r0 + j * rows_at_once;
      if (r >= rows || (r & (tokens - 1)) >= here) continue;
      const uint16_t* from = row_of(r, false);
      if constexpr (VECTOR) {
        x[j] = *reinterpret_cast<const u32x4*>(from + c0);
        if (turns && !side) y[j] = *reinterpret_cast<const u32x4*>(from + c1);
      } else {
        x1[j] = from[c0];
        if (turns) y1[j] = from[c1];
      }
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int r = r0 + j * rows_at_once;
      if (r >= rows || (r & (tokens - 1)) >= here) continue;
      uint16_t* to = row_of(r, true);
      const float2* angle = cs + (r & (tokens - 1)) * PITCH;
      if constexpr (VECTOR) {
        if (turns && side) {
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            uint16_t p = (uint16_t)x[j][w], o = (uint16_t)(x[j][w] >> 16);
            turn_pair<BF16>(p, o, angle[c0 / 2 + w]);
            x[j][w] = p | (uint32_t)o << 16;
          }
        } else if (turns) {
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            uint16_t p = (uint16_t)x[j][w], o = (uint16_t)y[j][w], p1 = (uint16_t)(x[j][w] >> 16), o1 = (uint16_t)(y[j][w] >> 16);
            turn_pair<BF16>(p, o, angle[c0 + 2 * w]);
            turn_pair<BF16>(p1, o1, angle[c0 + 2 * w + 1]);
            x[j][w] = p | (uint32_t)p1 << 16;
            y[j][w] = o | (uint32_t)o1 << 16;
          }
          *reinterpret_cast<u32x4*>(to + c1) = y[j];
        }
        *reinterpret_cast<u32x4*>(to + c0) = x[j];
      } else {
        if (turns) {
          turn_pair<BF16>(x1[j], y1[j], angle[piece]);
          to[c1] = y1[j];
        }
        to[c0] = x1[j];
      }
    }
  }
}

}  // namespace

hipError_t launch_rotate(const RopeArg& rope, int B, int L, int Hq, int Hkv, int d, bool bf16, const void* q, void* q_out, const void* k,
                         void* k_out, hipStream_t st) {
  int log_t = 0;
  while (log_t < 4 && 1 << log_t < L) ++log_t;
  const int chunks = (int)(((int64_t)L + (1 << log_t) - 1) >> log_t), heads = (q ? Hq : 0) + (k ? Hkv : 0);
  // all heads share a workgroup's angles where there are workgroups enough
  int shares = 1;
  while (shares < heads && (int64_t)chunks * B * shares < 1024) shares *= 2;
  shares = shares < heads ? shares : heads;
  const int per = (heads + shares - 1) / shares;
  const RotateParams p{(const uint16_t*)q, (const uint16_t*)k, (uint16_t*)q_out, (uint16_t*)k_out, rope, L, q ? Hq : 0, k ? Hkv : 0, per, log_t};
  const bool vector = rope.interleaved ? rope.dims % 8 == 0 : rope.dims % 16 == 0;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(chunks, (heads + per - 1) / per, B), dim3(256), 0, st, p); };
  auto with = [&](auto t, auto v) {
    constexpr bool T = decltype(t)::value, V = decltype(v)::value;
    if (d == 64) return go(rotate_kernel<T, 64, V>);
    if (d == 96) return go(rotate_kernel<T, 96, V>);
    go(rotate_kernel<T, 128, V>);
  };
  auto with_type = [&](auto t) { if (vector) with(t, std::true_type{}); else with(t, std::false_type{}); };
  if (bf16) with_type(std::true_type{}); else with_type(std::false_type{});
  return launch_status("rotate");
}

}  // namespace lq
