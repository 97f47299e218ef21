// Decode attention over the 8-bit cache.
//
// Per (row, kv head): logits s = scale * q . k over its tokens, p = softmax(s), o = sum p v, in one pass with the running
// maximum and sum of the softmax.  Both products are matrix instructions of 16 x 16 x 32 with up to 16 query heads of the kv
// head as the columns of one operand:
//   S^T = K Q^T   codes of keys, e4m3, which fp16 and bf16 hold exactly, against q as it came; the scale of a block is one
//                 factor of the fp32 logits of its tokens
//   O^T = V^T P^T codes of values as fp16 against the probabilities as the sum of two fp16 operands; the scale of a block is one
//                 factor of the fp32 sum over a unit of 32 tokens, which is then added to the running sums
// A lane of S^T holds four tokens of one head, which are the elements it owes to P^T (tokens permuted inside a unit, as they
// are stored), and the result of O^T has the heads in the same lanes: nothing but the maximum crosses lanes.
// Probabilities are 2^(s' - m) with s' = s log2(e) and m the largest s' when it was last looked up, at most 5 behind, less 10:
// they stay below 2^15, and one 2^-24 of the largest still is a normal fp16 number.  s' is rounded once, as m was, before they
// are subtracted, and m is no further from it than fp32 can tell (`reference`): from |s'| = 2^24 on, with 10 - m rounded and s'
// not, probabilities were off by powers of two or infinite (a token of 3000s in q and k, d = 128: NaN).
// The second operand is what the rounding of the first one left, so that a probability is held to 22 bits, or to 2^-35 of the
// largest.  Without it an output moves by 1.4e-4 of itself, which carries one bf16 output in twenty over a border of its own
// rounding: the outputs were 7.3e-4 (2-norm; 16 rows x 32 heads x 32768, d = 96) and 7.1e-4 (8 kv heads, 520 tokens) from those
// with probabilities in fp32, now 1.6e-4 and 5.5e-5.  It costs nothing with up to 16 heads in a workgroup (those 16 rows 520.5 us
// with and without, 131072 tokens x 8 kv heads 49.9) and up to 5 % with more (8 rows of 20000, 24 heads 19.9 -> 20.6 us).  The
// tail's operands are of T, two of fp16 or three of bf16 (a step over 520 tokens 6.1 -> 6.4 us with the third).  The sum of the
// probabilities is kept in fp32, before any rounding.
//
// Bound by the bytes of the codes.  A unit of d = 128 (8 KB) costs a wavefront about 200 vector and 24 matrix
// instructions, a quarter of what a compute unit has time for while its share of them arrives.  Keys of the next unit are
// loaded while the values of this one are used, in the same registers, so that 4 wavefronts fit a SIMD; one to three units
// more in flight brought nothing.  131072 tokens x 8 kv heads, bf16, 269 MB: 49.7 us, 5.4 TB/s; of these 1.7 us until the first
// keys are there, 40.5 in the loop (6.6 TB/s), 3 between the first and the last wavefront to end, 3 to join 32 parts.
// 16 rows x 32 heads x 32768, d = 96, 3.2 GB: 518 us, 6.2 TB/s, 0.97 of what a plain read reaches.
//
// Workgroups take items or parts of them (lq_plan8.h), their wavefronts unit by unit (lq_deal8.h).
#include <type_traits>

#include "lq_attn_parts.h"
#include "lq_cache8.h"
#include "lq_device.h"
#include "lq_internal.h"
#include "lq_quant8.h"

namespace lq {

namespace {

struct Attn8Params {
  const uint16_t* q;
  uint16_t* out;
  uint8_t *k_codes, *v_codes;                // (written by a step whose token fills up a block)
  float *k_scale, *v_scale;
  uint16_t *k_tail, *v_tail;
  const uint16_t *k_new, *v_new;             // step: the token that becomes the last row of the tail; else null
  int* counters;
  float* partials;
  const Row8* rows;
  float scale;                               // softmax scale times log2(e)
  int B, Hkv, gh, groups, hb, log_g, cap;
  Row8 same;                                 // ROWS_SAME: every row's entry
};

// eight codes as an operand of T
template <bool BF16>
__device__ __forceinline__ u32x4 codes_as(uint32_t a, uint32_t b) {
  if constexpr (BF16) {
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)a, 1.f, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)a, 1.f, true)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)b, 1.f, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)b, 1.f, true))};
  } else {
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)a, 1.f, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)a, 1.f, true)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)b, 1.f, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)b, 1.f, true))};
  }
}
// SETS: sets of 16 query heads, the columns of an operand, that share the loads and the converted codes.
template <bool BF16, int D, int NW, int SETS, int MODE, bool STEP>
__global__ void __launch_bounds__(64 * NW, SETS == 1 ? 4 : 2) attn8_kernel(const Attn8Params P, const Rows8<MODE> S) {
  (void)S;
  constexpr int ND = D / 32, NT = D / 16, UNIT = 32 * D;   // UNIT: bytes of a unit's codes
  extern __shared__ __align__(16) float o_lds[];       // [NW][hb][PITCH], m and l of a head behind its row; or a join
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int a = lane / 16, head = lane % 16;
  const int per_row = P.Hkv * P.groups;                // items of a row

  // row, item j of it, part of the item
  int b, n, parts, local;
  if constexpr (MODE == ROWS_SAME) {
    n = P.same.n;
    parts = P.same.parts;
    b = blockIdx.x / (per_row * parts);
    local = blockIdx.x - b * per_row * parts;
  } else {
    // The argument block lies in host memory: one load of all its rows, of which those are counted that begin here or before.
    const Row8Ptr rows = rows_ptr(P.rows, sizeof(Attn8Params));
    Row8 mine{};
    for (int i0 = 0; i0 < P.B; i0 += 64) {
      const int i = i0 + lane;
      Row8 r{};
      if (i < P.B) r = Row8{rows[i].n, rows[i].x, rows[i].parts, rows[i].b};
      const int c = __popcll(__ballot(i < P.B && r.x <= (int)blockIdx.x));
      if (!c) break;
      mine = Row8{__builtin_amdgcn_readlane(r.n, c - 1), __builtin_amdgcn_readlane(r.x, c - 1),
                  __builtin_amdgcn_readlane(r.parts, c - 1), __builtin_amdgcn_readlane(r.b, c - 1)};
    }
    n = mine.n;
    parts = mine.parts;
    b = mine.b;
    local = blockIdx.x - mine.x;
  }
  // Workgroups i and i + 8 are on the same die, with an L2 of its own: the head groups of a kv head, which read the same codes
  // in the same order, are that far apart.
  const Pair8 of = pair8(local, P.groups, P.Hkv * parts);
  const int pair = of.pair, g = of.g;                  // (kv head, part), head group
  const int h = pair / parts, part = pair - h * parts, j = h * P.groups + g;
  const int first_slot = (int)blockIdx.x - local + j * parts;               // of the item's partial results
  const Part8 mine = part8(n, part, parts, P.log_g, STEP);
  const int codes = mine.codes, rest = mine.rest, pos = mine.pos, stop = mine.stop, tails = mine.tails;
  const int64_t bh = (int64_t)b * P.Hkv + h;
  const int heads = P.hb < P.gh - g * P.hb ? P.hb : P.gh - g * P.hb;
  const int64_t head0 = bh * P.gh + g * P.hb;

  u32x4 q[SETS][ND];
  {
    const __amdgpu_buffer_rsrc_t rs = buffer(P.q + head0 * D, heads * D * 2);   // absent heads: zeros
#pragma unroll
    for (int x = 0; x < SETS; ++x)
#pragma unroll
      for (int nd = 0; nd < ND; ++nd) q[x][nd] = load16(rs, (16 * x + head) * D * 2 + a * 16 + nd * 64);
  }

  // (The first wavefronts, which have the tail, are the oldest, and their loads are served first.)
  const bool has_tail = wave < tails;
  const Deal8 deal = deal8(mine, wave, NW);
  int i = deal.first, step = deal.step;

  const __amdgpu_buffer_rsrc_t rk = buffer(P.k_codes + bh * P.cap * D, stop * UNIT);   // behind the last unit: zeros, no reads
  const __amdgpu_buffer_rsrc_t rv = buffer(P.v_codes + bh * P.cap * D, stop * UNIT);
  typedef const float __attribute__((address_space(4))) * ScalePtr;      // read by scalar loads
  const ScalePtr ks = (ScalePtr)(uintptr_t)(P.k_scale + bh * (P.cap >> P.log_g));
  const ScalePtr vs = (ScalePtr)(uintptr_t)(P.v_scale + bh * (P.cap >> P.log_g));
  // Workgroups begin somewhere in their part and go round.  All from the front, those of a launch would be at the same
  // distance into their slices all along, and with some capacities, whose slices lie a multiple of the memory's interleaving
  // apart, wait for the same few channels: 8 kv heads of 131072 tokens in slices of 132096 82.9 instead of 49.1 us, 64 rows
  // of 2048 in slices of 4128 55.3 instead of 47.0 (in slices of 4160 46.4 either way).
  const int len = stop - pos;
  const int turn = len > 0 ? (int)((uint64_t)((uint32_t)((int)blockIdx.x - local + pair) * 0x9E3779B1u) * (uint32_t)len >> 32) : 0;
  u32x4 k[ND], v[ND];
  float ck, cv;
  int unit;                                            // the i-th, counted from there
  auto load_k = [&]() {
    unit = turned8(mine, i, turn);
#pragma unroll
    for (int nd = 0; nd < ND; ++nd) k[nd] = load16(rk, unit * UNIT + lane * 16 + nd * 1024);
    const int block = i < stop ? unit >> (P.log_g - 5) : 0;
    ck = ks[block];
    cv = vs[block];
  };
  auto load_v = [&]() {
#pragma unroll
    for (int nd = 0; nd < ND; ++nd) v[nd] = load16(rv, unit * UNIT + lane * 16 + nd * 1024);
  };

  f32x4 acc[SETS][NT];
  float m[SETS], l[SETS];
#pragma unroll
  for (int x = 0; x < SETS; ++x) {
    m[x] = -INFINITY;
    l[x] = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[x][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // a lane's largest logit of a unit: when it is over the largest so far by more than SLACK anywhere, a new reference
  auto look_up = [&](int x, float top) {
    if (__any(top - m[x] > BIAS + SLACK)) {
      const float now = fmaxf(m[x], reference(head_max(top))), f = weight(m[x], now);
      m[x] = now;
      l[x] *= f;
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[x][t] *= f;
    }
  };

  // ---- rows of the tail
  bool ready = false;                                  // k, v hold codes that are not in memory yet
  if (tails) {
    uint16_t* k_tail = P.k_tail + (bh << P.log_g) * D;
    uint16_t* v_tail = P.v_tail + (bh << P.log_g) * D;
    const int left = rest - 32 * wave, live = left < 32 ? left : 32;
    u32x4 kt[2 * ND], vt[NT];
    if (has_tail) {
      // lanes whose rows are not there read nothing
      const __amdgpu_buffer_rsrc_t rkt = buffer(k_tail + 32 * wave * D, 64 * D), rvt = buffer(v_tail + 32 * wave * D, 64 * D);
      const int nothing = 64 * D;
#pragma unroll
      for (int t = 0; t < 2 * ND; ++t) kt[t] = load16(rkt, 16 * (t / ND) + head < live ? t * 1024 + lane * 16 : nothing);
#pragma unroll
      for (int t = 0; t < NT; ++t) vt[t] = load16(rvt, 4 * a < live ? t * 1024 + lane * 16 : nothing);
      if (STEP && left <= 32) {                        // the new row takes its place, here and (every head group) in the cache
        const int t = left - 1, r = 32 * wave + t, e = 4 * (t / 16) + t % 4;
        u32x4 k_new[ND];
        uint16_t v_new[NT];
#pragma unroll
        for (int nd = 0; nd < ND; ++nd) k_new[nd] = *reinterpret_cast<const u32x4*>(P.k_new + bh * D + 32 * nd + 8 * a);
#pragma unroll
        for (int n = 0; n < NT; ++n) v_new[n] = P.v_new[bh * D + 16 * n + head];
        if (head == t % 16) {
#pragma unroll
          for (int nd = 0; nd < ND; ++nd) {
            if (t < 16) kt[nd] = k_new[nd]; else kt[ND + nd] = k_new[nd];
            *reinterpret_cast<u32x4*>(k_tail + k_fp_index(r, 32 * nd + 8 * a, ND)) = k_new[nd];
          }
        }
        if (a == t % 16 / 4) {
          const uint32_t mask = e & 1 ? 0xFFFF0000u : 0xFFFFu;
#pragma unroll
          for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int w = 0; w < 4; ++w)
              if (w == e / 2) vt[n][w] = (vt[n][w] & ~mask) | ((v_new[n] * 0x10001u) & mask);
            v_tail[v_fp_index(r, 16 * n + head, NT)] = v_new[n];
          }
        }
      }
    }
    if (STEP && rest >> P.log_g) {
      // The new row fills up the block: quantized here as append8_kernel does it (operands of the tail and pieces of codes
      // have the same tokens and channels in a lane), and attended to as codes.
      __shared__ uint32_t tops[4];
      uint32_t top = 0;
      if (has_tail) {
        uint32_t top_k = 0, top_v = 0;
#pragma unroll
        for (int t = 0; t < 2 * ND; ++t)
#pragma unroll
          for (int w = 0; w < 4; ++w) top_k = max_pair(top_k, kt[t][w]);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int w = 0; w < 4; ++w) top_v = max_pair(top_v, vt[t][w]);
        top = max_pair(top_k & 0xFFFF, top_k >> 16) | (max_pair(top_v & 0xFFFF, top_v >> 16) << 16);
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) top = max_pair(top, (uint32_t)__shfl_xor((int)top, x));
        if (lane == 0) tops[wave] = top;
      }
      __syncthreads();
      if (has_tail) {
        for (int w = 0; w < tails; ++w) top = max_pair(top, tops[w]);
        const int ek = scale_exponent<BF16>(top & 0xFFFF), ev = scale_exponent<BF16>(top >> 16);
        const float ik = pow2(-ek), iv = pow2(-ev), cut = t2f<BF16>(cut_bits<BF16>());
        const float mk = fminf(448.f, cut * ik), mv = fminf(448.f, cut * iv);
        uint8_t* k_out = P.k_codes + bh * P.cap * D + (int64_t)(codes + wave) * UNIT + lane * 16;
        uint8_t* v_out = P.v_codes + bh * P.cap * D + (int64_t)(codes + wave) * UNIT + lane * 16;
#pragma unroll
        for (int nd = 0; nd < ND; ++nd) {
          k[nd] = u32x4{codes4<BF16>(kt[nd][0], kt[nd][1], ik, mk), codes4<BF16>(kt[nd][2], kt[nd][3], ik, mk),
                        codes4<BF16>(kt[ND + nd][0], kt[ND + nd][1], ik, mk), codes4<BF16>(kt[ND + nd][2], kt[ND + nd][3], ik, mk)};
          v[nd] = u32x4{codes4<BF16>(vt[2 * nd][0], vt[2 * nd][1], iv, mv), codes4<BF16>(vt[2 * nd][2], vt[2 * nd][3], iv, mv),
                        codes4<BF16>(vt[2 * nd + 1][0], vt[2 * nd + 1][1], iv, mv), codes4<BF16>(vt[2 * nd + 1][2], vt[2 * nd + 1][3], iv, mv)};
          *reinterpret_cast<u32x4*>(k_out + nd * 1024) = k[nd];
          *reinterpret_cast<u32x4*>(v_out + nd * 1024) = v[nd];
        }
        ck = pow2(ek);
        cv = pow2(ev);
        if (wave == 0 && lane == 0) {
          const int64_t block = bh * (P.cap >> P.log_g) + (codes >> (P.log_g - 5));
          P.k_scale[block] = ck;
          P.v_scale[block] = cv;
        }
        ready = true;
      }
    } else if (has_tail) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int w = 0; w < 4; ++w) {                  // rows that are not there have weight 0, but may hold anything
          const int t0 = 16 * (w / 2) + 4 * a + 2 * (w % 2);
          vt[t][w] &= (t0 < live ? 0xFFFFu : 0u) | (t0 + 1 < live ? 0xFFFF0000u : 0u);
        }
#pragma unroll
      for (int x = 0; x < SETS; ++x) {
        f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
        for (int nd = 0; nd < ND; ++nd) {
          s0 = mfma<BF16>(kt[nd], q[x][nd], s0);
          s1 = mfma<BF16>(kt[ND + nd], q[x][nd], s1);
        }
        float z[8], top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          z[e] = 16 * (e / 4) + 4 * a + e % 4 < live ? product(e < 4 ? s0[e] : s1[e - 4], P.scale) : -INFINITY;
          top = fmaxf(top, z[e]);
        }
        look_up(x, top);
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(z[e] - m[x]);
          l[x] += p[e];
        }
#pragma unroll
        for (int y = 0; y < (BF16 ? 3 : 2); ++y) {     // a bf16 operand keeps 8 bits, an fp16 one 11
          const u32x4 pb = operand<BF16>(p);
          take<BF16>(p, pb);
#pragma unroll
          for (int t = 0; t < NT; ++t) acc[x][t] = mfma<BF16>(vt[t], pb, acc[x][t]);
        }
      }
    }
  }

  // ---- codes; the keys of the next unit are under way while the values of this one are used
  if (!ready && i < stop) {
    load_k();
    load_v();
  }
  while (ready || i < stop) {
    f32x4 s0[SETS], s1[SETS];
#pragma unroll
    for (int x = 0; x < SETS; ++x) s0[x] = s1[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int nd = 0; nd < ND; ++nd) {
      const u32x4 k0 = codes_as<BF16>(k[nd][0], k[nd][1]), k1 = codes_as<BF16>(k[nd][2], k[nd][3]);
#pragma unroll
      for (int x = 0; x < SETS; ++x) {
        s0[x] = mfma<BF16>(k0, q[x][nd], s0[x]);
        s1[x] = mfma<BF16>(k1, q[x][nd], s1[x]);
      }
    }
    const float c = ck * P.scale, f = cv;
    if (!ready) {
      i += step;
      step = NW;
    }
    ready = false;
    load_k();
    u32x4 pb[SETS], pr[SETS];
#pragma unroll
    for (int x = 0; x < SETS; ++x) {
      float z[8], top = -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        z[e] = product(e < 4 ? s0[x][e] : s1[x][e - 4], c);
        top = fmaxf(top, z[e]);
      }
      look_up(x, top);
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(z[e] - m[x]);
        l[x] += p[e];
      }
      pb[x] = operand<false>(p);
      take<false>(p, pb[x]);
      pr[x] = operand<false>(p);
    }
#pragma unroll
    for (int nd = 0; nd < ND; ++nd) {
      const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
      const u32x4 v0 = codes_as<false>(v[nd][0], v[nd][1]), v1 = codes_as<false>(v[nd][2], v[nd][3]);
#pragma unroll
      for (int x = 0; x < SETS; ++x) {
        const f32x4 o0 = mfma<false>(v0, pr[x], mfma<false>(v0, pb[x], zero)), o1 = mfma<false>(v1, pr[x], mfma<false>(v1, pb[x], zero));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[x][2 * nd][e] = fmaf(o0[e], f, acc[x][2 * nd][e]);
          acc[x][2 * nd + 1][e] = fmaf(o1[e], f, acc[x][2 * nd + 1][e]);
        }
      }
    }
    load_v();
  }

  join_parts<D, NW, SETS>(o_lds, P.hb, heads, part, parts, first_slot, P.counters + (int64_t)(b * per_row + j) * CTR8, P.partials, acc, m, l,
                          [&](int hd, int c, f32x4 o, float, float sum) {
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    *reinterpret_cast<u32x2*>(P.out + (head0 + hd) * D + c) =
        u32x2{pair_as<BF16>(o[0] * inv, o[1] * inv), pair_as<BF16>(o[2] * inv, o[3] * inv)};
  });
}

template <int MODE, bool STEP>
hipError_t attn8(const Shape8& s, const Attn8Params& p, const Rows8<MODE>& rows, const Plan8& plan, hipStream_t st) {
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(plan.blocks), dim3(64 * plan.waves), lds_bytes8(plan.waves, plan.hb, s.d), st, p, rows);
  };
  auto with = [&](auto bf16, auto waves, auto sets) {
    constexpr bool T = decltype(bf16)::value;
    constexpr int NW = decltype(waves)::value, SETS = decltype(sets)::value;
    if (s.d == 64) return go(attn8_kernel<T, 64, NW, SETS, MODE, STEP>);
    if (s.d == 96) return go(attn8_kernel<T, 96, NW, SETS, MODE, STEP>);
    go(attn8_kernel<T, 128, NW, SETS, MODE, STEP>);
  };
  auto with_type = [&](auto bf16) {
    const std::integral_constant<int, 1> one;
    if (plan.hb > 16) return with(bf16, std::integral_constant<int, 4>{}, std::integral_constant<int, 2>{});
    if constexpr (MODE == ROWS_LISTED)                 // (plan8 has no 16 for rows that are alike)
      if (plan.waves == 16) return with(bf16, std::integral_constant<int, 16>{}, one);
    if (plan.waves == 8) return with(bf16, std::integral_constant<int, 8>{}, one);
    with(bf16, std::integral_constant<int, 4>{}, one);
  };
  if (s.bf16) with_type(std::true_type{}); else with_type(std::false_type{});
  return launch_status("attn8");
}

}  // namespace

hipError_t launch_attn8(const Shape8& s, const lq_cache8& c, const void* q, float scale, void* out, void* ws, const Plan8& plan,
                        const void* k_new, const void* v_new, const RowArg8& rows, hipStream_t st) {
  Attn8Params p{(const uint16_t*)q, (uint16_t*)out, c.k_codes, c.v_codes, c.k_scale, c.v_scale, (uint16_t*)c.k_tail, (uint16_t*)c.v_tail,
                (const uint16_t*)k_new, (const uint16_t*)v_new, (int*)ws, (float*)((char*)ws + counter_bytes8(s)), nullptr,
                scale * 1.44269504088896340736f, s.B, s.Hkv, s.gh, plan.groups, plan.hb, log2_of(s.G), s.cap,
                rows.host[0]};
  if (rows.same) {
    const Rows8<ROWS_SAME> none;
    return k_new ? attn8<ROWS_SAME, true>(s, p, none, plan, st) : attn8<ROWS_SAME, false>(s, p, none, plan, st);
  }
  Rows8<ROWS_LISTED> listed{};
  const hipError_t e = hand_over(rows, &listed, &p.rows, st);
  if (e != hipSuccess) return e;
  return k_new ? attn8<ROWS_LISTED, true>(s, p, listed, plan, st) : attn8<ROWS_LISTED, false>(s, p, listed, plan, st);
}

}  // namespace lq
