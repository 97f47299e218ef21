// Decode attention over the paged cache.
//
// Per (row, kv head): s = scale * q . k over its tokens, changed by a cap, a bias and a window, p = softmax(s), o = sum p v, in
// one pass with the running maximum and sum of the softmax, as over the 8-bit cache (lq_attn8.hip): S^T = K Q^T and
// O^T = V^T P^T by matrix instructions of 16 x 16 x 32, up to 16 query heads of a kv head as the columns, a lane's four tokens
// of a head being the elements that it owes to P^T.  Operands of keys and values are read from their pages as they lie, 16
// bytes a lane; a unit of 32 tokens never crosses a page, and its page is looked up by a scalar load one unit ahead.
// Probabilities are two operands of fp16 or three of bf16, what each rounding leaves going to the next, so that 2^-22 or 2^-24 of
// each is left of their roundings; of fp16 ones, whose second operand is subnormal for a probability below 2^-3, at least 2^-25, where
// the largest stands at 2^10 or more (BIAS): 2^-35 of it.  What is smaller adds to the sum (and to weights), not to the output.
#pragma once
#include <type_traits>

#include "lq_attn_paged_args.h"
#include "lq_attn_parts.h"
#include "lq_internal.h"
#include "lq_weights.h"

namespace lq {

// Keys and values are read past the caches: a step of a model reads every layer's once.  131072 tokens x 8 kv heads (537 MB) 95.4 and
// 84.5 us; with one to 64 layers in turn, launches of 67 MB and more 0.87 to 1.03 of the time, of 34 MB 0.93 to 1.00, of 2 and 8 MB, whose
// layers the last cache would hold, 0.98 to 1.04 (6.4 and 6.6 us); the values alone 86.3.  A choice by size in the kernel costs 1 %.
__device__ __forceinline__ u32x4 load_once(__amdgpu_buffer_rsrc_t rs, int off) {
  return __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, /* non-temporal */ 2);
}

// tanh: from |x| = 1/4 on by its definition, below by the first terms of its series (the next is 2^-27 of the result there).
__device__ __forceinline__ float tanh_of(float x) {
  const float e = __builtin_amdgcn_exp2f(fabsf(x) * 2.88539008177792681472f);     // e^(2 |x|)
  const float far = copysignf(1.f - 2.f * __builtin_amdgcn_rcpf(e + 1.f), x), y = x * x;
  const float near = x * fmaf(y, fmaf(y, fmaf(y, fmaf(y, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
  return fabsf(x) < 0.25f ? near : far;
}

// SETS: sets of 16 query heads, the columns of an operand, that share the loads.  MORE: with a cap, a bias or weights.
template <bool BF16, int D, int NW, int SETS, int MODE, bool STEP, bool MORE>
__global__ void __launch_bounds__(64 * NW, NW == 16 ? 4 : SETS == 1 ? 3 : 2) attn_paged_kernel(const AttnPagedParams P, const Rows8<MODE> S) {
  (void)S;
  constexpr int ND = D / 32, NT = D / 16, UNIT = 32 * D;                // UNIT: elements of a unit's keys, or values
  extern __shared__ __align__(16) float o_lds[];                        // lds_bytes8
  float* z_lds = o_lds + lds_bytes8(NW, P.hb, D) / 4;                   // with P.weights: logits, as they lie in memory
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int a = lane / 16, head = lane % 16;
  const int per_row = P.Hkv * P.groups;                                 // items of a row

  // row, item j of it, part of the item
  int rb, n, parts, local;
  if constexpr (MODE == ROWS_SAME) {
    n = P.same.n;
    parts = P.same.parts;
    const int b = blockIdx.x / (per_row * parts);
    local = blockIdx.x - b * per_row * parts;
    rb = P.same.b + b;
  } else {
    // one load of all rows' entries, of which those are counted that begin here or before
    const Row8Ptr rows = rows_ptr(P.rows, sizeof(AttnPagedParams));
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
    rb = mine.b;
    local = blockIdx.x - mine.x;
  }
  const int b = rb < P.B ? rb : rb - P.B;
  const Pair8 of = pair8(local, P.groups, P.Hkv * parts);               // (head groups of a kv head on the same die)
  const int pair = of.pair, g = of.g;
  const int h = pair / parts, part = pair - h * parts, j = h * P.groups + g;
  const int first_slot = (int)blockIdx.x - local + j * parts;
  const PartPaged mine = part_paged(n, P.window, part, parts);
  const int64_t bh = (int64_t)b * P.Hkv + h;
  const int heads = P.hb < P.gh - g * P.hb ? P.hb : P.gh - g * P.hb;
  const int64_t head0 = bh * P.gh + g * P.hb;

  // ---- queries.  Their loads come first: loads arrive in order.
  u32x4 q[SETS][ND];
  constexpr int K_NEW = 16 * SETS, V_NEW = K_NEW + 1, ROWS = (V_NEW + 1 + NW - 1) / NW;
  __shared__ __align__(16) uint16_t fresh[STEP ? (K_NEW + 2) * D : 1];  // step: queries, the new key (both turned) and value
  // A step's rows go round the wavefronts, two channels a lane: a pair that turns, or two neighbours of the rest.
  const int dims = STEP && P.rope.freq ? P.rope.dims : 0, pairs = dims / 2;
  const int c0 = lane >= pairs || P.rope.interleaved ? 2 * lane : lane, c1 = lane >= pairs || P.rope.interleaved ? c0 + 1 : lane + pairs;
  uint16_t x0[ROWS], x1[ROWS];
  double freq = 0.0;
  int position = n - 1;
  if constexpr (STEP) {
    if (lane < pairs) {
      freq = P.rope.freq[lane];
      if (P.rope.positions) position = P.rope.positions[b];
    }
#pragma unroll
    for (int y = 0; y < ROWS; ++y) {
      const int r = wave + y * NW;
      if (r >= heads + 2 || 2 * lane >= D) break;
      const uint16_t* from = r < heads ? P.q + (head0 + r) * D : (r == heads ? P.k_new : P.v_new) + bh * D;
      x0[y] = from[r <= heads ? c0 : 2 * lane];
      x1[y] = from[r <= heads ? c1 : 2 * lane + 1];
    }
  } else {
    const __amdgpu_buffer_rsrc_t rs = buffer(P.q + head0 * D, heads * D * 2);              // absent heads: zeros
#pragma unroll
    for (int x = 0; x < SETS; ++x)
#pragma unroll
      for (int nd = 0; nd < ND; ++nd) q[x][nd] = load16(rs, (16 * x + head) * D * 2 + a * 16 + nd * 64);
  }

  float slope[SETS];                                                    // times log2(e)
  if constexpr (MORE) {
    const __amdgpu_buffer_rsrc_t rs = buffer(P.slopes + h * P.gh + g * P.hb, P.slopes ? heads * 4 : 0);
#pragma unroll
    for (int x = 0; x < SETS; ++x)
      slope[x] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, (16 * x + head) * 4, 0, 0)) * 1.44269504088896340736f;
  }

  // ---- units of this wavefront: the i-th, counted from a place of the workgroup's own (in step, the workgroups of a launch
  // wait for the same memory channels where pages follow each other: lq_attn8.hip)
  typedef const int __attribute__((address_space(4))) * TablePtr;       // read by scalar loads
  const TablePtr table = (TablePtr)(uintptr_t)(P.table + (int64_t)rb * P.max_pages);
  const int len = mine.stop - mine.pos;
  const int turn = len > 0 ? (int)((uint64_t)((uint32_t)((int)blockIdx.x - local + pair) * 0x9E3779B1u) * (uint32_t)len >> 32) : 0;
  int i = mine.pos + wave;
  struct Unit { int u, id; };
  auto look = [&](int k) {                                              // behind the last: none
    const int u = turned_paged(mine, k < mine.stop ? k : mine.pos, turn);
    return Unit{u, k < mine.stop ? table[u >> (P.log_p - 5)] : -1};
  };
  u32x4 k[2 * ND], v[NT];
  Unit unit{}, next{};
  int64_t off = 0;                                                      // of the unit loaded last, and whether it is there
  bool there = false;
  auto load_k = [&]() {
    there = is_page(next.id, P.n_pages);
    off = there ? unit_offset(next.id, P.Hkv, h, P.log_p, next.u, D) : 0;
    const __amdgpu_buffer_rsrc_t rs = buffer(P.k_pages + off, there ? UNIT * 2 : 0);       // no page: zeros, no reads
#pragma unroll
    for (int t = 0; t < 2 * ND; ++t) k[t] = load_once(rs, t * 1024 + lane * 16);
  };
  auto load_v = [&]() {
    const __amdgpu_buffer_rsrc_t rs = buffer(P.v_pages + off, there ? UNIT * 2 : 0);
#pragma unroll
    for (int t = 0; t < NT; ++t) v[t] = load_once(rs, t * 1024 + lane * 16);
  };
  next = look(i);                                                       // (a wavefront that has none reads nothing)
  load_k();
  load_v();

  if constexpr (STEP) {
    float2 cs = make_float2(1.f, 0.f);
    if (lane < pairs) cs = turn_of(freq, position, P.rope.factor);
#pragma unroll
    for (int y = 0; y < ROWS; ++y) {
      const int r = wave + y * NW;
      if (r >= heads + 2 || 2 * lane >= D) break;
      uint16_t* to = fresh + (r < heads ? r : r == heads ? K_NEW : V_NEW) * D;
      if (r <= heads && lane < pairs) turn_pair<BF16>(x0[y], x1[y], cs);
      to[r <= heads ? c0 : 2 * lane] = x0[y];
      to[r <= heads ? c1 : 2 * lane + 1] = x1[y];
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < SETS; ++x)
#pragma unroll
      for (int nd = 0; nd < ND; ++nd)
        q[x][nd] = 16 * x + head < heads ? *reinterpret_cast<const u32x4*>(fresh + (16 * x + head) * D + 32 * nd + 8 * a) : u32x4{0, 0, 0, 0};
  }
  // What came before the keys is there from here on (the compiler, which counts loads, would wait for it, and with it for all
  // loads under way, in every round of the loop).
#pragma unroll
  for (int x = 0; x < SETS; ++x) {
    if constexpr (!STEP)
#pragma unroll
      for (int nd = 0; nd < ND; ++nd) asm volatile("" : "+v"(q[x][nd]));
    if constexpr (MORE) asm volatile("" : "+v"(slope[x]));
  }

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

  // ---- units; the keys of the next one are under way while the values of this one are used
  if (i < mine.stop) {
    unit = next;
    next = look(i + NW);
  }
  for (; i < mine.stop; i += NW) {
    // tokens low .. high - 1 of the unit get weight
    const int low = mine.seen - 32 * unit.u, high = there ? n - 32 * unit.u : 0;
    const bool whole = low <= 0 && high >= 32;
    if constexpr (STEP) {
      if (unit.u == (n - 1) / 32) {                                     // the new row takes its place, here and in the cache
        const int t = (n - 1) % 32, e = 4 * (t / 16) + t % 4;
        const bool store = there && g == 0;
        if (head == t % 16) {
#pragma unroll
          for (int nd = 0; nd < ND; ++nd) {
            const u32x4 x = *reinterpret_cast<const u32x4*>(fresh + K_NEW * D + 32 * nd + 8 * a);
            if (t < 16) k[nd] = x; else k[ND + nd] = x;
            if (store) *reinterpret_cast<u32x4*>(P.k_pages + off + k_fp_index(t, 32 * nd + 8 * a, ND)) = x;
          }
        }
        if (a == t % 16 / 4) {
          const uint32_t mask = e & 1 ? 0xFFFF0000u : 0xFFFFu;
#pragma unroll
          for (int c = 0; c < NT; ++c) {
            const uint16_t x = fresh[V_NEW * D + 16 * c + head];
#pragma unroll
            for (int w = 0; w < 4; ++w)
              if (w == e / 2) v[c][w] = (v[c][w] & ~mask) | ((x * 0x10001u) & mask);
            if (store) P.v_pages[off + v_fp_index(t, 16 * c + head, NT)] = x;
          }
        }
      }
    }
    f32x4 s0[SETS], s1[SETS];
#pragma unroll
    for (int x = 0; x < SETS; ++x) s0[x] = s1[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int nd = 0; nd < ND; ++nd)
#pragma unroll
      for (int x = 0; x < SETS; ++x) {
        s0[x] = mfma<BF16>(k[nd], q[x][nd], s0[x]);
        s1[x] = mfma<BF16>(k[ND + nd], q[x][nd], s1[x]);
      }
    const int u = unit.u;
    load_k();
    unit = next;
    next = look(i + 2 * NW);
    if (!whole) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int w = 0; w < 4; ++w) {                                   // values without weight may be anything
          const int t0 = 16 * (w / 2) + 4 * a + 2 * (w % 2);
          v[t][w] &= (t0 >= low && t0 < high ? 0xFFFFu : 0u) | (t0 + 1 >= low && t0 + 1 < high ? 0xFFFF0000u : 0u);
        }
    }
    __amdgpu_buffer_rsrc_t logits;
    if constexpr (MORE) logits = buffer(P.logits + ((bh * (P.max_pages << (P.log_p - 5)) + u) * (2 * P.gh) + g * P.hb) * 16, P.logits ? P.gh * 128 : 0);
    float z[SETS][8];
#pragma unroll
    for (int x = 0; x < SETS; ++x) {
#pragma unroll
      for (int e = 0; e < 8; ++e) z[x][e] = product(e < 4 ? s0[x][e] : s1[x][e - 4], P.scale);
      if constexpr (MORE) {
        if (P.cap > 0.f)
#pragma unroll
          for (int e = 0; e < 8; ++e) z[x][e] = product(tanh_of(z[x][e]), P.cap);
        if (P.slopes) {
          const float ahead = (float)(32 * u + 4 * a - (n - 1));
#pragma unroll
          for (int e = 0; e < 8; ++e) z[x][e] = fmaf(slope[x], ahead + (float)(16 * (e / 4) + e % 4), z[x][e]);
        }
      }
      if (!whole)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int t = 16 * (e / 4) + 4 * a + e % 4;
          if (t < low || t >= high) z[x][e] = -INFINITY;
        }
      if constexpr (MORE) {                                             // for the weights (heads that are not there: not stored)
        if (P.weights) {
          if (16 * x + head < heads) {
            float* to = z_lds + ((u - mine.seen / 32) * 2 * heads + 16 * x + head) * 16 + 4 * a;
            *reinterpret_cast<f32x4*>(to) = f32x4{z[x][0], z[x][1], z[x][2], z[x][3]};
            *reinterpret_cast<f32x4*>(to + 16 * heads) = f32x4{z[x][4], z[x][5], z[x][6], z[x][7]};
          }
        }
        const int at = 16 * x + head < heads ? (16 * x + head) * 64 + 16 * a : 0x7FFFF000;
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{z[x][0], z[x][1], z[x][2], z[x][3]}), logits, at, 0, 0);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{z[x][4], z[x][5], z[x][6], z[x][7]}), logits, at, P.gh * 64, 0);
      }
      float top = z[x][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top = fmaxf(top, z[x][e]);
      look_up(x, top);
      const float m0 = m[x] == -INFINITY ? 0.f : m[x];                  // (none of a unit without a page)
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(z[x][e] - m0);
        l[x] += p[e];
      }
#pragma unroll
      for (int y = 0; y < (BF16 ? 3 : 2); ++y) {                        // a bf16 operand keeps 8 bits, an fp16 one 11
        const u32x4 pb = operand<BF16>(p);
        take<BF16>(p, pb);
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[x][t] = mfma<BF16>(v[t], pb, acc[x][t]);
      }
    }
    load_v();
  }

  __shared__ float2 stats[MORE ? 16 * SETS : 1];
  join_parts<D, NW, SETS>(o_lds, P.hb, heads, part, parts, first_slot, P.counters + (int64_t)(b * per_row + j) * CTR8, P.partials, acc, m, l,
                          [&](int hd, int c, f32x4 o, float top, float sum) {
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    *reinterpret_cast<u32x2*>(P.out + (head0 + hd) * D + c) =
        u32x2{pair_as<BF16>(o[0] * inv, o[1] * inv), pair_as<BF16>(o[2] * inv, o[3] * inv)};
    if constexpr (MORE)
      if (c == 0) {
        stats[hd] = make_float2(top, inv);
        if (P.stats) *reinterpret_cast<float2*>(P.stats + 2 * (head0 + hd)) = make_float2(top, inv);
      }
  });
  if constexpr (MORE) {
    if (!P.weights) return;                            // (else parts == 1 and groups == 1)
    __syncthreads();
    const int first = mine.seen / 32 * 32;
    float* w = P.weights + (((int64_t)rb * P.Hkv + h) * P.max_pages << P.log_p);
    for (int t = first + 4 * threadIdx.x; t < n; t += 256 * NW)
      add_weights<STEP>(w + t, t, n, heads, [&](int g) { return stats[g]; }, z_lds + (t - first) / 16 * (16 * heads) + t % 16);
  }
}

template <int MODE, bool STEP, bool MORE>
hipError_t attn_paged(const ShapePaged& s, const AttnPagedParams& p, const Rows8<MODE>& rows, const Plan8& plan, hipStream_t st) {
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(plan.blocks), dim3(64 * plan.waves), lds_bytes8(plan.waves, plan.hb, s.d) + p.logits_lds, st, p, rows);
  };
  auto with = [&](auto bf16, auto waves, auto sets) {
    constexpr bool T = decltype(bf16)::value;
    constexpr int NW = decltype(waves)::value, SETS = decltype(sets)::value;
    if (s.d == 64) return go(attn_paged_kernel<T, 64, NW, SETS, MODE, STEP, MORE>);
    if (s.d == 96) return go(attn_paged_kernel<T, 96, NW, SETS, MODE, STEP, MORE>);
    go(attn_paged_kernel<T, 128, NW, SETS, MODE, STEP, MORE>);
  };
  auto with_type = [&](auto bf16) {
    const std::integral_constant<int, 1> one;
    if (plan.hb > 16) return with(bf16, std::integral_constant<int, 4>{}, std::integral_constant<int, 2>{});
    if constexpr (MODE == ROWS_LISTED)                                  // (no plan has 16 for rows that are alike, or for larger heads)
      if (plan.waves == 16) return go(attn_paged_kernel<decltype(bf16)::value, 64, 16, 1, MODE, STEP, MORE>);
    if (plan.waves == 8) return with(bf16, std::integral_constant<int, 8>{}, one);
    with(bf16, std::integral_constant<int, 4>{}, one);
  };
  if (s.bf16) with_type(std::true_type{}); else with_type(std::false_type{});
  return launch_status("attn_paged");
}

// One source file each.
#define LQ_ATTN_PAGED(MODE, STEP, MORE) \
  template hipError_t attn_paged<MODE, STEP, MORE>(const ShapePaged&, const AttnPagedParams&, const Rows8<MODE>&, const Plan8&, hipStream_t);

}  // namespace lq
