// Decode attention over the 8-bit cache.
//
// Per (row, kv head): logits s = scale * q . k over its tokens, p = softmax(s), o = sum p v, in one pass with the running
// maximum and sum of the softmax.  Both products are matrix instructions of 16 x 16 x 32 with up to 16 query heads of the kv
// head as the columns of one operand:
//   S^T = K Q^T   codes of keys, e4m3, which fp16 and bf16 hold exactly, against q as it came; the scale of a block is one
//                 factor of the fp32 logits of its tokens
//   O^T = V^T P^T codes of values as fp16 against the probabilities, rounded to fp16; the scale of a block is one factor of
//                 the fp32 sum over a unit of 32 tokens, which is then added to the running sums
// A lane of S^T holds four tokens of one head, which are the elements it owes to P^T (tokens permuted inside a unit, as they
// are stored), and the result of O^T has the heads in the same lanes: nothing but the maximum crosses lanes.
// Probabilities are 2^(s' - m + 10) with s' = s log2(e) and m the largest s' when it was last looked up, at most 5 behind:
// they stay below 2^15, and one 2^-24 of the largest still is a normal fp16 number.  The rounding to fp16 (2^-12 of each, unbiased) is
// left out of the sum of the probabilities, which is kept in fp32.
//
// Bound by the bytes of the codes.  Work is dealt along one line (Plan8), inside a workgroup unit by unit to its wavefronts.
#include <type_traits>

#include "lq_cache8.h"
#include "lq_device.h"
#include "lq_internal.h"

namespace lq {

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float BIAS = 10.f, SLACK = 5.f;
constexpr int DEVICE_COHERENT = 16;          // cache policy of partial results: past the caches of a die

struct Attn8Params {
  const uint16_t* q;
  uint16_t* out;
  const uint8_t *k_codes, *v_codes;
  const float *k_scale, *v_scale;
  uint16_t *k_tail, *v_tail;
  const uint16_t *k_new, *v_new;             // fused step: the token that belongs to the last row of the tail; else null
  int* counters;
  float* partials;
  const Row8* rows;
  float scale;                               // softmax scale times log2(e)
  int B, Hkv, gh, groups, hb, log_g, cap;
  int n, work;                               // ROWS_SAME: tokens and work of every row
  int total, quota;
};

__device__ __forceinline__ u32x4 load16(__amdgpu_buffer_rsrc_t rs, int off) {
  return __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, 0);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000);
}

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
template <bool BF16>
__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
}
template <bool BF16>
__device__ __forceinline__ uint32_t pair_as(float a, float b) {
  if constexpr (BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
  else return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), half2v));
}

// over the four lanes of a head (lane % 16)
__device__ __forceinline__ float head_max(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const uint32_t w = __float_as_uint(v);
  const auto s = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float head_sum(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  const uint32_t w = __float_as_uint(v);
  const auto s = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

__device__ __forceinline__ float weight(float m, float top) { return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top); }

template <bool BF16, int D, int NW, int MODE>
__global__ void __launch_bounds__(64 * NW) attn8_kernel(const Attn8Params P, const Rows8<MODE> S) {
  (void)S;
  constexpr int ND = D / 32, NT = D / 16, PITCH = D + 4, UNIT = 32 * D;   // UNIT: bytes of a unit's codes
  extern __shared__ __align__(16) float o_lds[];                     // [NW][hb][PITCH], m and l of a head behind its row
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int a = lane / 16, head = lane % 16;
  const int per_row = P.Hkv * P.groups;                // items of a row
  int x = blockIdx.x * P.quota;
  const int end = x + P.quota < P.total ? x + P.quota : P.total;
  bool first = true;

  // the item at x, and the place in it
  int b, j, n, work, pos;
  const Row8Ptr rows = MODE == ROWS_SAME ? nullptr : rows_ptr(P.rows, sizeof(Attn8Params));
  auto work_of = [&](int tokens) {
    const int full = tokens >> P.log_g << P.log_g, u = full / 32 + 2 * ((tokens - full + 31) / 32);
    return u > 0 ? u : 1;
  };
  if constexpr (MODE == ROWS_SAME) {
    n = P.n;
    work = P.work;
    const int item = x / work;
    pos = x - item * work;
    b = item / per_row;
    j = item - b * per_row;
  } else {
    int before = 0;                                    // rows that begin at or before x
    for (int i0 = 0; i0 < P.B; i0 += 64) {
      const int i = i0 + lane;
      const bool le = i < P.B && rows[i].x * per_row <= x;
      const int c = __popcll(__ballot(le));
      before += c;
      if (c < 64) break;
    }
    b = __builtin_amdgcn_readfirstlane(before - 1);
    n = rows[b].n;
    work = work_of(n);
    const int local = x - rows[b].x * per_row;
    j = local / work;
    pos = local - j * work;
  }

  while (x < end) {
    const int to = pos + (end - x) < work ? pos + (end - x) : work;       // [pos, to) of this item is ours
    const int h = j / P.groups, g = j - h * P.groups;
    const int64_t bh = (int64_t)b * P.Hkv + h;
    const int heads = P.hb < P.gh - g * P.hb ? P.hb : P.gh - g * P.hb;
    const int64_t head0 = bh * P.gh + g * P.hb;
    const int full = n >> P.log_g << P.log_g, codes = full / 32, rest = n - full;

    u32x4 q[ND];
    {
      const __amdgpu_buffer_rsrc_t rs = buffer(P.q + head0 * D, heads * D * 2);   // absent heads: zeros
#pragma unroll
      for (int nd = 0; nd < ND; ++nd) q[nd] = load16(rs, head * D * 2 + a * 16 + nd * 64);
    }
    f32x4 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;

    // a lane's largest logit of a unit: when it is over the reference by more than SLACK anywhere, a new reference
    auto look_up = [&](float top) {
      if (__any(top > m + SLACK)) {
        const float now = fmaxf(m, head_max(top)), f = weight(m, now);
        m = now;
        l *= f;
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[t] *= f;
      }
    };

    // ---- codes
    const int stop = to < codes ? to : codes;
    const __amdgpu_buffer_rsrc_t rk = buffer(P.k_codes + bh * P.cap * D, stop * UNIT);   // behind the last unit: no reads
    const __amdgpu_buffer_rsrc_t rv = buffer(P.v_codes + bh * P.cap * D, stop * UNIT);
    const float* ks = P.k_scale + bh * (P.cap >> P.log_g);
    const float* vs = P.v_scale + bh * (P.cap >> P.log_g);
    struct Unit { u32x4 k[ND], v[ND]; float ks, vs; };
    auto load = [&](Unit& u, int i) {
#pragma unroll
      for (int nd = 0; nd < ND; ++nd) u.k[nd] = load16(rk, i * UNIT + lane * 16 + nd * 1024);
#pragma unroll
      for (int nd = 0; nd < ND; ++nd) u.v[nd] = load16(rv, i * UNIT + lane * 16 + nd * 1024);
      const int block = (i < stop ? i : stop - 1) >> (P.log_g - 5);
      u.ks = ks[block];
      u.vs = vs[block];
    };
    auto attend = [&](const Unit& u) {
      f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
      for (int nd = 0; nd < ND; ++nd) {
        s0 = mfma<BF16>(codes_as<BF16>(u.k[nd][0], u.k[nd][1]), q[nd], s0);
        s1 = mfma<BF16>(codes_as<BF16>(u.k[nd][2], u.k[nd][3]), q[nd], s1);
      }
      const float c = u.ks * P.scale;
      look_up(fmaxf(fmaxf(fmaxf(s0[0], s0[1]), fmaxf(s0[2], s0[3])), fmaxf(fmaxf(s1[0], s1[1]), fmaxf(s1[2], s1[3]))) * c);
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(fmaf(e < 4 ? s0[e] : s1[e - 4], c, BIAS - m));
        l += p[e];
      }
      const u32x4 pb = {pair_as<false>(p[0], p[1]), pair_as<false>(p[2], p[3]), pair_as<false>(p[4], p[5]), pair_as<false>(p[6], p[7])};
#pragma unroll
      for (int nd = 0; nd < ND; ++nd) {
        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
        const f32x4 o0 = mfma<false>(codes_as<false>(u.v[nd][0], u.v[nd][1]), pb, zero);
        const f32x4 o1 = mfma<false>(codes_as<false>(u.v[nd][2], u.v[nd][3]), pb, zero);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[2 * nd][e] = fmaf(o0[e], u.vs, acc[2 * nd][e]);
          acc[2 * nd + 1][e] = fmaf(o1[e], u.vs, acc[2 * nd + 1][e]);
        }
      }
    };
    if (pos + wave < stop) {
      Unit u0, u1;
      int i = pos + wave;
      load(u0, i);
      while (true) {
        load(u1, i + NW);
        attend(u0);
        i += NW;
        if (i >= stop) break;
        load(u0, i + NW);
        attend(u1);
        i += NW;
        if (i >= stop) break;
      }
    }

    // ---- rows of the tail, from the last wavefront down
    for (int i = NW - 1 - wave; 32 * i < rest; i += NW) {
      const int at = codes + 2 * i;
      if (at < pos || at >= to) continue;
      uint16_t* k_tail = P.k_tail + (bh << P.log_g) * D;
      uint16_t* v_tail = P.v_tail + (bh << P.log_g) * D;
      if (P.k_new && 32 * i + 32 >= rest) {            // the new row first; every head group stores the same
        const int t = rest - 1;
        if (lane < D / 8)
          *reinterpret_cast<u32x4*>(k_tail + k_fp_index(t, 8 * lane, ND)) = *reinterpret_cast<const u32x4*>(P.k_new + bh * D + 8 * lane);
        for (int c = lane; c < D; c += 64) v_tail[v_fp_index(t, c, NT)] = P.v_new[bh * D + c];
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        __builtin_amdgcn_s_waitcnt(0);
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
      }
      const int live = rest - 32 * i < 32 ? rest - 32 * i : 32;
      f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
      for (int nd = 0; nd < ND; ++nd) {
        s0 = mfma<BF16>(*reinterpret_cast<const u32x4*>(k_tail + (((2 * i) * ND + nd) * 64 + lane) * 8), q[nd], s0);
        s1 = mfma<BF16>(*reinterpret_cast<const u32x4*>(k_tail + (((2 * i + 1) * ND + nd) * 64 + lane) * 8), q[nd], s1);
      }
      float z[8], top = -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        z[e] = 16 * (e / 4) + 4 * a + e % 4 < live ? (e < 4 ? s0[e] : s1[e - 4]) * P.scale : -INFINITY;
        top = fmaxf(top, z[e]);
      }
      look_up(top);
      float p[8], r[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(z[e] + (BIAS - m));
        l += p[e];
      }
      // a bf16 operand keeps 8 bits of a probability: the rest goes in as a second one
      const u32x4 pb = {pair_as<BF16>(p[0], p[1]), pair_as<BF16>(p[2], p[3]), pair_as<BF16>(p[4], p[5]), pair_as<BF16>(p[6], p[7])};
#pragma unroll
      for (int e = 0; e < 8; ++e) r[e] = p[e] - t2f<BF16>((uint16_t)(pb[e / 2] >> (16 * (e & 1))));
      const u32x4 pr = {pair_as<BF16>(r[0], r[1]), pair_as<BF16>(r[2], r[3]), pair_as<BF16>(r[4], r[5]), pair_as<BF16>(r[6], r[7])};
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        u32x4 v = *reinterpret_cast<const u32x4*>(v_tail + ((i * NT + t) * 64 + lane) * 8);
#pragma unroll
        for (int w = 0; w < 4; ++w) {                  // rows that are not there have weight 0, but may hold anything
          const int t0 = 16 * (w / 2) + 4 * a + 2 * (w % 2);
          v[w] &= (t0 < live ? 0xFFFFu : 0u) | (t0 + 1 < live ? 0xFFFF0000u : 0u);
        }
        acc[t] = mfma<BF16>(v, pb, acc[t]);
        if constexpr (BF16) acc[t] = mfma<BF16>(v, pr, acc[t]);
      }
    }

    // ---- the workgroup's wavefronts together
    l = head_sum(l);
    if (head < heads) {
      float* mine = o_lds + (wave * P.hb + head) * PITCH;
#pragma unroll
      for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4*>(mine + 16 * t + 4 * a) = acc[t];
      if (a == 0) {
        mine[D] = m;
        mine[D + 1] = l;
      }
    }
    __syncthreads();
    const bool whole = pos == 0 && to == work;
    const int slot = P.hb * PITCH;                     // floats of a partial result
    const __amdgpu_buffer_rsrc_t rp = buffer(P.partials + ((int64_t)blockIdx.x * 2 + (first ? 0 : 1)) * slot, slot * 4);
    auto write_out = [&](int hd, int c, f32x4 o, float sum) {
      const float inv = sum > 0.f ? 1.f / sum : 0.f;
      *reinterpret_cast<u32x2*>(P.out + (head0 + hd) * D + c) =
          u32x2{pair_as<BF16>(o[0] * inv, o[1] * inv), pair_as<BF16>(o[2] * inv, o[3] * inv)};
    };
    for (int i = threadIdx.x; i < heads * (D / 4); i += 64 * NW) {
      const int hd = i / (D / 4), c = 4 * (i % (D / 4));
      float top = -INFINITY, sum = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) top = fmaxf(top, o_lds[(w * P.hb + hd) * PITCH + D]);
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float* row = o_lds + (w * P.hb + hd) * PITCH;
        const float f = weight(row[D], top);
        sum = fmaf(row[D + 1], f, sum);
        o += *reinterpret_cast<const f32x4*>(row + c) * f;
      }
      if (whole) {
        write_out(hd, c, o, sum);
      } else {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, o), rp, (hd * PITCH + c) * 4, 0, DEVICE_COHERENT);
        if (c == 0)
          __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(top), __float_as_uint(sum)}, rp, (hd * PITCH + D) * 4, 0, DEVICE_COHERENT);
      }
    }

    // ---- the workgroups of an item together: the last one to come joins them, nobody waits
    if (!whole) {
      __shared__ int last;
      const int start = x - pos, w0 = start / P.quota, parts = (start + work - 1) / P.quota - w0 + 1;
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
      __builtin_amdgcn_s_waitcnt(0);                   // the partial results are where the other dies see them
      __syncthreads();
      if (threadIdx.x == 0) {
        int* ctr = P.counters + (int64_t)(b * per_row + j) * CTR8;
        last = __hip_atomic_fetch_add(ctr, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
        if (last) __hip_atomic_store(ctr, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // for the next launch
      }
      __syncthreads();
      if (last) {
        // w0 had the item as its last, the others as their first
        const float* base = P.partials + ((int64_t)w0 * 2) * slot;
        const __amdgpu_buffer_rsrc_t rs = buffer(base, parts * 2 * slot * 4);
        const int skip = start == w0 * P.quota ? 0 : slot;
        for (int i = threadIdx.x; i < heads * (D / 4); i += 64 * NW) {
          const int hd = i / (D / 4), c = 4 * (i % (D / 4));
          float top = -INFINITY, sum = 0.f;
          f32x4 o = {0.f, 0.f, 0.f, 0.f};
          for (int k = 0; k < parts; ++k) {
            const int off = (2 * k * slot + (k ? 0 : skip) + hd * PITCH) * 4;
            const u32x4 y = __builtin_amdgcn_raw_buffer_load_b128(rs, off + c * 4, 0, DEVICE_COHERENT);
            const u32x2 ml = __builtin_amdgcn_raw_buffer_load_b64(rs, off + D * 4, 0, DEVICE_COHERENT);
            const float now = fmaxf(top, __uint_as_float(ml[0]));
            const float f0 = weight(top, now), f1 = weight(__uint_as_float(ml[0]), now);
            sum = sum * f0 + __uint_as_float(ml[1]) * f1;
            o = o * f0 + __builtin_bit_cast(f32x4, y) * f1;
            top = now;
          }
          write_out(hd, c, o, sum);
        }
      }
    }
    __syncthreads();                                   // o_lds and `last` are free again

    x += to - pos;
    pos = 0;
    first = false;
    if (++j == per_row) {
      j = 0;
      ++b;
      if (MODE == ROWS_LISTED && x < end) {
        n = rows[b].n;
        work = work_of(n);
      }
    }
  }
}

template <int MODE>
hipError_t attn8(const Shape8& s, const Attn8Params& p, const Rows8<MODE>& rows, const Plan8& plan, hipStream_t st) {
  constexpr int NW = 4;
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(plan.blocks), dim3(64 * NW), NW * partial_floats8(plan.hb, s.d) * sizeof(float), st, p, rows);
  };
  auto with_type = [&](auto bf16) {
    constexpr bool T = decltype(bf16)::value;
    if (s.d == 64) return go(attn8_kernel<T, 64, NW, MODE>);
    if (s.d == 96) return go(attn8_kernel<T, 96, NW, MODE>);
    go(attn8_kernel<T, 128, NW, MODE>);
  };
  if (s.bf16) with_type(std::true_type{}); else with_type(std::false_type{});
  return launch_status("attn8");
}

}  // namespace

hipError_t launch_attn8(const Shape8& s, const lq_cache8& c, const void* q, float scale, void* out, void* ws, const Plan8& plan,
                        const void* k_new, const void* v_new, const RowArg8& rows, hipStream_t st) {
  Attn8Params p{(const uint16_t*)q, (uint16_t*)out, c.k_codes, c.v_codes, c.k_scale, c.v_scale, (uint16_t*)c.k_tail, (uint16_t*)c.v_tail,
                (const uint16_t*)k_new, (const uint16_t*)v_new, (int*)ws, (float*)((char*)ws + counter_bytes8(s)), nullptr,
                scale * 1.44269504088896340736f, s.B, s.Hkv, s.gh, plan.groups, plan.hb, log2_of(s.G), s.cap, rows.host[0].n,
                units8(rows.host[0].n, s.G), plan.total, plan.quota};
  if (rows.same) return attn8<ROWS_SAME>(s, p, Rows8<ROWS_SAME>{}, plan, st);
  Rows8<ROWS_LISTED> listed{};
  const hipError_t e = hand_over(rows, &listed, &p.rows, st);
  return e != hipSuccess ? e : attn8<ROWS_LISTED>(s, p, listed, plan, st);
}

}  // namespace lq
