// What attention over the 8-bit and the paged cache share: operands, the softmax's reference, and how the wavefronts of a
// workgroup and the workgroups of an item are joined.
#pragma once
#include <hip/hip_runtime.h>

#include "lq_deal8.h"
#include "lq_device.h"
#include "lq_quant8.h"

namespace lq {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float BIAS = 10.f, SLACK = 5.f;
constexpr int DEVICE_COHERENT = 16;          // cache policy of partial results: past the caches of a die

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

// eight probabilities as an operand, and what is left of them without it (exact)
template <bool BF16>
__device__ __forceinline__ u32x4 operand(const float* p) {
  return u32x4{pair_as<BF16>(p[0], p[1]), pair_as<BF16>(p[2], p[3]), pair_as<BF16>(p[4], p[5]), pair_as<BF16>(p[6], p[7])};
}
template <bool BF16>
__device__ __forceinline__ void take(float* p, u32x4 op) {
#pragma unroll
  for (int e = 0; e < 8; ++e) p[e] -= t2f<BF16>((uint16_t)(op[e / 2] >> (16 * (e & 1))));
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

// A logit, rounded: left to itself the compiler may join it to the subtraction behind it, where the reference was rounded.
__device__ __forceinline__ float product(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}
// What is subtracted from logits whose largest is t: t - BIAS, but never so far below t (where fp32 is coarser than that, from
// 2^27 on) that a probability would leave fp16.
__device__ __forceinline__ float reference(float t) {
  const float m = t - BIAS;
  return t - m > BIAS + SLACK ? t : m;
}

__device__ __forceinline__ float weight(float m, float top) { return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top); }

// The end of a kernel: the results of NW wavefronts (acc, m, l: the columns of SETS sets of 16 heads) and of the `parts`
// workgroups of an item become outputs; write_out(head, channel, four sums, reference, sum) is called by the last to come.
// o_lds: lds_bytes8 bytes; ctr: the item's counters; partials: room for results, the item's from first_slot on.
template <int D, int NW, int SETS, typename WriteOut>
__device__ __forceinline__ void join_parts(float* o_lds, int hb, int heads, int part, int parts, int first_slot, int* ctr, float* partials,
                                           f32x4 (&acc)[SETS][D / 16], float (&m)[SETS], float (&l)[SETS], WriteOut write_out) {
  constexpr int NT = D / 16, PITCH = D + 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int a = lane / 16, head = lane % 16;
  // ---- the workgroup's wavefronts together, set by set
  const int slot = hb * PITCH;                       // floats of a partial result
  auto partial = [&](int k) { return partials + (int64_t)(first_slot + k) * slot; };
  auto store_partial = [&](float* to, int hd, int c, f32x4 o, float top, float sum) {
    const __amdgpu_buffer_rsrc_t rs = buffer(to, slot * 4);
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, o), rs, (hd * PITCH + c) * 4, 0, DEVICE_COHERENT);
    if (c == 0)
      __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(top), __float_as_uint(sum)}, rs, (hd * PITCH + D) * 4, 0, DEVICE_COHERENT);
  };
  const int rows_lds = hb < 16 ? hb : 16;          // heads of a set that LDS has room for
#pragma unroll
  for (int x = 0; x < SETS; ++x) {
    const int in_set = heads - 16 * x < 16 ? heads - 16 * x : 16;
    if (x > 0) __syncthreads();                        // the set before is read
    l[x] = head_sum(l[x]);
    if (head < in_set) {
      float* mine = o_lds + (wave * rows_lds + head) * PITCH;
#pragma unroll
      for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4*>(mine + 16 * t + 4 * a) = acc[x][t];
      if (a == 0) {
        mine[D] = m[x];
        mine[D + 1] = l[x];
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < in_set * (D / 4); i += 64 * NW) {
      const int hd = i / (D / 4), c = 4 * (i % (D / 4));
      float top = -INFINITY, sum = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) top = fmaxf(top, o_lds[(w * rows_lds + hd) * PITCH + D]);
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float* row = o_lds + (w * rows_lds + hd) * PITCH;
        const float f = weight(row[D], top);
        sum = fmaf(row[D + 1], f, sum);
        o += *reinterpret_cast<const f32x4*>(row + c) * f;
      }
      if (parts == 1) write_out(16 * x + hd, c, o, top, sum); else store_partial(partial(part), 16 * x + hd, c, o, top, sum);
    }
  }
  if (parts == 1) return;

  // ---- the workgroups of an item together: the last one to come joins them, nobody waits.  Many are joined by sixteens first
  // (2 kv heads of 43162 tokens in 128 parts: 19.0 -> 11.8 us).
  constexpr int T = 64 * NW, BATCH = 8, FAN = FAN8;
  __shared__ int last;
  const int cols = heads * (D / 4), shares = cols < T ? T / cols : 1;
  const bool many = parts > FAN * shares;
  for (bool sixteens = many;; sixteens = false) {
    const bool again = many && !sixteens;              // the second time: one result in sixteen, in room of its own
    const int group = sixteens ? part / FAN : 0, stride = again ? FAN : 1;
    const int count = again ? (parts + FAN - 1) / FAN : sixteens && parts - group * FAN > FAN ? FAN : parts - group * FAN;
    float* base = partial(group * FAN) + (again ? (int64_t)MAX_PARTS8 * slot : 0);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_s_waitcnt(0);                     // the partial results are where the other dies see them
    __syncthreads();
    if (threadIdx.x == 0) {
      int* c = ctr + (sixteens ? 1 + group : 0);
      last = __hip_atomic_fetch_add(c, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == count - 1;
      if (last) __hip_atomic_store(c, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // for the next launch
    }
    __syncthreads();
    if (!last) return;
    auto joined = [&](int hd, int c, f32x4 o, float top, float sum) {
      if (sixteens) store_partial(base + (int64_t)MAX_PARTS8 * slot, hd, c, o, top, sum); else write_out(hd, c, o, top, sum);
    };
    // Every thread takes four channels of a head and, where there are more threads than those, a share of the parts; eight
    // parts' loads are under way at a time.
    const __amdgpu_buffer_rsrc_t rs = buffer(base, ((count - 1) * stride + 1) * slot * 4);
    for (int i = threadIdx.x; i < cols * shares; i += T) {
      const int share = i / cols, col = i - share * cols, hd = col / (D / 4), c = 4 * (col % (D / 4));
      float top = -INFINITY, sum = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
      for (int k0 = share; k0 < count; k0 += BATCH * shares) {
        u32x4 y[BATCH];
        u32x2 ml[BATCH];
#pragma unroll
        for (int e = 0; e < BATCH; ++e) {              // behind the last part: zeros, not read
          const int k = k0 + e * shares, off = k < count ? (k * stride * slot + hd * PITCH) * 4 : 0x7FFFF000;
          ml[e] = __builtin_amdgcn_raw_buffer_load_b64(rs, off + D * 4, 0, DEVICE_COHERENT);
          y[e] = __builtin_amdgcn_raw_buffer_load_b128(rs, off + c * 4, 0, DEVICE_COHERENT);
        }
        float now = top;
#pragma unroll
        for (int e = 0; e < BATCH; ++e)
          if (k0 + e * shares < count) now = fmaxf(now, __uint_as_float(ml[e][0]));
        const float f = weight(top, now);
        sum *= f;
        o *= f;
        top = now;
#pragma unroll
        for (int e = 0; e < BATCH; ++e) {
          const float w = k0 + e * shares < count ? weight(__uint_as_float(ml[e][0]), now) : 0.f;
          sum = fmaf(__uint_as_float(ml[e][1]), w, sum);
          o += __builtin_bit_cast(f32x4, y[e]) * w;
        }
      }
      if (shares > 1) {                                // (then this is the thread's only column)
        *reinterpret_cast<f32x4*>(o_lds + 4 * i) = o;
        o_lds[4 * T + i] = top;
        o_lds[5 * T + i] = sum;
      } else {
        joined(hd, c, o, top, sum);
      }
    }
    if (shares > 1) {
      __syncthreads();
      const int col = threadIdx.x;
      if (col < cols) {
        float top = -INFINITY, sum = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < shares; ++k) top = fmaxf(top, o_lds[4 * T + k * cols + col]);
        for (int k = 0; k < shares; ++k) {
          const float f = weight(o_lds[4 * T + k * cols + col], top);
          sum = fmaf(o_lds[5 * T + k * cols + col], f, sum);
          o += *reinterpret_cast<const f32x4*>(o_lds + 4 * (k * cols + col)) * f;
        }
        joined(col / (D / 4), 4 * (col % (D / 4)), o, top, sum);
      }
    }
    if (!sixteens) return;
  }
}

}  // namespace lq
