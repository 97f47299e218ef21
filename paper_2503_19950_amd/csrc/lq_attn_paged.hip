// Attention over the paged cache: which kernel, and the weights of a cache that keeps them.
#include "lq_attn_paged_args.h"
#include "lq_internal.h"

namespace lq {

namespace {

struct WeightsParams {
  const float *logits, *stats;
  float* weights;
  const Row8* rows;
  Row8 same;
  int B, Hkv, gh, cap, window;
};

// weights[t] += sum over a kv head's query heads of 2^(z - m) / l, z as attention left it.  Four tokens a thread; the newest
// one's weight is set by a step.  grid (1024 tokens each, Hkv, B)
constexpr int WEIGHTS_AT_ONCE = 1024;
template <int MODE, bool STEP>
__global__ void __launch_bounds__(256) weights_kernel(const WeightsParams P, const Rows8<MODE> S) {
  (void)S;
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  Row8 row = P.same;
  if constexpr (MODE == ROWS_LISTED) {
    const Row8Ptr r = rows_ptr(P.rows, sizeof(WeightsParams));
    row = Row8{r[blockIdx.z].n, 0, 1, r[blockIdx.z].b};
  } else {
    row.b += blockIdx.z;
  }
  const int b = row.b < P.B ? row.b : row.b - P.B, h = blockIdx.y;
  const int t = first_seen(row.n, P.window) / 32 * 32 + ((int)blockIdx.x * 256 + (int)threadIdx.x) * 4;
  if (t >= row.n) return;
  const int64_t head0 = ((int64_t)b * P.Hkv + h) * P.gh;
  const float* at = P.logits + (((int64_t)b * P.Hkv + h) * (P.cap / 16) + t / 16) * (P.gh * 16) + t % 16;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int g = 0; g < P.gh; ++g) {
    const float m = P.stats[2 * (head0 + g)], inv = P.stats[2 * (head0 + g) + 1];
    const f32x4 z = *reinterpret_cast<const f32x4*>(at + 16 * g);
    if (inv > 0.f)                                     // (else nothing had weight)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] = fmaf(__builtin_amdgcn_exp2f(z[e] - m), inv, sum[e]);
  }
  float* w = P.weights + ((int64_t)row.b * P.Hkv + h) * P.cap + t;
  const int fresh = STEP ? row.n - 1 - t : 4;          // of the four, the one that is new
  if (t + 4 <= row.n) {
    f32x4 x = *reinterpret_cast<const f32x4*>(w);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (e == fresh ? 0.f : x[e]) + sum[e];
    *reinterpret_cast<f32x4*>(w) = x;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (t + e < row.n) w[e] = (e == fresh ? 0.f : w[e]) + sum[e];
  }
}

template <int MODE>
hipError_t attend(const ShapePaged& s, const AttnPagedParams& p, const WeightsParams& w, const Rows8<MODE>& rows, const Plan8& plan,
                  bool step, int most, hipStream_t st) {
  const bool more = p.cap > 0.f || p.slopes || s.weighted;
  hipError_t e = step ? attn_paged<MODE, true, true>(s, p, rows, plan, st)
                      : more ? attn_paged<MODE, false, true>(s, p, rows, plan, st) : attn_paged<MODE, false, false>(s, p, rows, plan, st);
  if (e != hipSuccess || !s.weighted || !most) return e;
  const dim3 grid((most + 31 + WEIGHTS_AT_ONCE - 1) / WEIGHTS_AT_ONCE, s.Hkv, s.B);
  if (step) hipLaunchKernelGGL((weights_kernel<MODE, true>), grid, dim3(256), 0, st, w, rows);
  else hipLaunchKernelGGL((weights_kernel<MODE, false>), grid, dim3(256), 0, st, w, rows);
  return launch_status("weights");
}

}  // namespace

hipError_t launch_attn_paged(const ShapePaged& s, const lq_cache_paged& c, const ScoresArg& scores, const void* q, void* out, void* ws,
                             const Plan8& plan, const NewToken* step, int most, const RowArg8& rows, hipStream_t st) {
  const WorkspacePaged room = split_workspace(s, ws);
  const NewToken none{};
  const NewToken& x = step ? *step : none;
  AttnPagedParams p{(const uint16_t*)q, (uint16_t*)out, (uint16_t*)c.k_pages, (uint16_t*)c.v_pages, c.table, (const uint16_t*)x.k,
                    (const uint16_t*)x.v, x.rope, scores.slopes, room.logits, room.stats, room.counters, room.partials, nullptr,
                    scores.scale, scores.cap, scores.window, s.B, s.Hkv, s.gh, plan.groups, plan.hb, log2_of(s.P), s.n_pages, s.max_pages,
                    rows.host[0]};
  WeightsParams w{room.logits, room.stats, c.weights, nullptr, rows.host[0], s.B, s.Hkv, s.gh, s.cap(), scores.window};
  if (rows.same) return attend<ROWS_SAME>(s, p, w, Rows8<ROWS_SAME>{}, plan, step, most, st);
  Rows8<ROWS_LISTED> listed{};
  const hipError_t e = hand_over(rows, &listed, &p.rows, st);
  w.rows = p.rows;
  return e != hipSuccess ? e : attend<ROWS_LISTED>(s, p, w, listed, plan, step, most, st);
}

}  // namespace lq
