// Attention over the paged cache: which kernel, and the weights of a cache that keeps them.
#include <type_traits>

#include "lq_attn_paged_args.h"
#include "lq_internal.h"
#include "lq_weights.h"

namespace lq {

namespace {

struct WeightsParams {
  const float *logits, *stats;
  float* weights;
  const Row8* rows;
  Row8 same;
  int B, Hkv, gh, cap, window;
};

// The weights of rows whose items are split, from the logits that attention left in memory.  Four tokens a thread.
// grid (1024 tokens each, Hkv, B)
constexpr int WEIGHTS_AT_ONCE = 1024;
template <int MODE, bool STEP>
__global__ void __launch_bounds__(256) weights_kernel(const WeightsParams P, const Rows8<MODE> S) {
  (void)S;
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
  const int64_t bh = (int64_t)b * P.Hkv + h;
  const float2* stats = reinterpret_cast<const float2*>(P.stats) + bh * P.gh;
  add_weights<STEP>(P.weights + ((int64_t)row.b * P.Hkv + h) * P.cap + t, t, row.n, P.gh, [&](int g) { return stats[g]; },
                    P.logits + (bh * (P.cap / 16) + t / 16) * (P.gh * 16) + t % 16);
}

template <int MODE>
hipError_t attend(const ShapePaged& s, const AttnPagedParams& p, const WeightsParams& w, const Rows8<MODE>& rows, const Plan8& plan,
                  bool step, int most, hipStream_t st) {
  const bool more = p.cap > 0.f || p.slopes || s.weighted;
  auto go = [&](auto stepping, auto changed) {
    return attn_paged<MODE, decltype(stepping)::value, decltype(changed)::value>(s, p, rows, plan, st);
  };
  const std::true_type yes;
  const std::false_type no;
  const hipError_t e = step ? more ? go(yes, yes) : go(yes, no) : more ? go(no, yes) : go(no, no);
  if (e != hipSuccess || !s.weighted || p.weights || !most) return e;
  const dim3 grid((most + 31 + WEIGHTS_AT_ONCE - 1) / WEIGHTS_AT_ONCE, s.Hkv, s.B);
  if (step) hipLaunchKernelGGL((weights_kernel<MODE, true>), grid, dim3(256), 0, st, w, rows);
  else hipLaunchKernelGGL((weights_kernel<MODE, false>), grid, dim3(256), 0, st, w, rows);
  return launch_status("weights");
}

}  // namespace

hipError_t launch_attn_paged(const ShapePaged& s, const lq_cache_paged& c, const ScoresArg& scores, const void* q, void* out, void* ws,
                             const PlanPaged& plan, const NewToken* step, const RowArg8& rows, hipStream_t st) {
  const WorkspacePaged room = split_workspace(s, ws);
  const NewToken none{};
  const NewToken& x = step ? *step : none;
  AttnPagedParams p{(const uint16_t*)q, (uint16_t*)out, (uint16_t*)c.k_pages, (uint16_t*)c.v_pages, c.table, (const uint16_t*)x.k,
                    (const uint16_t*)x.v, x.rope, scores.slopes, plan.logits_lds ? nullptr : room.logits, plan.logits_lds ? nullptr : room.stats,
                    plan.logits_lds ? c.weights : nullptr, plan.logits_lds, room.counters, room.partials, nullptr,
                    scores.scale, scores.cap, scores.window, s.B, s.Hkv, s.gh, plan.deal.groups, plan.deal.hb, log2_of(s.P), s.n_pages, s.max_pages,
                    rows.host[0]};
  WeightsParams w{room.logits, room.stats, c.weights, nullptr, rows.host[0], s.B, s.Hkv, s.gh, s.cap(), scores.window};
  if (rows.same) return attend<ROWS_SAME>(s, p, w, Rows8<ROWS_SAME>{}, plan.deal, step, plan.most, st);
  Rows8<ROWS_LISTED> listed{};
  const hipError_t e = hand_over(rows, &listed, &p.rows, st);
  w.rows = p.rows;
  return e != hipSuccess ? e : attend<ROWS_LISTED>(s, p, w, listed, plan.deal, step, plan.most, st);
}

}  // namespace lq
