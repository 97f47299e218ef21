// Planning a launch of attention over the paged cache (host).
#pragma once
#include "lq_deal_paged.h"
#include "lq_plan8.h"

namespace lq {

inline Shape8 shape8_of(const ShapePaged& s) { return Shape8{s.B, s.Hq, s.Hkv, s.d, s.P, s.cap(), s.gh, s.bf16}; }

struct PlanPaged {
  Plan8 deal;
  int most;            // the most tokens of a row that get weight
  int logits_lds;      // bytes of LDS for the logits of a weighted cache; 0: they go through memory (or there are none)
};

// As for the 8-bit cache, whose unit of codes has half the bytes of a unit here.  rows: n tokens each.  What a step stages in LDS
// (its queries, the new key and value) counts towards what a workgroup may have.
// A weighted cache's logits stay in LDS where no item is split and the longest row's fit, so that the workgroup adds the weights
// itself: 64 rows of up to 4096 tokens x 8 kv heads, 4 heads each: 87 us, through memory and a second launch 107 (83 without
// weights).  Workgroups of 4 wavefronts leave room for a second one on the compute unit.
constexpr int LDS_OF_CU = 160 * 1024;
inline bool plan_paged(const ShapePaged& s, int window, bool step, bool same, Row8* rows, int n_rows, PlanPaged* p) {
  int64_t tokens = 0;
  p->most = 0;
  for (Row8* r = rows; r != rows + n_rows; ++r) {
    const int seen = first_seen(r->n, window);
    tokens += r->n - seen;
    p->most = std::max(p->most, r->n - seen);
    r->x = 2 * ((r->n + 31) / 32 - seen / 32);
  }
  const int staged = 512 + (step ? (16 * (s.gh > 16 ? 2 : 1) + 2) * s.d * 2 : 0);
  Plan8& d = p->deal;
  same = plan_work8(shape8_of(s), tokens * s.Hkv * s.d * 4, 65536 - staged, same, rows, n_rows, &d);
  if (d.waves == 16 && s.d > 64) d.waves = 8;          // (the registers of 16 wavefronts do not hold a unit of these)
  p->logits_lds = 0;
  if (s.weighted && p->most && d.groups == 1) {
    int parts = 1;
    for (Row8* r = rows; r != rows + n_rows; ++r) parts = std::max(parts, r->parts);
    const int64_t bytes = ((int64_t)p->most + 62) / 32 * 32 * d.hb * 4;       // (a window may begin within a unit)
    if (parts == 1 && bytes + lds_bytes8(d.waves, d.hb, s.d) + staged <= LDS_OF_CU / (d.waves == 4 ? 2 : 1)) p->logits_lds = (int)bytes;
  }
  return same;
}

}  // namespace lq
