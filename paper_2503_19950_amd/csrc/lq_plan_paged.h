// Planning a launch of attention over the paged cache (host).
#pragma once
#include "lq_deal_paged.h"
#include "lq_plan8.h"

namespace lq {

inline Shape8 shape8_of(const ShapePaged& s) { return Shape8{s.B, s.Hq, s.Hkv, s.d, s.P, s.cap(), s.gh, s.bf16}; }

// As for the 8-bit cache, whose unit of codes has half the bytes of a unit here.  rows: n tokens each; *most: the most of them
// that get weight.  What a step stages in LDS (its queries, the new key and value) counts towards what a workgroup may have.
inline bool plan_paged(const ShapePaged& s, int window, bool step, bool same, Row8* rows, int n_rows, Plan8* p, int* most) {
  int64_t tokens = 0;
  *most = 0;
  for (Row8* r = rows; r != rows + n_rows; ++r) {
    const int seen = first_seen(r->n, window);
    tokens += r->n - seen;
    *most = std::max(*most, r->n - seen);
    r->x = 2 * ((r->n + 31) / 32 - seen / 32);
  }
  const int staged = 64 + (step ? (16 * (s.gh > 16 ? 2 : 1) + 2) * s.d * 2 : 0);
  same = plan_work8(shape8_of(s), tokens * s.Hkv * s.d * 4, 65536 - staged, same, rows, n_rows, p);
  if (p->waves == 16 && s.d > 64) p->waves = 8;        // (the registers of 16 wavefronts do not hold a unit of these)
  return same;
}

}  // namespace lq
