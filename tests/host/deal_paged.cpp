// Plans of attention over the paged cache for random batches, dealt as the kernel deals them: every unit of 32 tokens that holds
// one with weight is taken once for every (row, kv head, head group), partial results have room of their own, no workgroup asks
// for more LDS than a launch may have, and what a unit's place in the pool is computed from stays within pool and table,
// whatever the table's entries are.
#include <math.h>
#include <stdio.h>
#include <stdlib.h>

#include <map>
#include <random>
#include <set>
#include <tuple>
#include <vector>

#include "lq_plan_paged.h"

using namespace lq;

#define CHECK(c)                                                 \
  do {                                                           \
    if (!(c)) {                                                  \
      printf("line %d: %s (case %d)\n", __LINE__, #c, the_case); \
      exit(1);                                                   \
    }                                                            \
  } while (0)

int main() {
  std::mt19937 rng(20261208);
  auto in = [&](int a, int b) { return (int)(a + rng() % (unsigned)(b - a + 1)); };
  auto log_in = [&](int b) { return (int)exp2(std::uniform_real_distribution<>(0, log2(b + 1.0))(rng)) - 1; };
  long split = 0, sets = 0, wide = 0, windows = 0, in_lds = 0;
  for (int the_case = 0; the_case < 3000; ++the_case) {
    ShapePaged s{};
    const int ds[] = {64, 96, 128}, Ps[] = {32, 64, 128}, ghs[] = {1, 2, 3, 4, 7, 8, 16, 17, 24, 32, 33, 71};
    s.B = 1 + log_in(the_case % 10 ? 80 : 400);
    s.Hkv = 1 + log_in(the_case % 7 ? 16 : 200);
    s.gh = ghs[in(0, 11)];
    s.Hq = s.gh * s.Hkv;
    s.d = ds[in(0, 2)];
    s.P = Ps[in(0, 2)];
    const int log_p = s.P == 32 ? 5 : s.P == 64 ? 6 : 7;
    const bool step = in(0, 1);
    const int longest = 1 + log_in(the_case % 5 ? 20000 : 300000);
    s.max_pages = (longest + s.P - 1) / s.P + in(0, 3);
    s.n_pages = 1 + log_in(1 << (31 - log_p - 1));
    if ((int64_t)s.B * s.Hkv * ((s.gh + 15) / 16) * (s.cap() / 16 + 8) > 4000000) continue;
    const int window = in(0, 2) ? 0 : 1 + log_in(longest);
    std::vector<Row8> rows(s.B);
    const bool alike = in(0, 2) == 0;
    for (int b = 0; b < s.B; ++b) {
      const int n = alike && b ? rows[0].n : the_case % 3 ? in(step, longest) : std::min(longest, step + log_in(longest));
      rows[b] = Row8{n, 0, 1, in(0, 1) * s.B + b};
    }
    std::vector<int> lengths(s.B);
    for (int b = 0; b < s.B; ++b) lengths[b] = rows[b].n;
    PlanPaged plan;
    s.weighted = in(0, 1);
    bool same = true;
    for (int b = 1; b < s.B; ++b) same = same && lengths[b] == lengths[0];
    same = plan_paged(s, window, step, same, rows.data(), s.B, &plan);
    const Plan8 p = plan.deal;
    const int sets_of = p.hb > 16 ? 2 : 1, staged = step ? (16 * sets_of + 2) * s.d * 2 : 0;
    CHECK(lds_bytes8(p.waves, p.hb, s.d) + staged <= 65536);
    CHECK(p.waves == 4 || (p.hb <= 16 && (p.waves == 8 || (p.waves == 16 && !same && s.d == 64))));
    CHECK(p.hb <= 32 && p.groups * p.hb >= s.gh && (p.groups - 1) * p.hb < s.gh);
    // logits in LDS: room for every row's, of items that are neither split nor shared, and a second workgroup of 4 wavefronts
    if (plan.logits_lds) {
      CHECK(s.weighted && p.groups == 1);
      for (Row8& r : rows) {
        const PartPaged all = part_paged(r.n, window, 0, 1);
        CHECK(r.parts == 1 && (int64_t)(all.stop - all.pos) * 32 * s.gh * 4 <= plan.logits_lds);
      }
      const int all = lds_bytes8(p.waves, p.hb, s.d) + staged + 512 + plan.logits_lds;
      CHECK(all <= LDS_OF_CU && (p.waves > 4 || 2 * all <= LDS_OF_CU));
      ++in_lds;
    }
    const int per_row = s.Hkv * p.groups;
    std::set<int> slots;
    std::map<int, int> row_of;
    for (int i = 0; i < s.B; ++i) row_of[rows[i].x] = i;
    std::vector<int> seen_rows(s.B, 0);
    for (int i = 0; i < s.B; ++i) {
      const Row8 r = rows[i];
      const int b = r.b < s.B ? r.b : r.b - s.B;
      seen_rows[b] += 1;
      CHECK(r.n == lengths[b] && r.parts >= 1 && r.parts <= 256);
      if (same) CHECK(r.x == rows[0].x + i * per_row * r.parts && r.parts == rows[0].parts);
      std::vector<std::vector<int>> taken(per_row, std::vector<int>((r.n + 31) / 32 + 1, 0));
      for (int local = 0; local < per_row * r.parts; ++local) {
        const Pair8 of = pair8(local, p.groups, s.Hkv * r.parts);
        const int h = of.pair / r.parts, part = of.pair - h * r.parts, j = h * p.groups + of.g;
        CHECK(h < s.Hkv && of.g < p.groups && of.g * p.hb < s.gh);
        if (r.parts > 1) {
          const int slot = r.x + j * r.parts + part;
          CHECK(slot < MAX_PARTS8 && slots.insert(slot).second);
          ++split;
        }
        const PartPaged mine = part_paged(r.n, window, part, r.parts);
        const int len = mine.stop - mine.pos, turn = len > 0 ? in(0, len - 1) : 0;
        for (int w = 0; w < p.waves; ++w)
          for (int k = mine.pos + w; k < mine.stop; k += p.waves) {
            const int u = turned_paged(mine, k, turn);
            CHECK(u >= mine.pos && u < mine.stop && u >= 0 && 32 * u < r.n && 32 * u + 31 >= mine.seen);
            CHECK(u >> (log_p - 5) < s.max_pages);
            taken[j][u] += 1;
          }
      }
      const int first = first_seen(r.n, window) / 32;
      for (auto& t : taken)
        for (int u = 0; u < (r.n + 31) / 32; ++u) CHECK(t[u] == (u >= first));
      if (window && r.n > window) ++windows;
    }
    for (int x : seen_rows) CHECK(x == 1);
    sets += p.hb > 16;
    wide += p.waves > 4;
    // places in the pool
    const int64_t elements = (int64_t)s.n_pages * s.Hkv * s.P * s.d;
    for (int k = 0; k < 50; ++k) {
      const int ids[] = {in(-5, 5), (int)rng(), s.n_pages - 1, s.n_pages, in(0, s.n_pages - 1)};
      const int id = ids[in(0, 4)];
      CHECK(is_page(id, s.n_pages) == (id >= 0 && id < s.n_pages));
      if (!is_page(id, s.n_pages)) continue;
      const int h = in(0, s.Hkv - 1), u = in(0, s.cap() / 32 - 1);
      const int64_t off = unit_offset(id, s.Hkv, h, log_p, u, s.d);
      CHECK(off >= 0 && off + 32 * s.d <= elements && off % (32 * s.d) == 0);
      CHECK(off / ((int64_t)s.Hkv * s.P * s.d) == id && off / (s.P * s.d) % s.Hkv == h && off / (32 * s.d) % (s.P / 32) == u % (s.P / 32));
    }
  }
  printf("%ld parts, %ld plans of two sets, %ld of more than 4 wavefronts, %ld rows behind a window, %ld with logits in LDS\n", split, sets, wide, windows, in_lds);
  return in_lds > 100 && split > 1000 && sets > 50 && wide > 50 && windows > 1000 ? 0 : 1;
}
