// Plans of attention over the 8-bit cache for random batches, dealt as the kernel deals them: every unit of codes and of the
// tail of every (row, kv head, head group) is taken once, partial results have room of their own within the workspace, and no
// workgroup asks for more LDS than a launch may have.
#include <math.h>
#include <stdio.h>
#include <stdlib.h>

#include <map>
#include <random>
#include <set>
#include <tuple>
#include <vector>

#include "lq_plan8.h"

using namespace lq;

#define CHECK(c)                                                                      \
  do {                                                                                \
    if (!(c)) {                                                                       \
      printf("line %d: %s (case %d)\n", __LINE__, #c, the_case);                      \
      exit(1);                                                                        \
    }                                                                                 \
  } while (0)

int main() {
  std::mt19937 rng(20250901);
  auto in = [&](int a, int b) { return (int)(a + rng() % (unsigned)(b - a + 1)); };
  auto log_in = [&](int b) { return (int)exp2(std::uniform_real_distribution<>(0, log2(b + 1.0))(rng)) - 1; };
  long large = 0, split = 0, sets = 0, sixteens = 0, uneven = 0;
  for (int the_case = 0; the_case < 4000; ++the_case) {
    Shape8 s{};
    const int ds[] = {64, 96, 128}, Gs[] = {32, 64, 128}, ghs[] = {1, 2, 3, 4, 7, 8, 15, 16, 17, 24, 31, 32, 33, 40, 64, 71};
    s.B = 1 + log_in(the_case % 10 ? 80 : 600);
    s.Hkv = 1 + log_in(the_case % 7 ? 16 : 300);
    s.gh = ghs[in(0, 15)];
    s.Hq = s.gh * s.Hkv;
    s.d = ds[in(0, 2)];
    s.G = Gs[in(0, 2)];
    const int log_g = s.G == 32 ? 5 : s.G == 64 ? 6 : 7;
    const bool step = in(0, 1);
    const int longest = 1 + log_in(the_case % 4 ? 9000 : 200000), kind = in(0, 4);
    std::vector<Row8> rows(s.B);
    for (int b = 0; b < s.B; ++b) {
      int n = kind == 0 ? longest : kind == 1 ? in(0, longest) : kind == 2 ? (b ? log_in(200) : longest) : kind == 3 ? log_in(longest)
              : s.G * in(0, 3) + (in(0, 1) ? s.G - 1 : 0);
      if (step && n == 0) n = 1;
      rows[b] = Row8{n, 0, 1, b};
    }
    std::vector<int> tokens(s.B);
    bool same = true;
    for (int b = 0; b < s.B; ++b) tokens[b] = rows[b].n, same = same && rows[b].n == rows[0].n;
    Plan8 p;
    same = plan8(s, same, step, rows.data(), s.B, &p);
    const int per_row = s.Hkv * p.groups;
    CHECK(p.groups * p.hb >= s.gh && (p.groups - 1) * p.hb < s.gh && p.hb <= 32);
    CHECK(p.groups <= head_groups8(s, false));
    const int most_hb = (s.gh + head_groups8(s, true) - 1) / head_groups8(s, true);
    CHECK(p.hb <= most_hb);                                           // the workspace has room for results of most_hb heads
    CHECK(p.waves == 4 || p.waves == 8 || p.waves == 16);
    CHECK(p.hb <= 16 || p.waves == 4);                                // what is built
    CHECK(lds_bytes8(p.waves, p.hb, s.d) <= 65536);
    std::set<int> slots, seen;
    std::map<std::tuple<int, int>, int> finished;                     // workgroups of an item
    int block = 0;
    for (int e = 0; e < s.B; ++e) {
      const Row8& r = rows[e];
      CHECK(r.x == block && r.parts >= 1);
      CHECK(r.n == tokens[r.b] && seen.insert(r.b).second);
      if (same) CHECK(r.parts == rows[0].parts && r.b == e);          // the kernel finds b by division
      const bool first_of_kind = e == 0 || r.n != rows[e - 1].n || r.parts != rows[e - 1].parts;
      std::vector<std::vector<int>> codes(per_row), tail(per_row);
      for (int local = 0; local < per_row * r.parts; ++local, ++block) {
        const Pair8 of = pair8(local, p.groups, s.Hkv * r.parts);
        CHECK(of.g >= 0 && of.g < p.groups && of.pair >= 0 && of.pair < s.Hkv * r.parts);
        const int h = of.pair / r.parts, part = of.pair % r.parts, j = h * p.groups + of.g;
        ++finished[{r.b, j}];
        if (r.parts > 1) {
          const int slot = block - local + j * r.parts + part;
          CHECK(slot >= 0 && slot < MAX_PARTS8 && slots.insert(slot).second);
        }
        if (!first_of_kind) continue;
        const Part8 m = part8(r.n, part, r.parts, log_g, step);
        CHECK(m.tails <= 4 && m.stop <= m.codes && m.rest <= s.G);
        const int len = m.stop - m.pos, turn = len > 0 ? (int)(rng() % (unsigned)len) : 0;
        for (int w = 0; w < p.waves; ++w) {
          Deal8 d = deal8(m, w, p.waves);
          if (w < m.tails) tail[j].push_back(w);
          int rounds = 0;
          for (int i = d.first, by = d.step; i < m.stop; i += by, by = p.waves) {
            CHECK(i >= m.pos);
            const int u = turned8(m, i, turn);
            CHECK(u >= m.pos && u < m.stop);
            codes[j].push_back(u);
            ++rounds;
          }
          CHECK(turned8(m, m.stop, turn) == m.stop && turned8(m, m.stop + 5, turn) == m.stop);
          if (len > 0) CHECK(rounds <= len / p.waves + 3);
        }
      }
      CHECK(r.parts <= FAN8 * (CTR8 - 1));                              // counters for sixteen parts each
      if (!first_of_kind) continue;
      const Part8 all = part8(r.n, 0, 1, log_g, step);
      for (int j = 0; j < per_row; ++j) {
        std::sort(codes[j].begin(), codes[j].end());
        CHECK((int)codes[j].size() == all.codes);
        for (int u = 0; u < all.codes; ++u) CHECK(codes[j][u] == u);
        CHECK((int)tail[j].size() == (all.rest + 31) / 32);
      }
      split += r.parts > 1;
      sixteens += r.parts > 32;
    }
    CHECK(block == p.blocks);
    CHECK((int)seen.size() == s.B);
    large += p.waves > 4;
    sets += p.hb > 16;
    uneven += !same;
  }
  printf("plans with large workgroups %ld, two sets %ld, rows split %ld, by sixteens %ld, rows listed %ld\n", large, sets, split, sixteens, uneven);
  if (!large || !sets || !split || !sixteens || !uneven) return 1;
  return 0;
}
