// Plans of attention over the 8-bit cache for random batches: what is built and allotted is what they can ask for.  Rows that are
// alike never get 16 wavefronts, and the partial results of rows that are split have room.
#include <math.h>
#include <stdio.h>
#include <stdlib.h>

#include <random>
#include <vector>

#include "lq_plan8.h"

using namespace lq;

int main() {
  static_assert(MAX_PARTS8 == 512, "the bound that lq_deal8.h derives");
  std::mt19937 rng(20251206);
  auto in = [&](int a, int b) { return (int)(a + rng() % (unsigned)(b - a + 1)); };
  auto log_in = [&](int b) { return (int)exp2(std::uniform_real_distribution<>(0, log2(b + 1.0))(rng)) - 1; };
  int most = 0, with16 = 0, with8_alike = 0;
  for (int the_case = 0; the_case < 60000; ++the_case) {
    Shape8 s{};
    const int ds[] = {64, 96, 128}, Gs[] = {32, 64, 128}, ghs[] = {1, 2, 3, 4, 7, 8, 15, 16, 17, 24, 31, 32, 33, 40, 64, 71};
    s.B = 1 + log_in(the_case % 10 ? 80 : 600);
    s.Hkv = 1 + log_in(the_case % 7 ? 16 : 300);
    s.gh = ghs[in(0, 15)];
    s.Hq = s.gh * s.Hkv;
    s.d = ds[in(0, 2)];
    s.G = Gs[in(0, 2)];
    const bool step = in(0, 1);
    const int longest = 1 + log_in(the_case % 4 ? 9000 : 2000000), kind = in(0, 4);
    std::vector<Row8> rows(s.B);
    bool same = true;
    for (int b = 0; b < s.B; ++b) {
      int n = kind == 0 ? longest : kind == 1 ? in(0, longest) : kind == 2 ? (b ? log_in(200) : longest) : kind == 3 ? log_in(longest)
              : longest - in(0, longest / 100);
      if (step && n == 0) n = 1;
      rows[b] = Row8{n, 0, 1, b};
      same = same && n == rows[0].n;
    }
    Plan8 p;
    same = plan8(s, same, step, rows.data(), s.B, &p);
    int behind = 0;                                     // workgroups up to the end of the last row that is split
    for (const Row8& r : rows)
      if (r.parts > 1) behind = std::max(behind, r.x + r.parts * s.Hkv * p.groups);
    if (behind > MAX_PARTS8 || (same && p.waves > 8)) {
      printf("case %d: %d partial results, %d wavefronts, alike %d\n", the_case, behind, p.waves, (int)same);
      return 1;
    }
    most = std::max(most, behind);
    with16 += p.waves == 16;
    with8_alike += same && p.waves == 8;
  }
  printf("at most %d partial results; 16 wavefronts %d times, 8 for rows alike %d times\n", most, with16, with8_alike);
  return most > 256 && with16 && with8_alike ? 0 : 1;
}
