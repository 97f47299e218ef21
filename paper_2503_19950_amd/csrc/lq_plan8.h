// Planning a launch of attention over the 8-bit cache (host).
#pragma once
#include <algorithm>

#include "lq_deal8.h"

namespace lq {

// Parts of an item of u units when none may be larger than `most`.  Up to 20 units, five to a wavefront, it stays whole
// (512 tokens x 8 kv heads: whole 4.9 us, 2 parts 6.4, 4 parts 6.0; 1024 tokens: 6.9, 7.2, 6.4 and 8 parts 5.8).
constexpr int WHOLE8 = 20;
inline int parts_of(int u, int most) { return u > most && u > WHOLE8 ? (u + most - 1) / most : 1; }

// The largest load of a compute unit, in units of work, when items of more than `over` units are split into parts of at most
// `most`: the 256 largest workgroups one each, the others from the largest down to the least loaded ones (beyond 512: evenly).
inline int64_t largest_load(const Row8* r, int rows, int per_row, int most, int over) {
  constexpr int CUS = 256;
  struct Class { int64_t size, n; };
  Class few[CUS];
  for (int b = 0; b < rows; ++b) {
    const int u = r[b].x, parts = u > over ? parts_of(u, most) : 1;
    few[b] = Class{(u + parts - 1) / parts, (int64_t)parts * per_row};
  }
  std::sort(few, few + rows, [](const Class& x, const Class& y) { return x.size > y.size; });
  int64_t load = few[0].size, left = CUS;
  int i = 0;                                           // the class that the 256 largest end in
  while (i < rows && few[i].n < left) left -= few[i++].n;
  if (i == rows) return load;
  int up = i, down = i;
  int64_t room = left, more = few[i].n - left;         // of class `up` among the 256; of class `down` behind them
  for (int64_t paired = 0; paired < CUS;) {
    while (more == 0 && ++down < rows) more = few[down].n;
    while (room == 0 && --up >= 0) room = few[up].n;
    if (down >= rows || up < 0) break;
    const int64_t n = std::min(room, more);
    load = std::max(load, few[up].size + few[down].size);
    room -= n;
    more -= n;
    paired += n;
  }
  int64_t rest = down < rows ? more * few[down].size : 0;
  for (int k = down + 1; k < rows; ++k) rest += few[k].n * few[k].size;
  return load + rest / CUS;
}

// Fills the rows' parts, order and first workgroups, and says whether the rows still are alike.
//
// A compute unit reads up to 1.5 times its share of the memory's rate, so a launch is as fast as the memory where no compute
// unit has much more than a 256th of the work, and 256 workgroups, of 4 wavefronts already, are placed one to a compute unit.
// Times in us, d = 128, 4 heads a kv head, before (items whole, or in parts of a 256th rounded up) and with each rule:
//  - items that are fewer: as many parts each as make up to 256 workgroups (24 items of 16384 tokens: 11 parts, 264
//    workgroups, 25.7; 10 parts 20.6), none of less than 4 units, one to a wavefront; a single item in up to 128 (160000
//    tokens: 128 parts 13.0, 256 15.2), and no more than are joined in one go where 20 units each are enough for that (8 heads,
//    4000 tokens: 16 parts 7.0, 31 8.5; 16 heads, 10000: 11.0 and 12.7).
//  - between 128 and 256 items that cannot be split evenly stay whole, up to 200 of them in workgroups of 8 wavefronts, which
//    use that reserve (132 items of 4096 tokens: 4 wavefronts 31.3, 8 27.7; 180 items 34.3 and 34.6); so do long parts of
//    d = 64, whose units are half as large (5 rows of 34665 x 8 kv heads 36.9 -> 34.8, 4 of 20000 x 4: 10.8 and 12.0).
//  - a few items more than 256: rows for 256 stay whole, the rest is split into 256 (260 items 59.5 -> 50.9; 304 items
//    64.4 -> 56.9; from 340 on the reserve covers the second item of a compute unit).
// Rows of different lengths:
//  - up to 256 items: parts no larger than it takes for 256 of them, if that is within 1.25 of the even share (4 rows of up to
//    30000 x 8 kv heads 29.0; 512 parts 30.4; 31 rows of 4000 to 5500: 54.2 and 57.8), else for 512, two to a compute unit (24
//    rows of up to 12000: 256 parts 66.8, 512 58.8; 16 of up to 8000: 32.1 and 30.5; 20 of up to 20000, d = 64: 54.3 and 43.6),
//    unless the next rule loads the compute units more evenly (1 of 65536 and 29 of 512: 40.9, with it 33.6).
//  - what is over a 200th of all work is split into parts of a 256th.  Few and large workgroups, of 8 wavefronts for up to 256 items
//    and of 16 for up to 1024, the longest first, leave the balance to their placement, where items have 24 units on average.  With
//    4, 8 and 16 wavefronts, items and average units in brackets, 8 kv heads: 64 rows of up to 4096 (512, 65) 55.0, 54.7, 49.6; 100 of
//    up to 4000 (800, 64) 80.8, 77.1, 76.7; 100 of up to 3000 (800, 48) 62.0, 58.3, 60.3; 64 of up to 1500 (512, 24) 23.1, 23.3, 22.9;
//    64 of up to 1000 (512, 17) 16.7, 17.2, 17.6.  Near 24 units many items would do better with fewer wavefronts (100 rows of up to
//    2000, 800 items, 32 units: 43.8, 40.8, 45.3; 200 x 4 kv heads 46.4, 44.7, 48.8; 100 of up to 1500 33.8, 32.4, 37.2), as do
//    more than 1024, which balance by their number (200 of up to 2000: 75.6 with 4, 84.6 with 16).
// The rows' work is in their x; `bytes`: what the launch reads, `lds`: bytes of LDS that its workgroups may ask for.
inline bool plan_work8(const Shape8& s, int64_t bytes, int lds, bool same, Row8* rows, int n_rows, Plan8* p) {
  constexpr int CUS = 256, LEAST = 4;
  p->groups = head_groups8(s, bytes >= 24000000);
  p->hb = (s.gh + p->groups - 1) / p->groups;
  p->waves = 4;
  const int per_row = s.Hkv * p->groups;
  const int64_t items = (int64_t)s.B * per_row;
  Row8 *first = rows, *last = rows + n_rows;
  if (same) {
    const int u = first->x, most_parts = u > WHOLE8 ? u / LEAST : 1;
    int parts = items <= CUS / 2 ? std::min({(int)(CUS / items), CUS / 2, most_parts}) : 1;
    const int at_once = FAN8 * std::max(64 * p->waves / (p->hb * s.d / 4), 1);          // parts that are joined in one go
    if (parts > at_once && u <= 20 * at_once) parts = at_once;
    for (Row8* r = first; r != last; ++r) r->parts = parts;
    if ((items > CUS / 2 && items <= 200) || (s.d == 64 && items <= CUS / 2 && u >= 100 * parts)) p->waves = 8;
    if (items > CUS && items < 340 && per_row <= CUS) {
      const int left = s.B - CUS / per_row;
      const int split = std::min({CUS / (left * per_row), CUS / 2, most_parts});
      if (split > 1) {
        for (Row8* r = first; r != first + left; ++r) r->parts = split;
        same = false;
      }
    }
  } else {
    int64_t work = 0;
    int longest = LEAST;
    for (Row8* r = first; r != last; ++r) {
      work += (int64_t)r->x * per_row;
      longest = std::max(longest, r->x);
    }
    // parts of a 256th of what is over a 200th
    const int even = (int)std::max<int64_t>((work + CUS - 1) / CUS, LEAST);
    int most = even, over = (int)(work / 200);
    bool by_share = true;                              // this rule
    if (items <= CUS) {
      auto smallest = [&](int limit) {                 // size of parts with which there are no more than `limit`, of an item 256
        int lo = std::max(LEAST, (longest + 255) / 256), hi = longest;
        while (lo < hi) {
          const int mid = lo + (hi - lo) / 2;
          int64_t n = 0;
          for (Row8* r = first; r != last; ++r) n += parts_of(r->x, mid);
          if (n * per_row <= limit) hi = mid; else lo = mid + 1;
        }
        return lo;
      };
      const int one = smallest(CUS);
      by_share = one > LEAST && 4 * (int64_t)one * CUS > 5 * work;
      const int two = by_share ? smallest(2 * CUS) : one;
      if (!by_share || largest_load(first, n_rows, per_row, two, 0) <= largest_load(first, n_rows, per_row, even, over)) {
        most = two;
        over = 0;
        by_share = false;
      }
    }
    for (Row8* r = first; r != last; ++r) r->parts = r->x > over ? parts_of(r->x, most) : 1;
    if (by_share && items <= 1024 && work >= 24 * items) p->waves = items <= CUS ? 8 : 16;
    // (by work, not by tokens: what is split has to come first)
    std::sort(first, last, [](const Row8& x, const Row8& y) { return x.x > y.x; });
  }
  while (lds_bytes8(p->waves, p->hb, s.d) > lds || (p->hb > 16 && p->waves > 4)) p->waves /= 2;   // (LDS that a launch may ask for)
  p->blocks = 0;
  for (Row8* r = first; r != last; ++r) {
    r->x = p->blocks;
    p->blocks += r->parts * per_row;
  }
  return same;
}

// Of the 8-bit cache: units of 32 tokens, as codes 1 and in the tail 2 each.
inline bool plan8(const Shape8& s, bool same, bool step, Row8* rows, int n_rows, Plan8* p) {
  int64_t tokens = 0;
  for (int b = 0; b < n_rows; ++b) {
    tokens += rows[b].n;
    rows[b].x = units8(rows[b].n, s.G, step);          // until the end
  }
  return plan_work8(s, tokens * s.Hkv * s.d * 2, 65536, same, rows, n_rows, p);
}

}  // namespace lq
