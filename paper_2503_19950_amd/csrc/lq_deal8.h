// How the work of attention over the 8-bit cache is dealt to workgroups and wavefronts.  Integer arithmetic only, used by the
// kernel, by the host, which plans launches (lq_plan8.h), and by the host test.
#pragma once
#include <stddef.h>
#include <stdint.h>
#ifdef __HIP__
#define LQ8_HD __host__ __device__ __forceinline__
#else
#define LQ8_HD inline
#endif

namespace lq {

struct Shape8 {
  int B, Hq, Hkv, d, G, cap;
  int gh;              // query heads of a kv head
  bool bf16;
};
inline int log2_of(int G) { return G == 32 ? 5 : G == 64 ? 6 : 7; }

// What a launch has to know of a batch row.
struct Row8 {
  int n;               // tokens that the row holds (append: before the call; a step: after it)
  int x;               // append: tokens that it takes; attention: its first workgroup
  int parts;           // attention: workgroups that share an item of it (Plan8)
  int b;               // attention: which row
};
constexpr int ROWS_IN_ARGS = 128;   // rows that travel in a launch's own arguments

// How attention is dealt to workgroups.  A (row, kv head, head group) is an item; its work is counted in units of 32
// tokens, codes as 1 and rows of the tail, twice as wide, as 2.  A workgroup takes an item, or one of `parts` equal parts
// of it, which the last of them to finish joins.  Rows with the most work come first.
struct Plan8 {
  int groups, hb;      // head groups of a kv head; heads in each (at most 32, two sets of 16; the last has the rest)
  int blocks, waves;
};
// (A fused step counts a block that its token fills up among the rows of the tail, which is what it reads.)
inline int units8(int n, int G, bool step) {
  const int full = (step ? n - 1 : n) & -G;            // (G is a power of two)
  return full / 32 + 2 * ((n - full + 31) / 32);
}

// What a part of an item has: units of codes [pos, stop), and, the last part, all units of the tail.
struct Part8 {
  int codes, rest;     // of the item: units of codes, rows of the tail
  int pos, stop, tails;
};
LQ8_HD Part8 part8(int n, int part, int parts, int log_g, bool step) {
  Part8 p;
  p.codes = (step ? n - 1 : n) >> log_g << (log_g - 5);
  p.rest = n - 32 * p.codes;
  const int work = p.codes + 2 * ((p.rest + 31) / 32), size = (work + parts - 1) / parts;
  p.pos = part * size;
  p.stop = p.pos + size < p.codes ? p.pos + size : p.codes;
  p.tails = part == parts - 1 ? (p.rest + 31) / 32 : 0;
  return p;
}

// Which (kv head, part) and head group the `local`-th workgroup of a row has: the head groups of a kv head are 8 workgroups
// apart (or as many as are left).
struct Pair8 { int pair, g; };
LQ8_HD Pair8 pair8(int local, int groups, int pairs) {
  if (groups == 1) return Pair8{local, 0};
  const int begin = local / (8 * groups) * 8, in = local - begin * groups;
  const int wide = pairs - begin < 8 ? pairs - begin : 8, g = in / wide;
  return Pair8{begin + in - g * wide, g};
}

// The units of codes of a wavefront: `first`, the next one `step` further, the others `waves` further each.  The units of the
// tail go to the first wavefronts, one each, which sit out two rounds of codes for it (unless all have one).
struct Deal8 { int first, step; };
LQ8_HD Deal8 deal8(const Part8& p, int wave, int waves) {
  const int workers = p.tails < waves ? waves - p.tails : waves;            // wavefronts in the first two rounds
  if (wave < p.tails && workers < waves) return Deal8{p.pos + wave + 2 * workers, waves};
  return Deal8{p.pos + wave - (waves - workers), workers};
}
// The i-th unit of a part that begins `turn` units behind its first and goes round; behind the last, `stop`.
LQ8_HD int turned8(const Part8& p, int i, int turn) {
  if (i >= p.stop) return p.stop;
  return i + turn < p.stop ? i + turn : i + turn - (p.stop - p.pos);
}

// A workspace: the counters of the items, each item's (one for all its parts, others for sixteen of them each) in a cache line,
// then room for the partial results of the workgroups that share an item (they come first in the grid), and as much again for
// those of sixteen joined.  No plan has more than MAX_PARTS8:
// rows that are alike are split into 256 workgroups at most, rows of different lengths into 512 or, what is over a 200th of the
// work (fewer than 200 items), into parts of a 256th, at most 256 and one more for each item.
constexpr int FAN8 = 16;           // parts joined at a time where there are many
constexpr int CTR8 = 32;           // ints from one counter to the next
constexpr int MAX_PARTS8 = 512;
// Head groups of a kv head.  More than 16 heads are two sets in one workgroup, which read the cache once, or two workgroups,
// which share the join's work: the former in launches that read 24 MB or more, where rows and kv heads are many (24 heads a kv
// head: 8 rows of 8192 x 8 kv heads, 134 MB, 36.2 us as two workgroups, 30.3 as two sets; 16 rows of 3000 x 4, 49 MB, 18.0 and
// 17.1; 1 row of 8192 x 8, 17 MB, 12.2 and 15.4).  A single kv head in many parts, whose join is long, would do better as
// two workgroups at any size (524288 tokens, 134 MB, 41.2 and 44.3; 94000 tokens, 24 MB, 17.7 and 22.1).
inline int head_groups8(const Shape8& s, bool large) { return (s.gh + (large ? 31 : 15)) / (large ? 32 : 16); }
inline size_t counter_bytes8(const Shape8& s) { return (size_t)s.B * s.Hkv * head_groups8(s, false) * CTR8 * sizeof(int); }
inline int partial_floats8(int hb, int d) { return hb * (d + 4); }   // o, then m and l, padded to 16 bytes
// LDS of a workgroup: each wavefront's results of a set of heads, or a join's (o, m and l of a share for every thread).
inline int lds_bytes8(int waves, int hb, int d) {
  const int merge = waves * partial_floats8(hb < 16 ? hb : 16, d), join = waves * 64 * 6;
  return (merge > join ? merge : join) * (int)sizeof(float);
}

}  // namespace lq
