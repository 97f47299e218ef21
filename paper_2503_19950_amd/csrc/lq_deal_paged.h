// Where things lie in a paged cache and how the work of attention over it is dealt out.  Integer arithmetic only, used by the
// kernels, by the host and by the host test.
#pragma once
#include "lq_deal8.h"

namespace lq {

struct ShapePaged {
  int B, Hq, Hkv, d, P, n_pages, max_pages;
  int gh;              // query heads of a kv head
  bool bf16, weighted;
  int cap() const { return max_pages * P; }
};
// Row8 of a paged cache: b counts the rows of both halves, half * B + row.

LQ8_HD bool is_page(int id, int n_pages) { return (uint32_t)id < (uint32_t)n_pages; }
// Elements from the start of a pool to unit `unit` of a row's tokens, kv head h, in page `id`: 32 tokens of keys are as many
// in one stretch as 32 tokens of values, and a page holds a whole number of units.
LQ8_HD int64_t unit_offset(int id, int Hkv, int h, int log_p, int unit, int d) {
  return ((((int64_t)id * Hkv + h) << log_p) + ((unit & ((1 << (log_p - 5)) - 1)) << 5)) * d;
}

// Where the angles of `wide` channels from c on begin among the dims / 2 of a token whose pairs are halves.  Channels that are not
// turned have angles that are there, too.
LQ8_HD int angle_of(int c, int dims, int wide) {
  const int half = dims / 2, last = half - wide;
  return c < half ? c : c - half < last ? c - half : last;
}

// Tokens seen .. n - 1 of a row get weight; the units that hold them, and those of one part of an item.
LQ8_HD int first_seen(int n, int window) { return window > 0 && n > window ? n - window : 0; }
struct PartPaged { int seen, pos, stop; };
LQ8_HD PartPaged part_paged(int n, int window, int part, int parts) {
  PartPaged p;
  p.seen = first_seen(n, window);
  const int first = p.seen / 32, units = (n + 31) / 32 - first, size = (units + parts - 1) / parts;
  p.pos = first + part * size;
  p.stop = p.pos + size < first + units ? p.pos + size : first + units;
  return p;
}
// The i-th unit of a part that begins `turn` units behind its first and goes round.
LQ8_HD int turned_paged(const PartPaged& p, int i, int turn) { return i + turn < p.stop ? i + turn : i + turn - (p.stop - p.pos); }

}  // namespace lq
