// C ABI of the 8-bit cache: argument checks on the host, then kernel launches.
#include <math.h>
#include <stdlib.h>

#include <algorithm>

#include "lq_cache8.h"
#include "lq_internal.h"

using namespace lq;

static lq_status make_shape8(const lq_config8* cfg, Shape8* s) {
  if (!cfg) return LQ_ERR_NULL;
  if (cfg->B <= 0 || cfg->Hq <= 0 || cfg->Hkv <= 0 || cfg->d <= 0 || cfg->block <= 0 || cfg->capacity <= 0) return LQ_ERR_SHAPE;
  if (cfg->Hq % cfg->Hkv) return LQ_ERR_SHAPE;
  if (cfg->dtype != LQ_F16 && cfg->dtype != LQ_BF16) return LQ_ERR_SHAPE;
  if (cfg->d != 64 && cfg->d != 96 && cfg->d != 128) return LQ_ERR_UNSUPPORTED;
  if (cfg->block != 32 && cfg->block != 64 && cfg->block != 128) return LQ_ERR_UNSUPPORTED;
  if (cfg->capacity % cfg->block) return LQ_ERR_SHAPE;
  // offsets within a (row, kv head) slice are 31 bits, those of slices 64
  if ((int64_t)cfg->capacity * cfg->d > ((int64_t)1 << 30)) return LQ_ERR_SHAPE;
  if ((int64_t)cfg->B * cfg->Hkv * cfg->capacity * cfg->d > ((int64_t)1 << 40)) return LQ_ERR_SHAPE;
  if ((int64_t)cfg->B * cfg->Hq > 65535) return LQ_ERR_UNSUPPORTED;
  // the work of all items (Plan8) is counted in 31 bits
  const int64_t items = (int64_t)cfg->B * cfg->Hkv * ((cfg->Hq / cfg->Hkv + 15) / 16);
  if (items * (cfg->capacity / 32 + 8) >= ((int64_t)1 << 31)) return LQ_ERR_SHAPE;
  *s = Shape8{cfg->B, cfg->Hq, cfg->Hkv, cfg->d, cfg->block, cfg->capacity, cfg->Hq / cfg->Hkv, cfg->dtype == LQ_BF16};
  return LQ_OK;
}

static bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Common start of the calls: shape, pointers, counts.
static lq_status begin8(const lq_config8* cfg, const lq_cache8* c, Shape8* s) {
  const lq_status st = make_shape8(cfg, s);
  if (st != LQ_OK) return st;
  if (!c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale || !c->k_tail || !c->v_tail || !c->n || !c->seq_state) return LQ_ERR_NULL;
  const void* buffers[] = {c->k_codes, c->v_codes, c->k_scale, c->v_scale, c->k_tail, c->v_tail, c->seq_state};
  for (const void* p : buffers)
    if (!aligned16(p)) return LQ_ERR_SHAPE;
  for (int b = 0; b < s->B; ++b)
    if (c->n[b] < 0 || c->n[b] > s->cap) return LQ_ERR_STATE;
  return LQ_OK;
}

// One entry for each batch row: on the stack for the batches that travel in a launch's arguments, else from the heap.
struct RowList {
  Row8 few[ROWS_IN_ARGS];
  Row8* many = nullptr;
  Row8* e;
  int n;
  explicit RowList(int rows) : e(few), n(rows) {
    if (n > ROWS_IN_ARGS) e = many = static_cast<Row8*>(malloc(n * sizeof(Row8)));
  }
  ~RowList() { free(many); }
  RowList(const RowList&) = delete;
  bool ok() const { return e != nullptr; }
  bool alike() const {
    for (int b = 1; b < n; ++b)
      if (e[b].n != e[0].n || e[b].x != e[0].x) return false;
    return true;
  }
  RowArg8 arg(const lq_cache8* c, bool same) const { return RowArg8{e, (Row8*)c->seq_state, n, same}; }
};

// Parts of an item of u units when none may be larger than `most`.  Up to 20 units, five to a wavefront, it stays whole
// (512 tokens x 8 kv heads: whole 4.9 us, 2 parts 6.4, 4 parts 6.0; 1024 tokens: 6.9, 7.2, 6.4 and 8 parts 5.8).
constexpr int WHOLE = 20;
static int parts_of(int64_t u, int64_t most) { return u > most && u > WHOLE ? (int)((u + most - 1) / most) : 1; }

// The largest load of a compute unit, in units of work, when items over a `whole`-th of it are split into parts of a
// `shares`-th: the 256 largest workgroups one each, the others from the largest down to the least loaded ones (beyond 512:
// evenly).
static int64_t largest_load(const RowList& rows, int per_row, int64_t work, int shares, int whole, const int64_t* units) {
  constexpr int CUS = 256;
  struct Class { int64_t size, n; };
  Class few[ROWS_IN_ARGS];
  if (rows.n > ROWS_IN_ARGS) return 0;
  const int64_t most = std::max<int64_t>((work + shares - 1) / shares, 4);
  for (int b = 0; b < rows.n; ++b) {
    const int parts = units[b] * whole <= work ? 1 : parts_of(units[b], most);
    few[b] = Class{(units[b] + parts - 1) / parts, (int64_t)parts * per_row};
  }
  std::sort(few, few + rows.n, [](const Class& x, const Class& y) { return x.size > y.size; });
  int64_t load = few[0].size, left = CUS;
  int i = 0;                                           // the class that the 256 largest end in
  while (i < rows.n && few[i].n < left) left -= few[i++].n;
  if (i == rows.n) return load;
  int up = i, down = i;
  int64_t room = left, more = few[i].n - left;         // of class `up` among the 256; of class `down` behind them
  for (int64_t paired = 0; paired < CUS;) {
    while (more == 0 && ++down < rows.n) more = few[down].n;
    while (room == 0 && --up >= 0) room = few[up].n;
    if (down >= rows.n || up < 0) break;
    const int64_t n = std::min(room, more);
    load = std::max(load, few[up].size + few[down].size);
    room -= n;
    more -= n;
    paired += n;
  }
  int64_t rest = down < rows.n ? more * few[down].size : 0;
  for (int k = down + 1; k < rows.n; ++k) rest += few[k].n * few[k].size;
  return load + rest / CUS;
}

// Fills the rows' parts, order and first workgroups, and says whether the rows still are alike.
//
// A compute unit reads up to 1.5 times its share of the memory's rate, so a launch is as fast as the memory where no compute
// unit has much more than a 256th of the work, and 256 workgroups, of 4 wavefronts already, are placed one to a compute unit.
// Times in us, d = 128, 4 heads a kv head, before (items whole, or in parts of a 256th rounded up) and with each rule:
//  - items that are fewer: as many parts each as make up to 256 workgroups (24 items of 16384 tokens: 11 parts, 264
//    workgroups, 25.7; 10 parts 20.6), none of less than 4 units, one to a wavefront.
//  - between 128 and 256 items that cannot be split evenly stay whole, up to 200 of them in workgroups of 8 wavefronts, which
//    use that reserve (132 items of 4096 tokens: 4 wavefronts 31.3, 8 27.7; 180 items 34.3 and 34.6); so do long parts of
//    d = 64, whose units are half as large (5 rows of 34665 x 8 kv heads 36.9 -> 34.8, 4 of 20000 x 4: 10.8 and 12.0).
//  - a few items more than 256: rows for 256 stay whole, the rest is split into 256 (260 items 59.5 -> 50.9; 304 items
//    64.4 -> 56.9; from 340 on the reserve covers the second item of a compute unit).
// Rows of different lengths:
//  - up to 256 items: the smallest `most` that makes no more than 256 parts (16 rows of up to 8000 x 8 kv heads 36.1 -> 31.9;
//    4 rows of up to 30000 34.8 -> 28.7), if that is within 1.5 of the even share.
//  - else what is over a 200th of all work is split into parts of a 256th, or, of up to 256 items, over a 300th into parts of
//    a 384th where that loads the compute units more evenly (45 rows of up to 24597 x 4 kv heads 132 -> 108, but 1 of 65536
//    and 29 of 512 x 8: 33.6 and 40.0).  Few and large workgroups, of 8 or 16 wavefronts, the longest first, leave the balance
//    to their placement (64 rows of up to 4096 x 8 kv heads: 4 wavefronts 54.5, 8 54.6, 16 49.5; 100 of up to 4000: 79.9, 75.8,
//    76.4; 30 of up to 9000, d = 96: 43.0, 43.6, 47.0), unless they are small (200 rows of up to 2000, 31 units each: 4
//    wavefronts 75.6, 16 84.6) or many, which balance by their number.
static bool plan8(const Shape8& s, bool same, bool step, RowList* rows, Plan8* p) {
  constexpr int CUS = 256, LEAST = 4;
  auto units = [&](const Row8& r) -> int64_t { return units8(r.n, s.G, step); };
  int64_t tokens = 0;
  for (int b = 0; b < rows->n; ++b) tokens += rows->e[b].n;
  p->groups = head_groups8(s, tokens * s.Hkv * s.d * 2 >= 24000000);
  p->hb = (s.gh + p->groups - 1) / p->groups;
  p->waves = 4;
  const int per_row = s.Hkv * p->groups;
  const int64_t items = (int64_t)s.B * per_row;
  Row8 *first = rows->e, *last = rows->e + rows->n;
  if (same) {
    const int u = (int)units(*first), most_parts = u > WHOLE ? u / LEAST : 1;
    const int parts = items <= CUS / 2 ? std::min((int)(CUS / items), most_parts) : 1;
    for (Row8* r = first; r != last; ++r) r->parts = parts;
    if ((items > CUS / 2 && items <= 200) || (s.d == 64 && items <= CUS / 2 && u >= 100 * parts)) p->waves = 8;
    if (items > CUS && items < 340 && per_row <= CUS) {
      const int left = s.B - CUS / per_row;
      const int split = std::min(CUS / (left * per_row), most_parts);
      if (split > 1) {
        for (Row8* r = first; r != first + left; ++r) r->parts = split;
        same = false;
      }
    }
  } else {
    int64_t work = 0, longest = LEAST, most = 0;
    for (Row8* r = first; r != last; ++r) {
      const int64_t u = units(*r);
      work += u * per_row;
      longest = std::max(longest, u);
    }
    if (items <= CUS) {
      int64_t lo = LEAST, hi = longest;
      while (lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        int64_t n = 0;
        for (Row8* r = first; r != last; ++r) n += parts_of(units(*r), mid);
        if (n * per_row <= CUS) hi = mid; else lo = mid + 1;
      }
      if (lo == LEAST || 2 * lo * CUS <= 3 * work) most = lo;
    }
    if (most) {
      for (Row8* r = first; r != last; ++r) r->parts = parts_of(units(*r), most);
    } else {
      int shares = CUS, whole = 200;
      if (items <= CUS && rows->n <= ROWS_IN_ARGS) {
        int64_t u[ROWS_IN_ARGS];
        for (int b = 0; b < rows->n; ++b) u[b] = units(rows->e[b]);
        if (largest_load(*rows, per_row, work, 384, 300, u) < largest_load(*rows, per_row, work, CUS, 200, u)) shares = 384, whole = 300;
      }
      most = std::max<int64_t>((work + shares - 1) / shares, LEAST);
      for (Row8* r = first; r != last; ++r) r->parts = units(*r) * whole <= work ? 1 : parts_of(units(*r), most);
      if (items <= 1024 && work >= 24 * items) p->waves = items <= CUS ? 8 : 16;
    }
    // (by work, not by tokens: what is split has to come first)
    std::sort(first, last, [&](const Row8& x, const Row8& y) { return units(x) > units(y); });
  }
  while (lds_bytes8(p->waves, p->hb, s.d) > 65536 || (p->hb > 16 && p->waves > 4)) p->waves /= 2;   // (LDS that a launch may ask for)
  p->blocks = 0;
  for (Row8* r = first; r != last; ++r) {
    r->x = p->blocks;
    p->blocks += r->parts * per_row;
  }
  return same;
}

static lq_status attend8(const Shape8& s, const lq_cache8& c, RowList* rows, const void* k_new, const void* v_new, const void* q,
                         float softmax_scale, void* out, void* workspace, hipStream_t stream) {
  Plan8 plan;
  const bool same = plan8(s, rows->alike(), k_new != nullptr, rows, &plan);
  if (!(softmax_scale > 0.f)) softmax_scale = 1.0f / sqrtf((float)s.d);
  return launch_attn8(s, c, q, softmax_scale, out, workspace, plan, k_new, v_new, rows->arg(&c, same), stream) == hipSuccess ? LQ_OK
                                                                                                                             : LQ_ERR_HIP;
}

extern "C" {

lq_status logquant_sizes8(const lq_config8* cfg, lq_sizes8* out) {
  if (!cfg || !out) return LQ_ERR_NULL;
  Shape8 s;
  const lq_status st = make_shape8(cfg, &s);
  if (st != LQ_OK) return st;
  const size_t bh = (size_t)s.B * s.Hkv;
  out->codes = bh * s.cap * s.d;
  out->scale = bh * (s.cap / s.G) * sizeof(float);
  out->tail = bh * s.G * s.d * 2;
  out->seq_state = s.B * sizeof(Row8);
  const int groups = head_groups8(s, true);
  out->workspace = counter_bytes8(s) + (size_t)2 * MAX_PARTS8 * partial_floats8((s.gh + groups - 1) / groups, s.d) * sizeof(float);
  return LQ_OK;
}

lq_status logquant_workspace_init8(const lq_config8* cfg, void* workspace, void* stream) {
  if (!cfg || !workspace) return LQ_ERR_NULL;
  Shape8 s;
  const lq_status st = make_shape8(cfg, &s);
  if (st != LQ_OK) return st;
  if (!aligned16(workspace)) return LQ_ERR_SHAPE;
  clear_stale_error();
  return launch_zero_ints((int*)workspace, (int)(counter_bytes8(s) / sizeof(int)), (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_HIP;
}

lq_status logquant_append8(const lq_config8* cfg, lq_cache8* cache, const void* k_new, const void* v_new, const int32_t* n_new,
                           int32_t n_max, void* stream) {
  if (!cfg || !cache || !k_new || !v_new) return LQ_ERR_NULL;
  Shape8 s;
  const lq_status st = begin8(cfg, cache, &s);
  if (st != LQ_OK) return st;
  if (n_max < 1 || !aligned16(k_new) || !aligned16(v_new)) return LQ_ERR_SHAPE;
  RowList rows(s.B);
  if (!rows.ok()) return LQ_ERR_CAPACITY;
  int blocks = 0;
  for (int b = 0; b < s.B; ++b) {
    const int take = n_new ? n_new[b] : n_max;
    if (take < 0 || take > n_max) return LQ_ERR_SHAPE;
    if (take > s.cap - cache->n[b]) return LQ_ERR_CAPACITY;
    rows.e[b] = Row8{cache->n[b], take, 1, b};
    // a workgroup for each block that becomes full, and one for the rest, unless the first has rows in the tail (append8_kernel)
    const int held = cache->n[b] % s.G, full = (held + take) / s.G, rest = (held + take) % s.G;
    const int need = !take ? 0 : full + (rest && !(held && full) ? 1 : 0);
    if (need > blocks) blocks = need;
  }
  if (!blocks) return LQ_OK;   // nobody takes a token
  clear_stale_error();
  if (launch_append8(s, *cache, k_new, v_new, n_max, blocks, rows.arg(cache, rows.alike()), (hipStream_t)stream) != hipSuccess) return LQ_ERR_HIP;
  for (int b = 0; b < s.B; ++b) cache->n[b] += rows.e[b].x;
  return LQ_OK;
}

lq_status logquant_read8(const lq_config8* cfg, const lq_cache8* cache, int32_t t0, int32_t n, void* k_out, void* v_out, void* stream) {
  if (!cfg || !cache || (!k_out && !v_out)) return LQ_ERR_NULL;
  Shape8 s;
  const lq_status st = begin8(cfg, cache, &s);
  if (st != LQ_OK) return st;
  if (t0 < 0 || n < 1 || t0 > s.cap || n > s.cap - t0 || !aligned16(k_out) || !aligned16(v_out)) return LQ_ERR_SHAPE;
  RowList rows(s.B);
  if (!rows.ok()) return LQ_ERR_CAPACITY;
  int longest = 0;
  for (int b = 0; b < s.B; ++b) {
    rows.e[b] = Row8{cache->n[b], 0, 1, b};
    if (cache->n[b] > longest) longest = cache->n[b];
  }
  if (longest <= t0) return LQ_OK;   // nothing of the range is there
  clear_stale_error();
  return launch_read8(s, *cache, t0, n, k_out, v_out, rows.arg(cache, rows.alike()), (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_HIP;
}

lq_status logquant_decode_attn8(const lq_config8* cfg, const lq_cache8* cache, const void* q, float softmax_scale, void* out,
                                void* workspace, void* stream) {
  if (!cfg || !cache || !q || !out || !workspace) return LQ_ERR_NULL;
  Shape8 s;
  const lq_status st = begin8(cfg, cache, &s);
  if (st != LQ_OK) return st;
  if (!aligned16(q) || !aligned16(out) || !aligned16(workspace)) return LQ_ERR_SHAPE;
  RowList rows(s.B);
  if (!rows.ok()) return LQ_ERR_CAPACITY;
  for (int b = 0; b < s.B; ++b) rows.e[b] = Row8{cache->n[b], 0, 1, b};
  clear_stale_error();
  return attend8(s, *cache, &rows, nullptr, nullptr, q, softmax_scale, out, workspace, (hipStream_t)stream);
}

lq_status logquant_decode_step8(const lq_config8* cfg, lq_cache8* cache, const void* k_new, const void* v_new, const void* q,
                                float softmax_scale, void* out, void* workspace, void* stream) {
  if (!cfg || !cache || !k_new || !v_new || !q || !out || !workspace) return LQ_ERR_NULL;
  Shape8 s;
  lq_status st = begin8(cfg, cache, &s);
  if (st != LQ_OK) return st;
  if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(q) || !aligned16(out) || !aligned16(workspace)) return LQ_ERR_SHAPE;
  RowList rows(s.B);
  if (!rows.ok()) return LQ_ERR_CAPACITY;
  for (int b = 0; b < s.B; ++b) {
    if (cache->n[b] == s.cap) return LQ_ERR_CAPACITY;
    rows.e[b] = Row8{cache->n[b] + 1, 0, 1, b};
  }
  clear_stale_error();
  st = attend8(s, *cache, &rows, k_new, v_new, q, softmax_scale, out, workspace, (hipStream_t)stream);
  if (st == LQ_OK)
    for (int b = 0; b < s.B; ++b) cache->n[b] += 1;
  return st;
}

}  // extern "C"
