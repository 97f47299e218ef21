// C ABI of rotary positions and of the paged cache: argument checks on the host, then kernel launches.
#include <math.h>

#include "lq_internal.h"
#include "lq_paged.h"

using namespace lq;

static lq_status make_shape_paged(const lq_config_paged* cfg, ShapePaged* s) {
  if (!cfg) return LQ_ERR_NULL;
  if (cfg->B <= 0 || cfg->Hq <= 0 || cfg->Hkv <= 0 || cfg->d <= 0 || cfg->page <= 0 || cfg->n_pages <= 0 || cfg->max_pages <= 0) return LQ_ERR_SHAPE;
  if (cfg->Hq % cfg->Hkv || (cfg->weighted != 0 && cfg->weighted != 1)) return LQ_ERR_SHAPE;
  if (cfg->dtype != LQ_F16 && cfg->dtype != LQ_BF16) return LQ_ERR_SHAPE;
  if (cfg->d != 64 && cfg->d != 96 && cfg->d != 128) return LQ_ERR_UNSUPPORTED;
  if (cfg->page != 32 && cfg->page != 64 && cfg->page != 128) return LQ_ERR_UNSUPPORTED;
  // tokens of a row, and slots of the pool, are counted in 31 bits; offsets in the pool in 64
  if ((int64_t)cfg->max_pages * cfg->page > ((int64_t)1 << 30) || (int64_t)cfg->n_pages * cfg->page >= ((int64_t)1 << 31)) return LQ_ERR_SHAPE;
  if ((int64_t)cfg->n_pages * cfg->page * cfg->Hkv > ((int64_t)1 << 40) / cfg->d) return LQ_ERR_SHAPE;
  if ((int64_t)cfg->B * cfg->Hq > 65535) return LQ_ERR_UNSUPPORTED;
  // the work of all items (Plan8) is counted in 31 bits
  const int64_t items = (int64_t)cfg->B * cfg->Hkv * ((cfg->Hq / cfg->Hkv + 15) / 16), cap = (int64_t)cfg->max_pages * cfg->page;
  if (items * (cap / 16 + 8) >= ((int64_t)1 << 31)) return LQ_ERR_SHAPE;
  *s = ShapePaged{cfg->B, cfg->Hq, cfg->Hkv, cfg->d, cfg->page, cfg->n_pages, cfg->max_pages, cfg->Hq / cfg->Hkv, cfg->dtype == LQ_BF16,
                  cfg->weighted == 1};
  return LQ_OK;
}

static bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

// Common start of the calls: shape, pointers, counts.
static lq_status begin_paged(const lq_config_paged* cfg, const lq_cache_paged* c, ShapePaged* s) {
  const lq_status st = make_shape_paged(cfg, s);
  if (st != LQ_OK) return st;
  if (!c->k_pages || !c->v_pages || !c->table || !c->n || !c->cur || !c->pages || !c->seq_state || (s->weighted && !c->weights)) return LQ_ERR_NULL;
  const void* buffers[] = {c->k_pages, c->v_pages, c->table, s->weighted ? c->weights : nullptr, c->seq_state};
  for (const void* p : buffers)
    if (!aligned16(p)) return LQ_ERR_SHAPE;
  for (int b = 0; b < s->B; ++b) {
    if (c->cur[b] != 0 && c->cur[b] != 1) return LQ_ERR_STATE;
    for (int half = 0; half < 2; ++half)
      if (c->pages[half * s->B + b] < 0 || c->pages[half * s->B + b] > s->max_pages) return LQ_ERR_STATE;
    if (c->n[b] < 0 || c->n[b] > c->pages[c->cur[b] * s->B + b] * s->P) return LQ_ERR_STATE;
  }
  return LQ_OK;
}

static lq_status make_rope(const lq_rope* rope, int d, const int32_t* positions, RopeArg* out) {
  *out = RopeArg{};
  if (!rope) return LQ_OK;
  if (!rope->freq) return LQ_ERR_NULL;
  if (rope->dims < 2 || rope->dims > d || rope->dims % 2 || (rope->interleaved != 0 && rope->interleaved != 1) || !isfinite(rope->factor)) return LQ_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(rope->freq) & 7) || !aligned4(positions)) return LQ_ERR_SHAPE;
  *out = RopeArg{rope->freq, positions, rope->dims, rope->interleaved, rope->factor};
  return LQ_OK;
}

static lq_status make_scores(const lq_scores* scores, const ShapePaged& s, float softmax_scale, ScoresArg* out) {
  const float log2e = 1.44269504088896340736f;
  if (!isfinite(softmax_scale)) return LQ_ERR_SHAPE;
  if (!(softmax_scale > 0.f)) softmax_scale = 1.0f / sqrtf((float)s.d);
  *out = ScoresArg{softmax_scale * log2e, 0.f, 0, nullptr};
  if (scores) {
    if (scores->window < 0 || !isfinite(scores->softcap) || !aligned4(scores->slopes)) return LQ_ERR_SHAPE;
    out->window = scores->window;
    out->slopes = scores->slopes;
    if (scores->softcap > 0.f) {
      out->scale = softmax_scale / scores->softcap;
      out->cap = scores->softcap * log2e;
    }
  }
  return isfinite(out->scale) && isfinite(out->cap) ? LQ_OK : LQ_ERR_SHAPE;
}

// Rows that a launch takes as one: the same counts in the same half.
static bool alike(const RowList& rows) {
  for (int b = 1; b < rows.n; ++b)
    if (rows.e[b].b - b != rows.e[0].b) return false;
  return rows.alike();
}

// rows: n tokens each, the step's among them.
static lq_status attend_paged(const ShapePaged& s, const lq_cache_paged& c, RowList* rows, const ScoresArg& scores, const NewToken* step,
                              const void* q, void* out, void* workspace, hipStream_t stream) {
  PlanPaged plan;
  const bool alone = plan_paged(s, scores.window, step, alike(*rows), rows->e, rows->n, &plan);
  return launch_attn_paged(s, c, scores, q, out, workspace, plan, step, rows->arg(c.seq_state, alone), stream) == hipSuccess ? LQ_OK
                                                                                                                                   : LQ_ERR_HIP;
}

extern "C" {

lq_status logquant_rope_frequencies(int32_t dims, double base, double stretch, double original, double slow, double fast, double* freq) {
  if (!freq) return LQ_ERR_NULL;
  if (dims < 2 || dims % 2 || !(base > 0) || !isfinite(base) || !(stretch > 0) || !isfinite(stretch) || !(original >= 0) || !isfinite(original))
    return LQ_ERR_SHAPE;
  if (original > 0 && !(isfinite(slow) && isfinite(fast) && fast > slow)) return LQ_ERR_SHAPE;
  for (int i = 0; i < dims / 2; ++i) {
    const double f = pow(base, -2.0 * i / dims);
    double w = 0.0;                                    // how much of it stays
    if (original > 0) w = fmin(fmax((original * f / 6.283185307179586477 - slow) / (fast - slow), 0.0), 1.0);
    freq[i] = w * f + (1.0 - w) * f / stretch;
  }
  return LQ_OK;
}

lq_status logquant_rotate(const lq_rope* rope, int32_t B, int32_t L, int32_t Hq, int32_t Hkv, int32_t d, int32_t dtype,
                          const int32_t* positions, const void* q, void* q_out, const void* k, void* k_out, void* stream) {
  if (!rope || !q != !q_out || !k != !k_out || (!q && !k)) return LQ_ERR_NULL;
  if (B <= 0 || L <= 0 || d <= 0 || (q && Hq <= 0) || (k && Hkv <= 0) || (dtype != LQ_F16 && dtype != LQ_BF16)) return LQ_ERR_SHAPE;
  if (d != 64 && d != 96 && d != 128) return LQ_ERR_UNSUPPORTED;
  if (!q) Hq = 0;
  if (!k) Hkv = 0;
  // (a row of a tensor and the heads of both are counted in 31 bits, the grid's z in 16)
  const int64_t most = ((int64_t)1 << 31) - 1;
  if (B > 65535 || (int64_t)Hq + Hkv > most / 16 || (int64_t)B * L > most || (int64_t)Hq * L > most / B || (int64_t)Hkv * L > most / B) return LQ_ERR_UNSUPPORTED;
  RopeArg r;
  const lq_status st = make_rope(rope, d, positions, &r);
  if (st != LQ_OK) return st;
  if (!aligned16(q) || !aligned16(q_out) || !aligned16(k) || !aligned16(k_out)) return LQ_ERR_SHAPE;
  clear_stale_error();
  return launch_rotate(r, B, L, Hq, Hkv, d, dtype == LQ_BF16, q, q_out, k, k_out, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_HIP;
}

lq_status logquant_sizes_paged(const lq_config_paged* cfg, lq_sizes_paged* out) {
  if (!cfg || !out) return LQ_ERR_NULL;
  ShapePaged s;
  const lq_status st = make_shape_paged(cfg, &s);
  if (st != LQ_OK) return st;
  out->pages = (size_t)s.n_pages * s.Hkv * s.P * s.d * 2;
  out->table = (size_t)2 * s.B * s.max_pages * sizeof(int);
  out->weights = s.weighted ? (size_t)2 * s.B * s.Hkv * s.cap() * sizeof(float) : 0;
  out->seq_state = s.B * sizeof(Row8);
  out->workspace = split_workspace(s, nullptr).bytes;
  return LQ_OK;
}

lq_status logquant_workspace_init_paged(const lq_config_paged* cfg, void* workspace, void* stream) {
  if (!cfg || !workspace) return LQ_ERR_NULL;
  ShapePaged s;
  const lq_status st = make_shape_paged(cfg, &s);
  if (st != LQ_OK) return st;
  if (!aligned16(workspace)) return LQ_ERR_SHAPE;
  clear_stale_error();
  return launch_zero_ints((int*)workspace, (int)(counter_bytes8(shape8_of(s)) / sizeof(int)), (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_HIP;
}

lq_status logquant_append_paged(const lq_config_paged* cfg, lq_cache_paged* cache, const lq_rope* rope, const int32_t* positions,
                                const void* k_new, const void* v_new, const int32_t* n_new, int32_t n_max, void* stream) {
  if (!cfg || !cache || !k_new || !v_new) return LQ_ERR_NULL;
  ShapePaged s;
  RopeArg r;
  lq_status st = begin_paged(cfg, cache, &s);
  if (st == LQ_OK) st = make_rope(rope, s.d, positions, &r);
  if (st != LQ_OK) return st;
  if (n_max < 1 || !aligned16(k_new) || !aligned16(v_new)) return LQ_ERR_SHAPE;
  RowList rows(s.B);
  if (!rows.ok()) return LQ_ERR_CAPACITY;
  int units = 0;
  for (int b = 0; b < s.B; ++b) {
    const int n = cache->n[b], rb = cache->cur[b] * s.B + b, take = n_new ? n_new[b] : n_max;
    if (take < 0 || take > n_max) return LQ_ERR_SHAPE;
    if (take > cache->pages[rb] * s.P - n) return LQ_ERR_CAPACITY;
    rows.e[b] = Row8{n, take, 1, rb};
    const int need = take ? (n + take + 31) / 32 - n / 32 : 0;
    if (need > units) units = need;
  }
  if (!units) return LQ_OK;   // nobody takes a token
  clear_stale_error();
  if (launch_append_paged(s, *cache, r, k_new, v_new, n_max, units, rows.arg(cache->seq_state, alike(rows)), (hipStream_t)stream) != hipSuccess)
    return LQ_ERR_HIP;
  for (int b = 0; b < s.B; ++b) cache->n[b] += rows.e[b].x;
  return LQ_OK;
}

lq_status logquant_decode_attn_paged(const lq_config_paged* cfg, lq_cache_paged* cache, const lq_scores* scores, const void* q,
                                     float softmax_scale, void* out, void* workspace, void* stream) {
  if (!cfg || !cache || !q || !out || !workspace) return LQ_ERR_NULL;
  ShapePaged s;
  ScoresArg sc;
  lq_status st = begin_paged(cfg, cache, &s);
  if (st == LQ_OK) st = make_scores(scores, s, softmax_scale, &sc);
  if (st != LQ_OK) return st;
  if (!aligned16(q) || !aligned16(out) || !aligned16(workspace)) return LQ_ERR_SHAPE;
  RowList rows(s.B);
  if (!rows.ok()) return LQ_ERR_CAPACITY;
  for (int b = 0; b < s.B; ++b) rows.e[b] = Row8{cache->n[b], 0, 1, cache->cur[b] * s.B + b};
  clear_stale_error();
  return attend_paged(s, *cache, &rows, sc, nullptr, q, out, workspace, (hipStream_t)stream);
}

lq_status logquant_decode_step_paged(const lq_config_paged* cfg, lq_cache_paged* cache, const lq_rope* rope, const int32_t* positions,
                                     const lq_scores* scores, const void* k_new, const void* v_new, const void* q, float softmax_scale,
                                     void* out, void* workspace, void* stream) {
  if (!cfg || !cache || !k_new || !v_new || !q || !out || !workspace) return LQ_ERR_NULL;
  ShapePaged s;
  ScoresArg sc;
  NewToken token{k_new, v_new, {}};
  lq_status st = begin_paged(cfg, cache, &s);
  if (st == LQ_OK) st = make_rope(rope, s.d, positions, &token.rope);
  if (st == LQ_OK) st = make_scores(scores, s, softmax_scale, &sc);
  if (st != LQ_OK) return st;
  if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(q) || !aligned16(out) || !aligned16(workspace)) return LQ_ERR_SHAPE;
  RowList rows(s.B);
  if (!rows.ok()) return LQ_ERR_CAPACITY;
  for (int b = 0; b < s.B; ++b) {
    const int rb = cache->cur[b] * s.B + b;
    if (cache->n[b] == cache->pages[rb] * s.P) return LQ_ERR_CAPACITY;
    rows.e[b] = Row8{cache->n[b] + 1, 0, 1, rb};
  }
  clear_stale_error();
  st = attend_paged(s, *cache, &rows, sc, &token, q, out, workspace, (hipStream_t)stream);
  if (st == LQ_OK)
    for (int b = 0; b < s.B; ++b) cache->n[b] += 1;
  return st;
}

lq_status logquant_evict_paged(const lq_config_paged* cfg, lq_cache_paged* cache, const int32_t* keep, int32_t recent, void* workspace,
                               void* stream) {
  if (!cfg || !cache || !keep || !workspace) return LQ_ERR_NULL;
  ShapePaged s;
  const lq_status st = begin_paged(cfg, cache, &s);
  if (st != LQ_OK) return st;
  if (!s.weighted) return LQ_ERR_STATE;
  if (recent < 0 || !aligned16(workspace)) return LQ_ERR_SHAPE;
  RowList rows(s.B);
  if (!rows.ok()) return LQ_ERR_CAPACITY;
  int count = 0, most_kept = 0;
  for (int b = 0; b < s.B; ++b) {
    if (keep[b] < 0) return LQ_ERR_SHAPE;
    if (cache->n[b] <= keep[b]) continue;
    if (recent > keep[b]) return LQ_ERR_SHAPE;
    if (keep[b] > cache->pages[(1 - cache->cur[b]) * s.B + b] * s.P) return LQ_ERR_CAPACITY;
    rows.e[count++] = Row8{cache->n[b], keep[b], 1, cache->cur[b] * s.B + b};
    if (keep[b] > most_kept) most_kept = keep[b];
  }
  if (most_kept) {
    RowArg8 arg = rows.arg(cache->seq_state, false);
    arg.n = count;
    clear_stale_error();
    if (launch_evict_paged(s, *cache, recent, most_kept, workspace, arg, count, (hipStream_t)stream) != hipSuccess) return LQ_ERR_HIP;
  }
  for (int i = 0; i < count; ++i) {
    const int b = rows.e[i].b % s.B;
    cache->n[b] = rows.e[i].x;
    cache->cur[b] ^= 1;
  }
  return LQ_OK;
}

}  // extern "C"
