// C ABI of the 8-bit cache: argument checks on the host, then kernel launches.
#include <math.h>

#include "lq_cache8.h"
#include "lq_internal.h"
#include "lq_plan8.h"

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

static lq_status attend8(const Shape8& s, const lq_cache8& c, RowList* rows, const void* k_new, const void* v_new, const void* q,
                         float softmax_scale, void* out, void* workspace, hipStream_t stream) {
  Plan8 plan;
  const bool same = plan8(s, rows->alike(), k_new != nullptr, rows->e, rows->n, &plan);
  if (!(softmax_scale > 0.f)) softmax_scale = 1.0f / sqrtf((float)s.d);
  return launch_attn8(s, c, q, softmax_scale, out, workspace, plan, k_new, v_new, rows->arg(c.seq_state, same), stream) == hipSuccess ? LQ_OK
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
  if (launch_append8(s, *cache, k_new, v_new, n_max, blocks, rows.arg(cache->seq_state, rows.alike()), (hipStream_t)stream) != hipSuccess) return LQ_ERR_HIP;
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
  return launch_read8(s, *cache, t0, n, k_out, v_out, rows.arg(cache->seq_state, rows.alike()), (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_HIP;
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
