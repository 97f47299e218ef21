// Host-side internals of rotary positions and of the paged cache: validated shapes and launchers.
#pragma once
#include "lq_cache8.h"
#include "lq_plan_paged.h"
#include "lq_rope.h"

namespace lq {

// A workspace: counters and partial results of attention as for the 8-bit cache (Shape8 of the same heads), and of a weighted
// cache behind them every query head's softmax reference and 1 / sum, and the logits, [B][Hkv][cap / 16][Hq / Hkv][16] (attention), or
// the slots of the tokens that stay, [B][Hkv][cap] (eviction).
// Rows of more than EVICT_SHORT tokens are counted in memory: three histograms and what they say, and two counts for every
// EVICT_PIECE tokens, of each kv head.
constexpr int EVICT_SHORT = 16384, EVICT_BINS = 2048, EVICT_PIECE = 2048, EVICT_MEMORY = 3 * EVICT_BINS + 8;
struct WorkspacePaged {
  int* counters;
  float *partials, *stats, *logits;
  int *slots, *found;
  size_t bytes;
};
inline WorkspacePaged split_workspace(const ShapePaged& s, void* ws) {
  const Shape8 s8 = shape8_of(s);
  const int groups = head_groups8(s8, true);
  char* at = (char*)ws;
  WorkspacePaged w{};
  w.counters = (int*)at;
  at += counter_bytes8(s8);
  w.partials = (float*)at;
  at += (size_t)2 * MAX_PARTS8 * partial_floats8((s.gh + groups - 1) / groups, s.d) * sizeof(float);
  if (s.weighted) {
    w.stats = (float*)at;
    at += ((size_t)s.B * s.Hq * 2 * sizeof(float) + 15) / 16 * 16;
    w.logits = (float*)at;
    w.slots = (int*)at;
    at += (size_t)s.B * s.Hq * s.cap() * sizeof(float);
    if (s.cap() > EVICT_SHORT) {
      w.found = (int*)at;
      at += (size_t)s.B * s.Hkv * (EVICT_MEMORY + 2 * ((s.cap() + EVICT_PIECE - 1) / EVICT_PIECE)) * sizeof(int);
    }
  }
  w.bytes = (size_t)(at - (char*)ws);
  return w;
}

hipError_t launch_rotate(const RopeArg& rope, int B, int L, int Hq, int Hkv, int d, bool bf16, const void* q, void* q_out, const void* k,
                         void* k_out, hipStream_t st);
// units: the most units of 32 tokens that a row's new tokens touch
hipError_t launch_append_paged(const ShapePaged& s, const lq_cache_paged& c, const RopeArg& rope, const void* k_new, const void* v_new,
                               int n_max, int units, const RowArg8& rows, hipStream_t st);

struct ScoresArg {
  float scale;         // on q . k: the softmax scale, times log2(e) or, with a cap, divided by it
  float cap;           // times log2(e); 0: none
  int window;
  const float* slopes;
};
struct NewToken {      // of a step
  const void *k, *v;
  RopeArg rope;
};
hipError_t launch_attn_paged(const ShapePaged& s, const lq_cache_paged& c, const ScoresArg& scores, const void* q, void* out, void* ws,
                             const PlanPaged& plan, const NewToken* step, const RowArg8& rows, hipStream_t st);
// Entries of `rows` that are evicted from, `count` of them: n, x = tokens that stay.
hipError_t launch_evict_paged(const ShapePaged& s, const lq_cache_paged& c, int recent, int most_kept, void* ws, const RowArg8& rows,
                              int count, hipStream_t st);

}  // namespace lq
