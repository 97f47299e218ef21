// Arguments of the kernels of attention over the paged cache, and their launchers, which have a source file for each kind.
#pragma once
#include "lq_paged.h"

namespace lq {

struct AttnPagedParams {
  const uint16_t* q;
  uint16_t* out;
  uint16_t *k_pages, *v_pages;               // (a step writes its token)
  const int* table;
  const uint16_t *k_new, *v_new;             // step
  RopeArg rope;
  const float* slopes;
  float *logits, *stats;                     // of a weighted cache whose items are split: what weights_kernel reads; else null
  float* weights;                            // of a weighted cache whose items are not, else null
  int logits_lds;                            // bytes of logits in LDS, for them
  int* counters;
  float* partials;
  const Row8* rows;
  float scale, cap;
  int window, B, Hkv, gh, groups, hb, log_p, n_pages, max_pages;
  Row8 same;                                 // ROWS_SAME: every row's entry
};

template <int MODE, bool STEP, bool MORE>
hipError_t attn_paged(const ShapePaged& s, const AttnPagedParams& p, const Rows8<MODE>& rows, const Plan8& plan, hipStream_t st);

}  // namespace lq
