// Kernels of attention over the paged cache: a step.
#include "lq_attn_paged.h"

namespace lq {
LQ_ATTN_PAGED(ROWS_SAME, true, true)
LQ_ATTN_PAGED(ROWS_LISTED, true, true)
}  // namespace lq
