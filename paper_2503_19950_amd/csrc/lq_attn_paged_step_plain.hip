// Kernels of attention over the paged cache: a step whose scores are as they are.
#include "lq_attn_paged.h"

namespace lq {
LQ_ATTN_PAGED(ROWS_SAME, true, false)
LQ_ATTN_PAGED(ROWS_LISTED, true, false)
}  // namespace lq
