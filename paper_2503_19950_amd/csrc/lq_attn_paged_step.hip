// Kernels of attention over the paged cache: a step with a cap, a bias or weights.
#include "lq_attn_paged.h"

namespace lq {
LQ_ATTN_PAGED(ROWS_SAME, true, true)
LQ_ATTN_PAGED(ROWS_LISTED, true, true)
}  // namespace lq
