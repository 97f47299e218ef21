// Kernels of attention over the paged cache: with a cap, a bias or weights.
#include "lq_attn_paged.h"

namespace lq {
LQ_ATTN_PAGED(ROWS_SAME, false, true)
LQ_ATTN_PAGED(ROWS_LISTED, false, true)
}  // namespace lq
