// Kernels of attention over the paged cache: scores as they are.
#include "lq_attn_paged.h"

namespace lq {
LQ_ATTN_PAGED(ROWS_SAME, false, false)
LQ_ATTN_PAGED(ROWS_LISTED, false, false)
}  // namespace lq
