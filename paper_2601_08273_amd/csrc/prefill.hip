// Attention of whole prompts, or of their next pieces, packed without padding: rows_attention.h has the kernel.
#include "rows_attention.h"

namespace hippo {

hipError_t launch_prefill(const RowsParams& p, const RowsPlan& pl, int dtype, int head_dim, hipStream_t st) {
  return launch_rows<false>(p, pl, dtype, head_dim, st);
}

}  // namespace hippo
