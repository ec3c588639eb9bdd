// Attention of a tree of drafted tokens over a cache: rows_attention.h has the kernel.
#include "rows_attention.h"

namespace hippo {

hipError_t launch_tree(const RowsParams& p, const RowsPlan& pl, int dtype, int head_dim, hipStream_t st) {
  return launch_rows<true>(p, pl, dtype, head_dim, st);
}

}  // namespace hippo
