// Attention of the tokens of drafted trees over the paged cache, few rows of queries per key / value head: kernels in pattn_kernel.h.
#include "pattn_kernel.h"

namespace sna {

hipError_t launch_tree_attention(PagedAttnArgs a, int dtype, int head_dim, int max_len, void* workspace, hipStream_t s) {
  return launch_attention<true>(a, dtype, head_dim, max_len, a.window == INT_MAX ? 0 : tree_window(a.window, a.words), workspace, s);
}

}  // namespace sna
