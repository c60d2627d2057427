// Attention of the tokens of drafted trees over the paged cache, many rows of queries per key / value head: kernels in pprefill_kernel.h.
#include "pprefill_kernel.h"

namespace sna {

hipError_t launch_tree_chunks(const PagedAttnArgs& a, int dtype, int head_dim, hipStream_t s) { return launch_chunks<true>(a, dtype, head_dim, s); }

}  // namespace sna
