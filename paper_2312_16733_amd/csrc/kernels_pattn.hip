// Attention of a step's new tokens over the paged cache, causal: kernels in pattn_kernel.h.
#include "pattn_kernel.h"

namespace sna {

size_t paged_attention_workspace(int n_seqs, int n_tokens, int kv_heads, int group, int max_new, int max_len, int window, int head_dim) {
  const AttnPlan p = plan_of(n_seqs, n_tokens, kv_heads, group, max_new, max_len, window, head_dim);
  return p.parts + p.chunk_parts;
}

hipError_t launch_paged_attention(PagedAttnArgs a, int dtype, int head_dim, int max_len, void* workspace, hipStream_t s) {
  return launch_attention<false>(a, dtype, head_dim, max_len, a.window == INT_MAX ? 0 : a.window, workspace, s);
}

}  // namespace sna
