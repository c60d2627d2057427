// Attention of the tokens of drafted trees over the paged cache, few rows of queries per key / value head: kernels in pattn_kernel.h.
#include "pattn_kernel.h"

namespace sna {

static AttnPlan plan_of(const PagedSeqs& s, int kv_heads, int group, int max_new, int max_len, int window, int words, int head_dim) {
  return plan_of_tree(s.B, s.T, kv_heads, group, max_new, max_len, window == INT_MAX ? 0 : tree_window(window, words), head_dim);
}

size_t tree_attention_workspace(const PagedSeqs& s, int kv_heads, int group, int max_new, int max_len, int window, int words, int head_dim) {
  return plan_of(s, kv_heads, group, max_new, max_len, window, words, head_dim).parts;
}

hipError_t launch_tree_attention(PagedAttnArgs a, int dtype, int head_dim, int max_len, void* workspace, hipStream_t s) {
  const AttnPlan p = plan_of(a.s, a.kv.heads, a.G, a.max_new, max_len, a.window, a.words, head_dim);
  a.most = p.most;
  a.parts = p.blocks ? workspace : nullptr;
  a.blocks = p.blocks;
  a.waves = p.waves;
  return p.mb ? launch_rows<true>(a, p.mb, dtype, head_dim, s) : launch_tree_chunks(a, dtype, head_dim, s);
}

}  // namespace sna
