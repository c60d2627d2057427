// Attention of a step's new tokens over the paged cache, causal: kernels in pattn_kernel.h.
#include "pattn_kernel.h"

namespace sna {

size_t paged_attention_workspace(int n_seqs, int n_tokens, int kv_heads, int group, int max_new, int max_len, int window, int head_dim) {
  const AttnPlan p = plan_of(n_seqs, n_tokens, kv_heads, group, max_new, max_len, window, head_dim);
  return p.parts + p.chunk_parts;
}

hipError_t launch_paged_attention(PagedAttnArgs a, int dtype, int head_dim, int max_len, void* workspace, hipStream_t s) {
  const AttnPlan p = plan_of(a.s.B, a.s.T, a.kv.heads, a.G, a.max_new, max_len, a.window == INT_MAX ? 0 : a.window, head_dim);
  a.most = p.most;
  a.waves = p.chunk.waves;
  a.splits = p.chunk.splits;
  if (p.chunks && !chunks_fit_a_launch(a)) return hipErrorInvalidConfiguration;        // before anything is launched
  if (p.mb) {
    PagedAttnArgs r = a;
    r.parts = p.blocks ? workspace : nullptr;
    r.blocks = p.blocks;
    r.waves = p.waves;
    const hipError_t e = launch_rows<false>(r, p.mb, dtype, head_dim, s);
    if (e != hipSuccess || !p.chunks) return e;
  }
  a.parts = (char*)workspace + p.parts;
  return launch_paged_chunks(a, dtype, head_dim, s);
}

}  // namespace sna
