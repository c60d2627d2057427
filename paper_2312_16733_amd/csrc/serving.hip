// C entries of the autoregressive serving operators: argument checks, then one or two launches.  Nothing here allocates or
// throws.
#include <cmath>

#include "host.h"
#include "paged.h"

namespace sna {

static bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

static sna_status check_cache(const sna_paged_cache* c) {
  if (!c || !c->k_pages_dev || !c->v_pages_dev) return fail(SNA_E_NULL, "paged cache: NULL pages");
  if (c->dtype != SNA_DTYPE_BF16 && c->dtype != SNA_DTYPE_FP16) return fail(SNA_E_CFG_RANGE, "paged cache: dtype %d (bf16 and fp16 are supported)", c->dtype);
  if (c->head_dim != 64 && c->head_dim != 128) return fail(SNA_E_CFG_RANGE, "paged cache: head_dim %d (64 and 128 are supported)", c->head_dim);
  if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)))
    return fail(SNA_E_CFG_RANGE, "paged cache: page_size %d (a power of two from 16 to 1024 is supported)", c->page_size);
  if (c->n_pages < 1 || c->kv_heads < 1 || c->kv_heads > 4096) return fail(SNA_E_CFG_RANGE, "paged cache: %d pages, %d heads", c->n_pages, c->kv_heads);
  const int64_t dense = (int64_t)c->kv_heads * c->page_size * c->head_dim;
  if (c->k_page_stride < dense || c->v_page_stride < dense) return fail(SNA_E_CFG_RANGE, "paged cache: pages overlap");
  if (!aligned16(c->k_pages_dev) || !aligned16(c->v_pages_dev) || c->k_page_stride % 8 || c->v_page_stride % 8)
    return fail(SNA_E_CFG_ALIGN, "paged cache: pages are not aligned to 16 bytes");
  return SNA_OK;
}

static sna_status check_batch(const sna_paged_batch* b) {
  if (!b) return fail(SNA_E_NULL, "paged batch: NULL");
  if (b->n_seqs < 0 || b->n_seqs > (1 << 20) || b->n_tokens < 0 || b->n_tokens > (1 << 26))
    return fail(SNA_E_CFG_RANGE, "paged batch: %d sequences, %d tokens", b->n_seqs, b->n_tokens);
  if (b->n_tokens == 0) return SNA_OK;                               // no work
  if (b->n_seqs == 0) return fail(SNA_E_CFG_RANGE, "paged batch: %d tokens of no sequence", b->n_tokens);
  if (!b->starts_dev || !b->lens_dev || !b->page_table_dev) return fail(SNA_E_NULL, "paged batch: NULL starts, lens or page table");
  if (b->table_width < 1 || b->table_stride < 0 || b->table_stride > INT32_MAX) return fail(SNA_E_CFG_RANGE, "paged batch: page table of %d columns", b->table_width);
  if (b->max_new < 1 || b->max_new > b->n_tokens || (int64_t)b->max_new * b->n_seqs < b->n_tokens)
    return fail(SNA_E_CFG_RANGE, "paged batch: max_new %d cannot hold for %d tokens of %d sequences", b->max_new, b->n_tokens, b->n_seqs);
  if (b->max_len < b->max_new || b->max_len > (1 << 30)) return fail(SNA_E_CFG_RANGE, "paged batch: max_len %d with max_new %d", b->max_len, b->max_new);
  return SNA_OK;
}

static sna_status check_heads(const sna_paged_cache* c, const sna_paged_batch* b, int32_t q_heads) {
  if (q_heads < 1 || q_heads % c->kv_heads || q_heads / c->kv_heads > 64)
    return fail(SNA_E_CFG_RANGE, "%d query heads over %d key / value heads (a multiple, up to 64 times, is supported)", q_heads, c->kv_heads);
  if (((int64_t)b->n_tokens + 2 * (int64_t)b->n_seqs) * q_heads > 1 << 30)         // so that no count of rows or blocks leaves 31 bits
    return fail(SNA_E_CFG_RANGE, "%d tokens of %d sequences and %d heads are more than one step takes", b->n_tokens, b->n_seqs, q_heads);
  return SNA_OK;
}

static sna_status check_rows(const sna_rows* r, const char* name) {
  if (!r || !r->dev) return fail(SNA_E_NULL, "%s is NULL", name);
  if (!aligned16(r->dev) || r->token_stride % 8 || r->head_stride % 8) return fail(SNA_E_CFG_ALIGN, "%s: rows are not aligned to 16 bytes", name);
  return SNA_OK;
}

// Rows that are written: none shares an element with another.  Of tokens and heads one changes fastest, and the other steps over
// all of its rows (so it is for every slice and transposition of a dense tensor).
static sna_status check_out(const sna_rows* r, const char* name, int64_t tokens, int64_t heads, int64_t dim) {
  const sna_status st = check_rows(r, name);
  if (st != SNA_OK) return st;
  typedef __int128 wide;                                             // strides are any 64-bit numbers
  const wide far = (wide)1 << 100, ts = r->token_stride, hs = r->head_stride;
  const wide t = tokens == 1 ? far : ts < 0 ? -ts : ts, h = heads == 1 ? far : hs < 0 ? -hs : hs;
  const wide inner = t < h ? t : h, outer = t < h ? h : t, rows = t < h ? tokens : heads;
  if (inner < dim || (outer != far && outer < inner * (rows - 1) + dim))
    return fail(SNA_E_CFG_RANGE, "%s: rows overlap", name);
  return SNA_OK;
}

static sna_status launched(hipError_t e, const char* what) {
  if (e == hipErrorInvalidConfiguration) return fail(SNA_E_CFG_RANGE, "%s: more blocks than a launch has", what);
  return e == hipSuccess ? SNA_OK : fail(SNA_E_HIP, "%s: %s", what, hipGetErrorString(e));
}

static PagedSeqs seqs_of(const sna_paged_batch* b) {
  return PagedSeqs{b->starts_dev, b->lens_dev, b->page_table_dev, b->n_seqs, b->n_tokens, b->table_width < (1 << 20) ? b->table_width : 1 << 20, (int)b->table_stride, b->max_len};   // 2^30 slots
}
static PagedKV kv_of(const sna_paged_cache* c) {
  return PagedKV{(char*)c->k_pages_dev, (char*)c->v_pages_dev, 2 * c->k_page_stride, 2 * c->v_page_stride, c->n_pages, __builtin_ctz(c->page_size), c->kv_heads};
}

}  // namespace sna

using namespace sna;

extern "C" {

sna_status sna_kv_append(const sna_paged_cache* cache, const sna_paged_batch* batch, int32_t q_heads, const sna_rows* q,
                         const sna_rows* k, const sna_rows* v, const sna_rows* q_out, const float* inv_freq_dev,
                         int32_t rot_dim, int32_t interleaved, const float* q_norm_dev, const float* k_norm_dev, float eps,
                         void* hip_stream) {
  sna_status st;
  if ((st = check_cache(cache)) != SNA_OK || (st = check_batch(batch)) != SNA_OK || (st = check_heads(cache, batch, q_heads)) != SNA_OK) return st;
  if (rot_dim < 0 || rot_dim > cache->head_dim || rot_dim % 16) return fail(SNA_E_CFG_RANGE, "rot_dim %d (a multiple of 16 up to head_dim is supported)", rot_dim);
  if (rot_dim && !inv_freq_dev) return fail(SNA_E_NULL, "inv_freq is NULL");
  if (!q_norm_dev != !k_norm_dev) return fail(SNA_E_NULL, "one of q_norm and k_norm is NULL");
  if (batch->n_tokens == 0) return SNA_OK;
  if ((st = check_rows(q, "q")) != SNA_OK || (st = check_rows(k, "k")) != SNA_OK || (st = check_rows(v, "v")) != SNA_OK ||
      (st = check_out(q_out, "q_out", batch->n_tokens, q_heads, cache->head_dim)) != SNA_OK) return st;
  AppendArgs a = {};
  a.s = seqs_of(batch);
  a.s.max_len = 1 << 30;                                             // a token is stored at its place, or nowhere
  a.kv = kv_of(cache);
  a.q = (const char*)q->dev; a.k = (const char*)k->dev; a.v = (const char*)v->dev; a.qo = (char*)q_out->dev;
  a.inv_freq = inv_freq_dev; a.q_norm = q_norm_dev; a.k_norm = k_norm_dev;
  a.q_t = 2 * q->token_stride; a.q_h = 2 * q->head_stride;
  a.k_t = 2 * k->token_stride; a.k_h = 2 * k->head_stride;
  a.v_t = 2 * v->token_stride; a.v_h = 2 * v->head_stride;
  a.o_t = 2 * q_out->token_stride; a.o_h = 2 * q_out->head_stride;
  a.Hq = q_heads; a.half = rot_dim / 2;
  a.eps = eps;
  a.interleaved = interleaved != 0;
  a.one = batch->max_new == 1 && batch->n_tokens == batch->n_seqs;
  const hipError_t e = launch_append(a, cache->dtype, cache->head_dim, (hipStream_t)hip_stream);
  return launched(e, "kv_append");
}


int64_t sna_paged_attention_workspace_bytes(const sna_paged_cache* cache, const sna_paged_batch* batch, int32_t q_heads, int32_t window) {
  sna_status st;
  if ((st = check_cache(cache)) != SNA_OK || (st = check_batch(batch)) != SNA_OK || (st = check_heads(cache, batch, q_heads)) != SNA_OK) return st;
  if (window < 0) return fail(SNA_E_CFG_RANGE, "window %d", window);
  if (batch->n_tokens == 0) return 0;
  return (int64_t)paged_attention_workspace(batch->n_seqs, batch->n_tokens, cache->kv_heads, q_heads / cache->kv_heads, batch->max_new, batch->max_len, window, cache->head_dim);
}

sna_status sna_paged_attention(const sna_paged_cache* cache, const sna_paged_batch* batch, int32_t q_heads,
                               const sna_rows* q, const sna_rows* out, float scale, int32_t window, void* workspace_dev,
                               size_t workspace_bytes, void* hip_stream) {
  sna_status st;
  const int64_t need = sna_paged_attention_workspace_bytes(cache, batch, q_heads, window);
  if (need < 0) return (sna_status)need;
  const float scale2 = scale * 1.44269504088896340736f;              // of powers of two
  if (!(scale > 0.f && scale2 < INFINITY)) return fail(SNA_E_CFG_RANGE, "scale %g (a positive number is needed)", (double)scale);
  if (batch->n_tokens == 0) return SNA_OK;
  if ((st = check_rows(q, "q")) != SNA_OK || (st = check_out(out, "out", batch->n_tokens, q_heads, cache->head_dim)) != SNA_OK) return st;
  if (need > 0 && (!workspace_dev || workspace_bytes < (size_t)need || !aligned16(workspace_dev)))
    return fail(SNA_E_WORKSPACE, "paged_attention: a workspace of %lld bytes, 16-byte aligned, is needed", (long long)need);
  PagedAttnArgs a = {};
  a.s = seqs_of(batch);
  a.kv = kv_of(cache);
  a.q = (const char*)q->dev; a.o = (char*)out->dev;
  a.q_t = 2 * q->token_stride; a.q_h = 2 * q->head_stride;
  a.o_t = 2 * out->token_stride; a.o_h = 2 * out->head_stride;
  a.G = q_heads / cache->kv_heads;
  a.window = window ? window : INT32_MAX;
  a.scale2 = scale2;
  a.max_new = batch->max_new;
  const hipError_t e = launch_paged_attention(a, cache->dtype, cache->head_dim, batch->max_len, workspace_dev, (hipStream_t)hip_stream);
  return launched(e, "paged_attention");
}

sna_status sna_verify_draft(const float* target_dev, int64_t target_seq_stride, int64_t target_row_stride, const float* draft_dev,
                            int64_t draft_seq_stride, int64_t draft_row_stride, const void* tokens_dev, int32_t token_bytes,
                            const float* uniforms_dev, const int32_t* n_draft_dev, int32_t n_seqs, int32_t n_steps, int32_t vocab,
                            int32_t* out_dev, int32_t* accepted_dev, void* hip_stream) {
  if (n_seqs < 0 || n_seqs > (1 << 24) || n_steps < 0 || n_steps > (1 << 16) || vocab < 1 || vocab > (1 << 28))
    return fail(SNA_E_CFG_RANGE, "verify_draft: %d sequences, %d drafts, vocabulary of %d", n_seqs, n_steps, vocab);
  if (token_bytes != 4 && token_bytes != 8) return fail(SNA_E_CFG_RANGE, "verify_draft: tokens of %d bytes (4 and 8 are supported)", token_bytes);
  if (target_seq_stride < 0 || target_row_stride < 0 || draft_seq_stride < 0 || draft_row_stride < 0) return fail(SNA_E_CFG_RANGE, "verify_draft: negative strides");
  if (n_seqs == 0) return SNA_OK;
  if (!target_dev || (n_steps && !tokens_dev) || !uniforms_dev || !out_dev || !accepted_dev) return fail(SNA_E_NULL, "verify_draft: a required pointer is NULL");
  if (((uintptr_t)target_dev | (uintptr_t)draft_dev | (uintptr_t)uniforms_dev | (uintptr_t)n_draft_dev | (uintptr_t)out_dev | (uintptr_t)accepted_dev) & 3 ||
      (uintptr_t)tokens_dev & (token_bytes - 1))
    return fail(SNA_E_CFG_ALIGN, "verify_draft: a pointer is not aligned to its elements");
  const VerifyArgs a = {target_dev, draft_dev, target_seq_stride, target_row_stride, draft_seq_stride, draft_row_stride, tokens_dev, uniforms_dev,
                        n_draft_dev, out_dev, accepted_dev, n_steps, vocab};
  const hipError_t e = launch_verify(a, token_bytes, n_seqs, (hipStream_t)hip_stream);
  return launched(e, "verify_draft");
}

}
