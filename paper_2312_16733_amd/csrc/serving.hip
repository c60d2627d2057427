// C entries of the autoregressive serving operators: argument checks, then one or two launches.  Nothing here allocates or
// throws.
#include <cmath>

#include "host.h"
#include "paged.h"

namespace sna {

typedef __int128 wide;                                               // strides are any 64-bit numbers

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
  return sna_kv_append_at(cache, batch, q_heads, q, k, v, q_out, inv_freq_dev, rot_dim, interleaved, q_norm_dev, k_norm_dev, eps, nullptr, hip_stream);
}

sna_status sna_kv_append_at(const sna_paged_cache* cache, const sna_paged_batch* batch, int32_t q_heads, const sna_rows* q,
                            const sna_rows* k, const sna_rows* v, const sna_rows* q_out, const float* inv_freq_dev,
                            int32_t rot_dim, int32_t interleaved, const float* q_norm_dev, const float* k_norm_dev, float eps,
                            const int32_t* positions_dev, void* hip_stream) {
  sna_status st;
  if ((st = check_cache(cache)) != SNA_OK || (st = check_batch(batch)) != SNA_OK || (st = check_heads(cache, batch, q_heads)) != SNA_OK) return st;
  if (rot_dim < 0 || rot_dim > cache->head_dim || rot_dim % 16) return fail(SNA_E_CFG_RANGE, "rot_dim %d (a multiple of 16 up to head_dim is supported)", rot_dim);
  if (rot_dim && !inv_freq_dev) return fail(SNA_E_NULL, "inv_freq is NULL");
  if (!q_norm_dev != !k_norm_dev) return fail(SNA_E_NULL, "one of q_norm and k_norm is NULL");
  if ((uintptr_t)positions_dev & 3) return fail(SNA_E_CFG_ALIGN, "positions are not aligned to their elements");
  if (batch->n_tokens == 0) return SNA_OK;
  if ((st = check_rows(q, "q")) != SNA_OK || (st = check_rows(k, "k")) != SNA_OK || (st = check_rows(v, "v")) != SNA_OK ||
      (st = check_out(q_out, "q_out", batch->n_tokens, q_heads, cache->head_dim)) != SNA_OK) return st;
  AppendArgs a = {};
  a.s = seqs_of(batch);
  a.s.max_len = 1 << 30;                                             // a token is stored at its place, or nowhere
  a.kv = kv_of(cache);
  a.q = (const char*)q->dev; a.k = (const char*)k->dev; a.v = (const char*)v->dev; a.qo = (char*)q_out->dev;
  a.inv_freq = inv_freq_dev; a.q_norm = q_norm_dev; a.k_norm = k_norm_dev;
  a.positions = positions_dev;
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

static sna_status attend(const sna_paged_cache* cache, const sna_paged_batch* batch, int32_t q_heads, const sna_rows* q, const sna_rows* out, float scale, int32_t window,
                         int64_t need, void* workspace_dev, size_t workspace_bytes, PagedAttnArgs a, void* hip_stream, const char* name) {
  sna_status st;
  if (need < 0) return (sna_status)need;
  const float scale2 = scale * 1.44269504088896340736f;              // of powers of two
  if (!(scale > 0.f && scale2 < INFINITY)) return fail(SNA_E_CFG_RANGE, "scale %g (a positive number is needed)", (double)scale);
  if (batch->n_tokens == 0) return SNA_OK;
  if ((st = check_rows(q, "q")) != SNA_OK || (st = check_out(out, "out", batch->n_tokens, q_heads, cache->head_dim)) != SNA_OK) return st;
  if (need > 0 && (!workspace_dev || workspace_bytes < (size_t)need || !aligned16(workspace_dev)))
    return fail(SNA_E_WORKSPACE, "%s: a workspace of %lld bytes, 16-byte aligned, is needed", name, (long long)need);
  a.s = seqs_of(batch);
  a.kv = kv_of(cache);
  a.q = (const char*)q->dev; a.o = (char*)out->dev;
  a.q_t = 2 * q->token_stride; a.q_h = 2 * q->head_stride;
  a.o_t = 2 * out->token_stride; a.o_h = 2 * out->head_stride;
  a.G = q_heads / cache->kv_heads;
  a.window = window ? window : INT32_MAX;
  a.scale2 = scale2;
  a.max_new = batch->max_new;
  const hipError_t e = (a.masks ? launch_tree_attention : launch_paged_attention)(a, cache->dtype, cache->head_dim, batch->max_len, workspace_dev, (hipStream_t)hip_stream);
  return launched(e, name);
}

sna_status sna_paged_attention(const sna_paged_cache* cache, const sna_paged_batch* batch, int32_t q_heads,
                               const sna_rows* q, const sna_rows* out, float scale, int32_t window, void* workspace_dev,
                               size_t workspace_bytes, void* hip_stream) {
  const int64_t need = sna_paged_attention_workspace_bytes(cache, batch, q_heads, window);
  return attend(cache, batch, q_heads, q, out, scale, window, need, workspace_dev, workspace_bytes, PagedAttnArgs{}, hip_stream, "paged_attention");
}

int64_t sna_tree_attention_workspace_bytes(const sna_paged_cache* cache, const sna_paged_batch* batch, int32_t q_heads, int32_t mask_words, int32_t window) {
  sna_status st;
  if (mask_words < 1 || mask_words > 64) return fail(SNA_E_CFG_RANGE, "masks of %d words (1 to 64 are supported)", mask_words);
  if ((st = check_cache(cache)) != SNA_OK || (st = check_batch(batch)) != SNA_OK || (st = check_heads(cache, batch, q_heads)) != SNA_OK) return st;
  if (window < 0) return fail(SNA_E_CFG_RANGE, "window %d", window);
  if (batch->n_tokens == 0) return 0;
  return (int64_t)tree_attention_workspace(seqs_of(batch), cache->kv_heads, q_heads / cache->kv_heads, batch->max_new, batch->max_len, window ? window : INT32_MAX, mask_words, cache->head_dim);
}

sna_status sna_tree_attention(const sna_paged_cache* cache, const sna_paged_batch* batch, int32_t q_heads, const sna_rows* q, const sna_rows* out,
                              const uint64_t* masks_dev, int32_t mask_words, const int32_t* prefix_dev, const int32_t* positions_dev, float scale,
                              int32_t window, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  const int64_t need = sna_tree_attention_workspace_bytes(cache, batch, q_heads, mask_words, window);
  if (need < 0) return (sna_status)need;
  if (batch->n_tokens > 0 && !masks_dev) return fail(SNA_E_NULL, "masks are NULL");
  if (batch->n_tokens > 0 && !prefix_dev && batch->max_new > 64 * mask_words)
    return fail(SNA_E_CFG_RANGE, "masks of %d words do not reach the last of %d tokens", mask_words, batch->max_new);
  if ((uintptr_t)masks_dev & 7 || ((uintptr_t)prefix_dev | (uintptr_t)positions_dev) & 3) return fail(SNA_E_CFG_ALIGN, "masks, prefix or positions are not aligned to their elements");
  PagedAttnArgs a = {};
  a.masks = (const unsigned long long*)masks_dev;
  a.words = mask_words;
  a.prefix = prefix_dev;
  a.positions = positions_dev;
  return attend(cache, batch, q_heads, q, out, scale, window, need, workspace_dev, workspace_bytes, a, hip_stream, "tree_attention");
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

// No byte of both
struct Bytes { const void* at; int64_t n; };
static bool apart(const Bytes& a, const Bytes& b) {
  const uintptr_t p = (uintptr_t)a.at, q = (uintptr_t)b.at;
  return a.n <= 0 || b.n <= 0 || (p <= q ? q - p >= (uintptr_t)a.n : p - q >= (uintptr_t)b.n);
}
// The same of rows of bytes, which may lie between each other's
struct ByteRows { Bytes row; int64_t n; wide stride; };
static bool apart(const ByteRows& a, const ByteRows& b) {
  const auto last = [](const ByteRows& x) { return (wide)(uintptr_t)x.row.at + (x.n - 1) * x.stride; };
  const auto first = [](const ByteRows& x) { return (wide)(uintptr_t)x.row.at; };
  if (!a.row.at || !b.row.at || last(a) + a.row.n <= first(b) || last(b) + b.row.n <= first(a)) return true;
  for (int64_t i = 0; i < a.n; ++i) {
    const wide x = first(a) + i * a.stride, before = x - first(b) - b.row.n;                   // a row of b that begins no later ends before this one
    const wide j = before < 0 ? 0 : b.stride ? before / b.stride + 1 : b.n;
    if (j < b.n && first(b) + j * b.stride < x + a.row.n) return false;
  }
  return true;
}

sna_status sna_verify_tree(const sna_paged_batch* batch, const void* sampled_dev, int32_t sampled_bytes, const void* tokens_dev, int32_t token_bytes,
                           const int32_t* parents_dev, int32_t* kept_dev, int32_t* counts_dev, int32_t* next_dev, void* hip_stream) {
  if (!batch) return fail(SNA_E_NULL, "paged batch: NULL");
  if (batch->n_seqs < 0 || batch->n_seqs > (1 << 20) || batch->n_tokens < 0 || batch->n_tokens > (1 << 26) || batch->max_new < 0 || batch->max_new > kTreeTokens)
    return fail(SNA_E_CFG_RANGE, "verify_tree: %d sequences, %d tokens, trees of %d (up to %d are supported)", batch->n_seqs, batch->n_tokens, batch->max_new, kTreeTokens);
  for (const int32_t bytes : {sampled_bytes, token_bytes})
    if (bytes != 4 && bytes != 8) return fail(SNA_E_CFG_RANGE, "verify_tree: tokens of %d bytes (4 and 8 are supported)", bytes);
  if (batch->n_seqs == 0) return batch->n_tokens ? fail(SNA_E_CFG_RANGE, "paged batch: %d tokens of no sequence", batch->n_tokens) : SNA_OK;
  if (!batch->starts_dev || !batch->lens_dev || (batch->n_tokens && (!sampled_dev || !tokens_dev || !parents_dev)) || (batch->max_new && !kept_dev) || !counts_dev || !next_dev)
    return fail(SNA_E_NULL, "verify_tree: a required pointer is NULL");
  if (((uintptr_t)parents_dev | (uintptr_t)kept_dev | (uintptr_t)counts_dev | (uintptr_t)next_dev) & 3 || (uintptr_t)sampled_dev & (sampled_bytes - 1) || (uintptr_t)tokens_dev & (token_bytes - 1))
    return fail(SNA_E_CFG_ALIGN, "verify_tree: a pointer is not aligned to its elements");
  const int64_t n = batch->n_seqs, tokens = batch->n_tokens;
  const Bytes out[] = {{kept_dev, 4 * n * batch->max_new}, {counts_dev, 4 * n}, {next_dev, 4 * n}};
  const Bytes in[] = {{batch->starts_dev, 4 * n + 4}, {batch->lens_dev, 4 * n}, {sampled_dev, sampled_bytes * tokens}, {tokens_dev, token_bytes * tokens}, {parents_dev, 4 * tokens}};
  for (int i = 0; i < 3; ++i) {
    bool free = true;
    for (const Bytes& x : in) free = free && apart(out[i], x);
    for (int j = 0; j < i; ++j) free = free && apart(out[i], out[j]);
    if (!free) return fail(SNA_E_CFG_RANGE, "verify_tree: a result is written over another or over what is read");
  }
  const TreeWalkArgs a = {seqs_of(batch), sampled_dev, tokens_dev, sampled_bytes, token_bytes, parents_dev, kept_dev, counts_dev, next_dev, batch->max_new};
  return launched(launch_verify_tree(a, (hipStream_t)hip_stream), "verify_tree");
}

sna_status sna_kv_compact(const sna_paged_cache* cache, const sna_paged_batch* batch, const int32_t* kept_dev, int32_t kept_width, const int32_t* counts_dev,
                          int32_t* lens_dev, void* hip_stream) {
  sna_status st;
  if ((st = check_cache(cache)) != SNA_OK) return st;
  if (!batch) return fail(SNA_E_NULL, "paged batch: NULL");
  if (batch->n_seqs < 0 || batch->n_seqs > (1 << 20) || batch->max_new < 0 || batch->max_new > (1 << 26) || kept_width < 0 || kept_width > (1 << 26))
    return fail(SNA_E_CFG_RANGE, "kv_compact: %d sequences, %d new tokens, %d kept", batch->n_seqs, batch->max_new, kept_width);
  if (batch->n_seqs == 0) return SNA_OK;
  if (!batch->starts_dev || !batch->lens_dev || !batch->page_table_dev || (kept_width && !kept_dev) || !counts_dev || !lens_dev)
    return fail(SNA_E_NULL, "kv_compact: a required pointer is NULL");
  if (batch->table_width < 1 || batch->table_stride < 0 || batch->table_stride > INT32_MAX) return fail(SNA_E_CFG_RANGE, "paged batch: page table of %d columns", batch->table_width);
  const int64_t n = batch->n_seqs;
  for (const Bytes& x : {Bytes{batch->lens_dev, 4 * n}, Bytes{batch->starts_dev, 4 * n + 4}, Bytes{batch->page_table_dev, 4 * ((n - 1) * batch->table_stride + batch->table_width)},
                         Bytes{counts_dev, 4 * n}, Bytes{kept_dev, 4 * n * kept_width}})
    if (!apart(Bytes{lens_dev, 4 * n}, x)) return fail(SNA_E_CFG_RANGE, "kv_compact: the new lengths are written over what is read");
  if (((uintptr_t)kept_dev | (uintptr_t)counts_dev | (uintptr_t)lens_dev) & 3) return fail(SNA_E_CFG_ALIGN, "kv_compact: a pointer is not aligned to its elements");
  CompactArgs a = {};
  a.s = seqs_of(batch);
  a.s.T = INT32_MAX / 2;                                             // rows are not looked at
  a.s.max_len = 1 << 30;
  a.kv = kv_of(cache);
  a.kept = kept_dev; a.counts = counts_dev; a.lens = lens_dev;
  a.width = kept_width;
  a.max_new = batch->max_new;
  a.dim = cache->head_dim;
  return launched(launch_compact(a, (hipStream_t)hip_stream), "kv_compact");
}

sna_status sna_copy_pages(const sna_paged_cache* cache, const int32_t* source_dev, const int32_t* target_dev, int32_t n, void* hip_stream) {
  sna_status st;
  if ((st = check_cache(cache)) != SNA_OK) return st;
  if (n < 0) return fail(SNA_E_CFG_RANGE, "copy_pages: %d pages", n);
  if (n == 0) return SNA_OK;
  if (!source_dev || !target_dev) return fail(SNA_E_NULL, "copy_pages: a required pointer is NULL");
  if (((uintptr_t)source_dev | (uintptr_t)target_dev) & 3) return fail(SNA_E_CFG_ALIGN, "copy_pages: a pointer is not aligned to its elements");
  PageCopyArgs a = {};
  a.kv = kv_of(cache);
  a.source = source_dev; a.target = target_dev;
  a.bytes = 2l * cache->kv_heads * cache->page_size * cache->head_dim;
  return launched(launch_copy_pages(a, n, (hipStream_t)hip_stream), "copy_pages");
}

static sna_status check_sampling(const sna_sampling* s) {
  if (!s) return fail(SNA_E_NULL, "sampling: NULL");
  if (s->n_rows < 0 || s->n_rows > (1 << 24) || s->vocab < 1 || s->vocab > (1 << 20) || s->row_stride < 0)
    return fail(SNA_E_CFG_RANGE, "sample_tokens: %d rows, vocabulary of %d (up to 2^20 is supported)", s->n_rows, s->vocab);
  if (s->dtype < SNA_DTYPE_FP32 || s->dtype > SNA_DTYPE_FP16) return fail(SNA_E_CFG_RANGE, "sample_tokens: dtype %d", s->dtype);
  if (!s->temperature_dev && !(s->temperature >= 0.f && s->temperature < INFINITY)) return fail(SNA_E_CFG_RANGE, "sample_tokens: temperature %g", (double)s->temperature);
  if (!s->top_k_dev && s->top_k < 0) return fail(SNA_E_CFG_RANGE, "sample_tokens: top_k %d", s->top_k);
  if (!s->top_p_dev && !(s->top_p >= 0.f && s->top_p <= 1.f)) return fail(SNA_E_CFG_RANGE, "sample_tokens: top_p %g", (double)s->top_p);
  if (!s->min_p_dev && !(s->min_p >= 0.f && s->min_p <= 1.f)) return fail(SNA_E_CFG_RANGE, "sample_tokens: min_p %g", (double)s->min_p);
  return SNA_OK;
}

int64_t sna_sample_tokens_workspace_bytes(const sna_sampling* s) {
  const sna_status st = check_sampling(s);
  return st != SNA_OK ? st : s->n_rows ? (int64_t)sample_workspace(s->n_rows, s->vocab) : 0;
}

sna_status sna_sample_tokens(const sna_sampling* s, int32_t* tokens_dev, float* probs_dev, int64_t probs_stride, void* workspace_dev, size_t workspace_bytes,
                             void* hip_stream) {
  const int64_t need = sna_sample_tokens_workspace_bytes(s);
  if (need < 0) return (sna_status)need;
  if (s->n_rows == 0) return SNA_OK;
  if (!s->logits_dev || !s->uniforms_dev || !tokens_dev) return fail(SNA_E_NULL, "sample_tokens: a required pointer is NULL");
  if (probs_dev && s->n_rows > 1 && probs_stride < s->vocab) return fail(SNA_E_CFG_RANGE, "sample_tokens: rows of probabilities overlap");
  if (((uintptr_t)s->uniforms_dev | (uintptr_t)s->temperature_dev | (uintptr_t)s->top_k_dev | (uintptr_t)s->top_p_dev | (uintptr_t)s->min_p_dev | (uintptr_t)tokens_dev | (uintptr_t)probs_dev) & 3 ||
      (uintptr_t)s->logits_dev & (s->dtype == SNA_DTYPE_FP32 ? 3 : 1))
    return fail(SNA_E_CFG_ALIGN, "sample_tokens: a pointer is not aligned to its elements");
  if (need > 0 && (!workspace_dev || workspace_bytes < (size_t)need || !aligned16(workspace_dev)))
    return fail(SNA_E_WORKSPACE, "sample_tokens: a workspace of %lld bytes, 16-byte aligned, is needed", (long long)need);
  const int64_t n = s->n_rows, size = s->dtype == SNA_DTYPE_FP32 ? 4 : 2;
  const ByteRows tokens = {{tokens_dev, 4 * n}, 1, 0}, probs = {{probs_dev, 4l * s->vocab}, n, (wide)4 * probs_stride}, logits = {{s->logits_dev, size * s->vocab}, n, (wide)size * s->row_stride};
  bool free = apart(tokens, probs) && apart(tokens, logits) && apart(probs, logits);
  for (const void* x : {(const void*)s->uniforms_dev, (const void*)s->temperature_dev, (const void*)s->top_p_dev, (const void*)s->min_p_dev, (const void*)s->top_k_dev})
    free = free && apart(tokens, ByteRows{{x, 4 * n}, 1, 0}) && apart(ByteRows{{x, 4 * n}, 1, 0}, probs);
  if (!free) return fail(SNA_E_CFG_RANGE, "sample_tokens: a result is written over another or over what is read");
  SampleArgs a = {};
  a.logits = s->logits_dev; a.stride = s->row_stride;
  a.u = s->uniforms_dev;
  a.temperature_of = s->temperature_dev; a.top_k_of = s->top_k_dev; a.top_p_of = s->top_p_dev; a.min_p_of = s->min_p_dev;
  a.temperature = s->temperature; a.top_k = s->top_k; a.top_p = s->top_p; a.min_p = s->min_p;
  a.V = s->vocab; a.n = s->n_rows;
  a.tokens = tokens_dev; a.probs = probs_dev; a.p_stride = probs_stride;
  a.work = workspace_dev;
  return launched(launch_sample(a, s->dtype, (hipStream_t)hip_stream), "sample_tokens");
}

}
