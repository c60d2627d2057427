"""Autoregressive serving over a paged key / value cache: the operators of include/subnetact.h on torch tensors.

    cache = PagedCache(k_pages, v_pages)                      # one layer's pages
    batch = PagedBatch(starts, lens, page_table, max_new, max_len)
    q = kv_append(cache, batch, q, k, v, inv_freq=inv_freq)   # norms, rotation, k and v into their pages
    out = paged_attention(cache, batch, q)
    tokens, accepted = verify_draft(target, drafted, uniforms)      # speculative decoding: which drafts stand, and the next token

Rows are the new tokens of all sequences of a step, one after the other.  Nothing here reads device memory or waits for it;
`PagedBatch.validate` does, for a caller in doubt about what its arrays hold.
"""
import torch

from . import binding
from .binding import PagedBatchC, PagedCacheC, RowsC, _check

_DTYPES = {torch.bfloat16: binding.DTYPE["bf16"], torch.float16: binding.DTYPE["fp16"]}


class _On:
    """The stream a call is enqueued on and its outputs belong to: the current one, a torch stream, or a raw handle."""

    def __init__(self, device, stream):
        if not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(stream, device=device)
        self.context = torch.cuda.stream(stream)

    def __enter__(self):
        self.context.__enter__()

    def __exit__(self, *a):
        return self.context.__exit__(*a)


def _need(ok, text):
    if not ok:
        raise ValueError(text)


def _index(t, name, device):
    _need(t.dtype == torch.int32 and t.device == device, f"{name}: int32 on {device} is needed, got {t.dtype} on {t.device}")


class PagedCache:
    """One layer's pages: keys [pages][kv_heads][page_size][head_dim], values [pages][kv_heads][head_dim][page_size], bf16 or
    fp16, dense within a page; the layers of a pool may take turns (any stride between pages).  Borrowed, not copied."""
    __slots__ = ("k_pages", "v_pages", "dtype", "device", "kv_heads", "page_size", "head_dim", "n_pages", "c")

    def __init__(self, k_pages, v_pages):
        _need(k_pages.dim() == 4 and v_pages.dim() == 4, "k_pages and v_pages have four dimensions")
        n, h, ps, d = k_pages.shape
        _need(v_pages.shape == (n, h, d, ps), f"v_pages: {(n, h, d, ps)} is needed, got {tuple(v_pages.shape)}")
        _need(k_pages.dtype in _DTYPES and v_pages.dtype == k_pages.dtype, f"pages of {k_pages.dtype} and {v_pages.dtype}: both bf16 or both fp16 are needed")
        _need(k_pages.is_cuda and v_pages.device == k_pages.device, f"pages on {k_pages.device} and {v_pages.device}: one GPU is needed")
        ks, vs = k_pages.stride(), v_pages.stride()
        _need(ks[1:] == (ps * d, d, 1) and vs[1:] == (d * ps, ps, 1), "pages have to be dense")
        self.k_pages, self.v_pages, self.dtype, self.device = k_pages, v_pages, k_pages.dtype, k_pages.device
        self.n_pages, self.kv_heads, self.page_size, self.head_dim = n, h, ps, d
        dense = h * ps * d
        self.c = PagedCacheC(k_pages.data_ptr(), v_pages.data_ptr(), ks[0] if n > 1 else dense, vs[0] if n > 1 else dense, n, h, ps, d, _DTYPES[k_pages.dtype])


class PagedBatch:
    """The sequences of one step.  starts int32 [n + 1]: sequence b brings rows starts[b] .. starts[b + 1] - 1 (none is fine);
    lens int32 [n]: its cached tokens once these are in; page_table int32 [n][width].  max_new and max_len bound the new tokens
    and the length of any sequence; they choose the launches, so bounds near the truth are faster."""
    __slots__ = ("starts", "lens", "page_table", "max_new", "max_len", "n_seqs", "device", "c")

    def __init__(self, starts, lens, page_table, max_new, max_len):
        n, device = lens.shape[0] if lens.dim() == 1 else -1, lens.device
        _need(n >= 0 and lens.is_cuda, "lens: one dimension on a GPU is needed")
        for t, name in ((starts, "starts"), (lens, "lens"), (page_table, "page_table")):
            _index(t, name, device)
        _need(starts.shape == (n + 1,), f"starts: {n + 1} entries are needed for {n} sequences, got {tuple(starts.shape)}")
        _need(page_table.dim() == 2 and page_table.shape[0] == n, f"page_table: {n} rows are needed, got {tuple(page_table.shape)}")
        _need(starts.is_contiguous() and lens.is_contiguous() and (page_table.stride(1) == 1 or page_table.shape[1] <= 1), "starts, lens and the rows of page_table have to be dense")
        self.starts, self.lens, self.page_table, self.n_seqs, self.device = starts, lens, page_table, n, device
        self.max_new, self.max_len = int(max_new), int(max_len)
        self.c = PagedBatchC(starts.data_ptr(), lens.data_ptr(), page_table.data_ptr(), page_table.stride(0), n, 0, page_table.shape[1], self.max_new, self.max_len)

    def validate(self, cache, n_tokens):
        """Reads the arrays back (waits for the GPU) and raises ValueError where they do not fit the cache, each other or the bounds."""
        starts, lens, table = (t.cpu().long() for t in (self.starts, self.lens, self.page_table))
        new = starts[1:] - starts[:-1]
        _need(int(starts[0]) == 0 and int(starts[-1]) == n_tokens and bool((new >= 0).all()), f"starts have to rise from 0 to {n_tokens}")
        _need(bool((new <= self.max_new).all()), f"a sequence brings more than max_new = {self.max_new} tokens")
        _need(bool((lens >= new).all()), "a sequence is shorter than its new tokens")
        _need(bool((lens <= self.max_len).all()), f"a sequence is longer than max_len = {self.max_len}")
        pages = (lens + cache.page_size - 1) // cache.page_size
        _need(bool((pages <= table.shape[1]).all()), f"a sequence is longer than its {table.shape[1]} table entries")
        used = torch.arange(table.shape[1])[None] < pages[:, None]
        _need(bool(((table >= 0) & (table < cache.n_pages))[used].all()), f"a page outside the {cache.n_pages} of the pool")


def _rows(t, name, heads, cache):
    _need(t.dim() == 3 and t.shape[2] == cache.head_dim and (heads is None or t.shape[1] == heads),
          f"{name}: [tokens][{heads or 'heads'}][{cache.head_dim}] is needed, got {tuple(t.shape)}")
    _need(t.dtype == cache.dtype and t.device == cache.device, f"{name}: {cache.dtype} on {cache.device} is needed, got {t.dtype} on {t.device}")
    s = t.stride()
    _need(s[2] == 1, f"{name}: a head's elements have to be dense")
    return RowsC(t.data_ptr(), s[0], s[1])


def _vector(t, name, n, cache):
    _need(t.dtype == torch.float32 and t.device == cache.device and t.is_contiguous() and (t.dim() == 1 if n is None else t.shape == (n,)),
          f"{name}: a dense fp32 vector{'' if n is None else f' of {n}'} on {cache.device} is needed, got {tuple(t.shape)} of {t.dtype} on {t.device}")
    return t.data_ptr()


def _step(cache, batch, q, out):
    """Checks that the step's parts belong together; the rows of q and of the output, which is `out` or a new tensor."""
    _need(batch.device == cache.device, f"the batch is on {batch.device}, the cache on {cache.device}")
    rows = _rows(q, "q", None, cache)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    else:
        _need(out.shape == q.shape, f"out: {tuple(q.shape)} is needed, got {tuple(out.shape)}")
    batch.c.n_tokens = q.shape[0]
    return rows, out, _rows(out, "out", None, cache)


def kv_append(cache, batch, q, k, v, inv_freq=None, interleaved=False, q_norm=None, k_norm=None, eps=1e-6, out=None, stream=None):
    """Stores the step's k and v [tokens][kv_heads][head_dim] in the cache and returns its q [tokens][heads][head_dim], q and k
    normalised per head (fp32 q_norm and k_norm [head_dim], both or neither) and rotated (fp32 inv_freq [rot_dim / 2]; pairs
    i and i + rot_dim / 2, or 2 i and 2 i + 1 where `interleaved`).  Strided q, k and v are read in place.  `out` may be q."""
    if stream is not None:
        with _On(cache.device, stream):
            return kv_append(cache, batch, q, k, v, inv_freq, interleaved, q_norm, k_norm, eps, out)
    qr, out, outr = _step(cache, batch, q, out)
    kr, vr = _rows(k, "k", cache.kv_heads, cache), _rows(v, "v", cache.kv_heads, cache)
    _need(k.shape[0] == q.shape[0] and v.shape[0] == q.shape[0], f"{q.shape[0]} tokens of q, {k.shape[0]} of k, {v.shape[0]} of v")
    rot = 0 if inv_freq is None else 2 * inv_freq.numel()
    with torch.cuda.device(cache.device):
        _check(binding.lib().sna_kv_append(
            cache.c, batch.c, q.shape[1], qr, kr, vr, outr, None if inv_freq is None else _vector(inv_freq, "inv_freq", None, cache), rot, int(interleaved),
            None if q_norm is None else _vector(q_norm, "q_norm", cache.head_dim, cache), None if k_norm is None else _vector(k_norm, "k_norm", cache.head_dim, cache),
            eps, torch.cuda.current_stream(cache.device).cuda_stream))
    return out


def paged_attention(cache, batch, q, scale=None, window=0, out=None, workspace=None, stream=None):
    """Causal attention of the step's q [tokens][heads][head_dim] over the cached keys and values, these tokens' own among them
    (after kv_append).  heads is a multiple of kv_heads.  window: keys that a token sees, its own among them; 0: all.
    workspace: a dense uint8 tensor that is used where it is large enough, instead of one from the allocator."""
    if stream is not None:
        with _On(cache.device, stream):
            return paged_attention(cache, batch, q, scale, window, out, workspace)
    qr, out, outr = _step(cache, batch, q, out)
    need = _check(binding.lib().sna_paged_attention_workspace_bytes(cache.c, batch.c, q.shape[1], window))
    if need and (workspace is None or workspace.numel() < need):
        workspace = torch.empty(need, dtype=torch.uint8, device=cache.device)
    elif need:
        _need(workspace.dtype == torch.uint8 and workspace.device == cache.device and workspace.is_contiguous(), f"workspace: dense uint8 on {cache.device} is needed")
    with torch.cuda.device(cache.device):
        _check(binding.lib().sna_paged_attention(cache.c, batch.c, q.shape[1], qr, outr, cache.head_dim ** -0.5 if scale is None else scale, window,
                                                 workspace.data_ptr() if need else None, need, torch.cuda.current_stream(cache.device).cuda_stream))
    return out


def verify_draft(target, tokens, uniforms, draft_probs=None, n_draft=None, stream=None):
    """Which drafted tokens stand, and the token after them.  target fp32 [n][K + 1][V]: the target's probabilities at every
    drafted place and at the one after the last; tokens [n][K] (int32 or int64); uniforms fp32 [n][K + 1] from [0, 1): one for
    each draft, the last for the draw; draft_probs fp32 [n][K][V] that the drafts were drawn from, or None where they were
    chosen without chance; n_draft int32 [n]: how many of the K each sequence has (all).  Returns (out int32 [n][K + 1],
    accepted int32 [n]): the accepted drafts, the drawn token, -1 behind it."""
    if stream is not None:
        with _On(target.device, stream):
            return verify_draft(target, tokens, uniforms, draft_probs, n_draft)
    _need(target.dim() == 3 and target.dtype == torch.float32 and target.is_cuda and target.stride(2) == 1, "target: fp32 [sequences][drafts + 1][vocabulary], dense rows on a GPU are needed")
    n, K, V = target.shape
    K -= 1
    device = target.device
    _need(K >= 0 and tokens.shape == (n, K) and tokens.dtype in (torch.int32, torch.int64) and tokens.device == device and tokens.is_contiguous(),
          f"tokens: dense int32 or int64 [{n}][{K}] on {device} is needed, got {tuple(tokens.shape)} of {tokens.dtype} on {tokens.device}")
    _need(uniforms.shape == (n, K + 1) and uniforms.dtype == torch.float32 and uniforms.device == device and uniforms.is_contiguous(), f"uniforms: dense fp32 [{n}][{K + 1}] on {device} is needed")
    _need(draft_probs is None or draft_probs.shape == (n, K, V) and draft_probs.dtype == torch.float32 and draft_probs.device == device and draft_probs.stride(2) == 1,
          f"draft_probs: fp32 [{n}][{K}][{V}], dense rows on {device} are needed")
    _need(n_draft is None or n_draft.shape == (n,) and n_draft.dtype == torch.int32 and n_draft.device == device and n_draft.is_contiguous(), f"n_draft: dense int32 [{n}] on {device} is needed")
    out = torch.empty((n, K + 1), dtype=torch.int32, device=device)
    accepted = torch.empty(n, dtype=torch.int32, device=device)
    with torch.cuda.device(device):
        _check(binding.lib().sna_verify_draft(
            target.data_ptr(), target.stride(0), target.stride(1), None if draft_probs is None else draft_probs.data_ptr(),
            0 if draft_probs is None else draft_probs.stride(0), 0 if draft_probs is None else draft_probs.stride(1), tokens.data_ptr(), tokens.element_size(),
            uniforms.data_ptr(), None if n_draft is None else n_draft.data_ptr(), n, K, V, out.data_ptr(), accepted.data_ptr(),
            torch.cuda.current_stream(device).cuda_stream))
    return out, accepted
