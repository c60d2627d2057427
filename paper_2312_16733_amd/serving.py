"""Autoregressive serving over a paged key / value cache: the operators of include/subnetact.h on torch tensors.

    cache = PagedCache(k_pages, v_pages)                      # one layer's pages
    batch = PagedBatch(starts, lens, page_table, max_new, max_len)
    q = kv_append(cache, batch, q, k, v, inv_freq=inv_freq)   # norms, rotation, k and v into their pages
    out = paged_attention(cache, batch, q)
    tokens, accepted = verify_draft(target, drafted, uniforms)      # speculative decoding: which drafts stand, and the next token

Rows are the new tokens of all sequences of a step, one after the other.  Nothing here reads device memory or waits for it;
`PagedBatch.validate` does, for a caller in doubt about what its arrays hold.  Every call enqueues on the current stream, or on
`stream` (a torch stream or a raw handle), which its outputs and workspace then belong to.  No gradients: these are serving steps.
"""
import torch

from . import binding

binding.lib()                                                          # the library, or the error that says how to build it
try:
    from . import _serving
except ImportError as e:
    raise binding.SnaError(-8, f"the serving binding is not built ({e}): run `python -m paper_2312_16733_amd.build` first") from e

kv_append, paged_attention, verify_draft = _serving.kv_append, _serving.paged_attention, _serving.verify_draft


class PagedCache(_serving.PagedCache):
    """PagedCache(k_pages, v_pages): one layer's pages, keys [pages][kv_heads][page_size][head_dim], values
    [pages][kv_heads][head_dim][page_size], bf16 or fp16, dense within a page; the layers of a pool may take turns (any stride
    between pages).  Borrowed, not copied: pages that are resized or replaced in place (resize_, set_, .data) need a new
    PagedCache, which the calls say."""
    __slots__ = ()


class PagedBatch(_serving.PagedBatch):
    """PagedBatch(starts, lens, page_table, max_new, max_len): the sequences of one step.  starts int32 [n + 1]: sequence b
    brings rows starts[b] .. starts[b + 1] - 1 (none is fine); lens int32 [n]: its cached tokens once these are in; page_table
    int32 [n][width].  max_new and max_len bound the new tokens and the length of any sequence; they choose the launches, so
    bounds near the truth are faster.  Borrowed as the pages are: the arrays' contents may change from call to call, their
    memory and shapes may not."""
    __slots__ = ()

    def validate(self, cache, n_tokens):
        """Reads the arrays back (waits for the GPU) and raises ValueError where they do not fit the cache, each other or the bounds."""
        _validate(self.starts, self.lens, self.page_table, self.max_new, self.max_len, cache.page_size, cache.n_pages, n_tokens)


def _validate(starts, lens, table, max_new, max_len, page_size, n_pages, n_tokens):
    starts, lens, table = (t.cpu().long() for t in (starts, lens, table))
    new = starts[1:] - starts[:-1]
    pages = (lens + page_size - 1) // page_size
    used = torch.arange(table.shape[1])[None] < pages[:, None]
    for ok, text in ((int(starts[0]) == 0 and int(starts[-1]) == n_tokens and bool((new >= 0).all()), f"starts have to rise from 0 to {n_tokens}"),
                     (bool((new <= max_new).all()), f"a sequence brings more than max_new = {max_new} tokens"),
                     (bool((lens >= new).all()), "a sequence is shorter than its new tokens"),
                     (bool((lens <= max_len).all()), f"a sequence is longer than max_len = {max_len}"),
                     (bool((pages <= table.shape[1]).all()), f"a sequence is longer than its {table.shape[1]} table entries"),
                     (bool(((table >= 0) & (table < n_pages))[used].all()), f"a page outside the {n_pages} of the pool")):
        if not ok:
            raise ValueError(text)
