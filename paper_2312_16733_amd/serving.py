"""Autoregressive serving over a paged key / value cache: the operators of include/subnetact.h on torch tensors.

    cache = PagedCache(k_pages, v_pages)                      # one layer's pages
    batch = PagedBatch(starts, lens, page_table, max_new, max_len)
    q = kv_append(cache, batch, q, k, v, inv_freq=inv_freq)   # norms, rotation, k and v into their pages
    out = paged_attention(cache, batch, q)
    tokens, accepted = verify_draft(target, drafted, uniforms)      # speculative decoding: which drafts stand, and the next token
    tokens = sample_tokens(logits, uniforms, temperature=0.8, top_p=0.9)

Trees of drafted tokens take the place of chains: several tokens for the same place, of which at most one will stand.

    masks, depths = tree_masks(parents)                       # of the tree's shape, once
    q = kv_append(cache, batch, q, k, v, inv_freq=inv_freq, positions=positions)         # first slot of the tree + depth
    out = tree_attention(cache, batch, q, masks)
    kept, counts, token = verify_tree(batch, sample_tokens(logits, uniforms), tokens, parents)
    lens = kv_compact(cache, batch, kept, counts)             # what stands moves up, the rest is forgotten

Pages are a PagePool's to give; sequences that part share the full ones, and copy_pages copies the last.

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
sample_tokens, tree_attention, verify_tree = _serving.sample_tokens, _serving.tree_attention, _serving.verify_tree
kv_compact, copy_pages = _serving.kv_compact, _serving.copy_pages


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


def tree_masks(parents):
    """Masks for tree_attention (int64 [tokens][words], on the CPU) and depths of one tree (a list), from the parents of its tokens: the first
    is the root, whose parent is not looked at; the others' come before them."""
    seen, depths = [], []
    for i, p in enumerate(parents):
        if i and not 0 <= p < i:
            raise ValueError(f"the parent of token {i} is {p}: it has to come before it")
        seen.append(1 << i | (seen[p] if i else 0))
        depths.append(depths[p] + 1 if i else 0)
    words = max(1, -(-len(seen) // 64))
    signed = lambda m: m - (1 << 64) if m >> 63 else m  # noqa: E731
    return torch.tensor([[signed(m >> 64 * w & (1 << 64) - 1) for w in range(words)] for m in seen], dtype=torch.int64).view(len(seen), words), depths


class PagePool:
    """PagePool(n_pages, page_size): which pages of a cache are whose, on the host.  A page may be several sequences'; it is free again
    when the last of them frees it.  Pages are lists of numbers, as they go into a page table."""

    def __init__(self, n_pages, page_size):
        if n_pages < 1 or page_size < 1:
            raise ValueError(f"{n_pages} pages of {page_size} slots")
        self.page_size = page_size
        self._owners = [0] * n_pages
        self._free = list(range(n_pages - 1, -1, -1))

    @property
    def n_free(self):
        return len(self._free)

    def alloc(self, n):
        """n pages that are nobody's; ValueError where there are not as many, and none is taken."""
        if not 0 <= n <= len(self._free):
            raise ValueError(f"{n} pages are wanted, {len(self._free)} are free")
        pages = [self._free.pop() for _ in range(n)]
        for p in pages:
            self._owners[p] = 1
        return pages

    def fork(self, pages, length):
        """A second sequence with the first `length` slots of one that has these pages: (its pages, source, target).  It shares the pages
        that are full; one that is not is copied, from source to target (lists of one page or none, for copy_pages), so that both
        may go on.  What else the first one has stays its own."""
        full, rest = divmod(length, self.page_size)
        if length < 0 or full + (rest > 0) > len(pages):
            raise ValueError(f"{length} slots are more than {len(pages)} pages of {self.page_size}")
        self._check(pages)
        target = self.alloc(1) if rest else []
        for p in pages[:full]:
            self._owners[p] += 1
        return pages[:full] + target, pages[full: full + len(target)], target

    def free(self, pages):
        """Gives back what a sequence has of these pages."""
        self._check(pages)
        for p in pages:
            self._owners[p] -= 1
            if self._owners[p] == 0:
                self._free.append(p)

    def _check(self, pages):
        for p in pages:
            if not 0 <= p < len(self._owners) or self._owners[p] < 1:
                raise ValueError(f"page {p} is nobody's")
        if len(set(pages)) != len(pages):
            raise ValueError("a page is named twice")


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
