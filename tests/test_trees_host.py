"""What the operators of sampling and drafted trees refuse, and the bookkeeping of pages and masks, without a GPU."""
import ctypes as C
import random

import pytest
import torch

import paper_2312_16733_amd as sna
from paper_2312_16733_amd.binding import SamplingC
from test_serving_host import ALIGN, AT, BATCHES, CACHES, NULL, RANGE, append, batch, cache, rows


def tree(c=None, b=None, heads=4, q=None, out=None, masks=AT, words=1, prefix=None, positions=None, scale=0.1, window=0, ws=AT, size=1 << 40):
    return sna.lib().sna_tree_attention(c or cache(), b or batch(), heads, q or rows(), out or rows(), masks, words, prefix, positions, scale, window, ws, size, None)


def test_tree_attention_is_refused():
    for bad, status in CACHES:
        assert tree(c=cache(**bad)) == status, bad
    for bad, status in BATCHES:
        assert tree(b=batch(**bad)) == status, bad
    for heads in (0, 3, -2, 130):
        assert tree(heads=heads) == RANGE
    for bad, status in ((rows(dev=None), NULL), (rows(dev=AT + 2), ALIGN), (rows(token_stride=511), ALIGN), (rows(head_stride=4), ALIGN)):
        assert tree(q=bad) == status and tree(out=bad) == status
    assert tree(out=rows(token_stride=0)) == RANGE
    assert tree(masks=None) == NULL
    for bad in (dict(masks=AT + 4), dict(prefix=AT + 2), dict(positions=AT + 1)):
        assert tree(**bad) == ALIGN, bad
    for bad in (dict(words=0), dict(words=65), dict(words=-1), dict(window=-1), dict(scale=0.0), dict(scale=float("nan")), dict(scale=3e38)):
        assert tree(**bad) == RANGE, bad
    large = dict(n_tokens=300, max_new=129, max_len=200)
    assert tree(b=batch(**large), words=2) == RANGE                                  # the 129th token has no bit
    assert tree(b=batch(**large), words=2, prefix=AT, out=rows(dev=None)) == NULL    # with a prefix the masks may begin anywhere: the next check
    assert tree(b=batch(**large), words=3, out=rows(dev=None)) == NULL
    long = batch(max_len=100000)
    need = sna.lib().sna_tree_attention_workspace_bytes(cache(), long, 4, 1, 0)
    assert need > 0
    for bad in (dict(ws=None), dict(ws=AT + 8), dict(size=need - 1)):
        assert tree(b=long, **bad) == -7, bad
    assert sna.lib().sna_tree_attention_workspace_bytes(cache(), long, 4, 1, 500) == 0
    assert sna.lib().sna_tree_attention_workspace_bytes(cache(), long, 4, 0, 0) == RANGE
    assert tree(b=batch(n_tokens=0)) == 0 and tree(b=batch(n_tokens=0), masks=None) == 0
    assert tree(b=batch(n_seqs=0)) == RANGE


def test_launches_of_trees():
    """What the workspace tells of them: none where a block walks whole rows, the causal form's up to 32 rows a key / value head, parts of
    128 rows for more, from keys on whose sharing pays."""
    bytes_of = lambda n, nodes, length, words=1, window=0: sna.lib().sna_tree_attention_workspace_bytes(  # noqa: E731
        cache(kv_heads=8, k_page_stride=8 * 16 * 64, v_page_stride=8 * 16 * 64), batch(n_seqs=n, n_tokens=n * nodes, max_new=nodes, max_len=length, table_width=length), 32, words, window)
    causal = lambda n, nodes, length: sna.lib().sna_paged_attention_workspace_bytes(  # noqa: E731
        cache(kv_heads=8, k_page_stride=8 * 16 * 64, v_page_stride=8 * 16 * 64), batch(n_seqs=n, n_tokens=n * nodes, max_new=nodes, max_len=length, table_width=length), 32, 0)
    for nodes in (1, 4, 8):
        for length in (100, 5000, 50000):
            assert bytes_of(3, nodes, length) == causal(3, nodes, length)
    assert bytes_of(16, 30, 300) == 0 and bytes_of(1, 60, 300) == 0
    for nodes, planes in ((32, 1), (33, 2), (77, 3), (500, 16), (600, 19)):
        shares = 512 // planes // 8 * 8
        assert bytes_of(4, nodes, 60000, 10) == -(-shares * planes * (16 + 2 * 4 * (min(nodes, 32) * 4 * 66)) // 256) * 256, nodes
    assert bytes_of(1, 2100, 60000, 60) == -(-7 * 66 * (16 + 2 * 4 * (32 * 4 * 66)) // 256) * 256     # fewer shares than there are XCDs
    assert bytes_of(64, 600, 60000, 10) == 0                                         # rows enough to fill the chip
    assert bytes_of(1, 40, 5000) == causal(1, 40, 5000) > 0                          # little to do: blocks of few rows
    assert bytes_of(4, 77, 60000, 2, 100) == 0                                       # few keys in the window


def test_positions_are_refused():
    at = lambda p: sna.lib().sna_kv_append_at(cache(), batch(), 4, rows(), rows(), rows(), rows(), AT, 64, 0, None, None, 1e-6, p, None)  # noqa: E731
    assert at(AT + 2) == ALIGN
    assert append(out=rows(dev=None)) == NULL


def walk(b=None, sampled=AT, sb=4, tokens=AT, tb=4, parents=AT, kept=AT, counts=AT, following=AT):
    return sna.lib().sna_verify_tree(b or batch(), sampled, sb, tokens, tb, parents, kept, counts, following, None)


def test_walks_are_refused():
    for bad in ("sampled", "tokens", "parents", "kept", "counts", "following"):
        assert walk(**{bad: None}) == NULL and walk(**{bad: AT + 2}) == ALIGN, bad
    assert walk(b=batch(starts_dev=None)) == NULL and walk(b=batch(lens_dev=None)) == NULL
    assert walk(tokens=AT + 4, tb=8) == ALIGN and walk(sampled=AT + 4, sb=8) == ALIGN
    for bad in (dict(sb=2), dict(tb=3), dict(b=batch(n_seqs=-1)), dict(b=batch(n_tokens=-1)), dict(b=batch(max_new=4097)), dict(b=batch(max_new=-1)), dict(b=batch(n_seqs=0))):
        assert walk(**bad) == RANGE, bad
    assert walk(b=batch(n_seqs=0, n_tokens=0)) == 0


def test_results_over_what_is_read_are_refused():
    at = lambda i: 0x100000 * (i + 1)  # noqa: E731
    b = dict(n_seqs=3, n_tokens=40, max_new=20, starts_dev=at(0), lens_dev=at(1), page_table_dev=at(2), table_stride=50, table_width=7)
    read = dict(starts=(at(0), 16), lens=(at(1), 12), sampled=(at(3), 8 * 40), tokens=(at(4), 4 * 40), parents=(at(5), 4 * 40))
    results = dict(kept=(at(6), 4 * 60), counts=(at(7), 12), following=(at(8), 12))
    good = dict(sampled=at(3), sb=8, tokens=at(4), parents=at(5), **{k: p for k, (p, _) in results.items()})
    for name, (_, size) in results.items():
        for other, (p, n) in (read | results).items():
            if other != name:
                for over in (p, p + n - 4, p - size + 4):
                    assert walk(b=batch(**b), **(good | {name: over})) == RANGE, (name, other)
    for p, n in (read["starts"], read["lens"], (at(2), 4 * (2 * 50 + 7)), (at(4), 4 * 3 * 5), (at(5), 12)):
        for over in (p, p + n - 4, p - 8):
            assert compact(b=batch(**b), kept=at(4), width=5, counts=at(5), lens=over) == RANGE


def compact(c=None, b=None, kept=AT, width=3, counts=2 * AT, lens=3 * AT):
    return sna.lib().sna_kv_compact(c or cache(), b or batch(), kept, width, counts, lens, None)


def test_compaction_is_refused():
    for bad, status in CACHES:
        assert compact(c=cache(**bad)) == status, bad
    for bad in (dict(starts_dev=None), dict(lens_dev=None), dict(page_table_dev=None)):
        assert compact(b=batch(**bad)) == NULL, bad
    for bad in (dict(n_seqs=-1), dict(table_width=0), dict(table_stride=-1), dict(max_new=-1)):
        assert compact(b=batch(**bad)) == RANGE, bad
    for bad in ("kept", "counts", "lens"):
        assert compact(**{bad: None}) == NULL, bad
        assert compact(**{bad: 5 * AT + 2}) == ALIGN, bad
    assert compact(width=-1) == RANGE
    for over in (dict(lens=AT), dict(lens=2 * AT)):                                  # over starts, lens and kept; over counts
        assert compact(**over) == RANGE, over
    assert compact(b=batch(n_seqs=0)) == 0
    wide = dict(c=cache(kv_heads=4096, k_page_stride=4096 * 16 * 64, v_page_stride=4096 * 16 * 64), b=batch(n_seqs=1 << 20))
    assert compact(**wide, lens=1 << 40) == RANGE and b"more blocks than a launch has" in sna.lib().sna_last_error()


def test_copies_are_refused():
    copy = lambda c=None, s=AT, t=AT, n=3: sna.lib().sna_copy_pages(c or cache(), s, t, n, None)  # noqa: E731
    for bad, status in CACHES:
        assert copy(c=cache(**bad)) == status, bad
    assert copy(s=None) == NULL and copy(t=None) == NULL and copy(s=AT + 2) == ALIGN and copy(t=AT + 1) == ALIGN and copy(n=-1) == RANGE
    assert copy(n=0) == 0 and copy(n=0, s=None) == 0
    assert copy(n=1 << 30) == RANGE and b"more blocks than a launch has" in sna.lib().sna_last_error()


def sampling(**k):
    d = dict(logits_dev=AT, row_stride=1000, n_rows=3, vocab=1000, dtype=0, top_k=0, temperature=1.0, top_p=1.0, min_p=0.0, uniforms_dev=AT)
    return SamplingC(**{**d, **k})


def sample(tokens=AT, probs=None, stride=1000, ws=AT, size=1 << 40, **k):
    return sna.lib().sna_sample_tokens(sampling(**k), tokens, probs, stride, ws, size, None)


def test_sampling_is_refused():
    for bad in (dict(logits_dev=None), dict(uniforms_dev=None), dict(tokens=None)):
        assert sample(**bad) == NULL, bad
    for bad in ("logits_dev", "uniforms_dev", "tokens", "probs", "temperature_dev", "top_p_dev", "min_p_dev", "top_k_dev"):
        assert sample(**{bad: AT + 2}) == ALIGN, bad
    assert sample(dtype=1, logits_dev=AT + 1) == ALIGN
    inf, nan = float("inf"), float("nan")
    for bad in (dict(n_rows=-1), dict(n_rows=(1 << 24) + 1), dict(vocab=0), dict(vocab=(1 << 20) + 1), dict(row_stride=-1), dict(dtype=3), dict(dtype=-1), dict(temperature=-0.1), dict(temperature=inf),
                dict(temperature=nan), dict(top_k=-1), dict(top_p=-0.1), dict(top_p=1.1), dict(top_p=nan), dict(min_p=-0.1), dict(min_p=1.5), dict(min_p=nan), dict(probs=AT, stride=999)):
        assert sample(**bad) == RANGE, bad
        assert sna.lib().sna_last_error()
    assert sna.lib().sna_sample_tokens(None, AT, None, 0, AT, 1 << 40, None) == NULL
    # numbers that a row's own settings stand in for are not looked at
    for name, bad in (("temperature", nan), ("top_p", 7.0), ("min_p", nan), ("top_k", -5)):
        assert sample(**{name: bad, name + "_dev": AT}, tokens=None) == NULL, name
    assert sample(n_rows=0) == 0 and sample(n_rows=0, logits_dev=None) == 0
    need = sna.lib().sna_sample_tokens_workspace_bytes(C.byref(sampling(vocab=200000)))
    assert need >= 0
    if need:
        for bad in (dict(ws=None), dict(ws=AT + 8), dict(size=need - 1)):
            assert sample(vocab=200000, **bad) == -7, bad


def test_calls_are_refused():
    for call, least, most in ((sna.sample_tokens, 2, 10), (sna.tree_attention, 4, 11), (sna.verify_tree, 4, 5), (sna.kv_compact, 4, 5), (sna.copy_pages, 3, 4)):
        with pytest.raises(TypeError):
            call(*[None] * (least - 1))
        with pytest.raises(TypeError):
            call(*[None] * least, nonsense=1)
        with pytest.raises(TypeError):
            call(*[None] * (most + 1))
        with pytest.raises((TypeError, ValueError)):
            call(*[None] * least)
    with pytest.raises(ValueError):
        sna.sample_tokens(torch.zeros(2, 10), torch.zeros(2))                        # not on a GPU


def test_masks_of_a_tree():
    masks, depths = sna.tree_masks([-1, 0, 0, 1, 3, 2])
    assert masks.tolist() == [[1], [3], [5], [11], [27], [37]] and depths == [0, 1, 1, 2, 3, 2]
    masks, depths = sna.tree_masks(list(range(-1, 129)))                             # a chain of 130
    assert masks.shape == (130, 3) and depths == list(range(130))
    for i in range(130):
        assert sum((int(w) % (1 << 64)) << 64 * j for j, w in enumerate(masks[i])) == (1 << (i + 1)) - 1
    assert sna.tree_masks([])[0].shape == (0, 1)
    for bad in ([-1, 1], [-1, 0, -1], [-1, 2, 0]):
        with pytest.raises(ValueError):
            sna.tree_masks(bad)


def test_pages_of_sequences_that_part():
    pool = sna.PagePool(6, 16)
    a = pool.alloc(3)
    b, source, target = pool.fork(a, 40)                                             # two full pages, and 8 slots of the third
    assert b[:2] == a[:2] and source == a[2:] and target == b[2:] and b[2] not in a and pool.n_free == 2
    c, source, target = pool.fork(b, 32)                                             # full ones only
    assert c == a[:2] and source == target == [] and pool.n_free == 2
    pool.free(a)
    assert pool.n_free == 3                                                          # its last page; the others are b's and c's
    pool.free(b)
    assert pool.n_free == 4
    pool.free(c)
    assert pool.n_free == 6
    for bad in (lambda: pool.free(c), lambda: pool.alloc(7), lambda: pool.alloc(-1), lambda: pool.fork([0], 3), lambda: pool.free([99]), lambda: sna.PagePool(0, 16)):
        with pytest.raises(ValueError):
            bad()
    d = pool.alloc(6)
    for bad in (lambda: pool.fork(d, 97), lambda: pool.fork(d, -1), lambda: pool.fork(d, 90), lambda: pool.free([d[0], d[0]])):
        with pytest.raises(ValueError):
            bad()
    assert pool.n_free == 0
    pool.free(d)
    assert sorted(pool.alloc(6)) == list(range(6))


def test_no_page_is_lost_or_given_twice():
    """Sequences at random: every page is free or of those that have it, and what is not shared has one owner."""
    r = random.Random(5)
    pool, live = sna.PagePool(40, 16), []
    for _ in range(3000):
        what = r.random()
        try:
            if what < 0.3:
                live.append(pool.alloc(r.randint(0, 6)))
            elif what < 0.6 and live:
                s = r.choice(live)
                live.append(pool.fork(s, r.randint(0, 16 * len(s)))[0])
            elif what < 0.7 and live:
                r.choice(live).extend(pool.alloc(1))
            elif live:
                pool.free(live.pop(r.randrange(len(live))))
        except ValueError:
            pass
        assert pool.n_free == 40 - len({p for s in live for p in s})


def test_samples_over_what_is_read_are_refused():
    """Tokens and probabilities share no byte with each other, the logits, the random numbers or the settings; rows may lie between rows.
    What passes is refused for its size, behind every other check: no call here is launched."""
    n, V, at = 1 << 22, 1000, lambda i: (i + 1) << 40
    given = dict(n_rows=n, vocab=V, uniforms_dev=at(1), temperature_dev=at(2), top_p_dev=at(3), min_p_dev=at(4), top_k_dev=at(5), tokens=at(6))
    launched = lambda **k: (sample(**k), b"more blocks than a launch has" in sna.lib().sna_last_error())  # noqa: E731
    for dtype, size in ((0, 4), (1, 2), (2, 2)):
        good = dict(given, dtype=dtype, logits_dev=at(0), row_stride=V, probs=at(7), stride=V)
        assert launched(**good) == (RANGE, True)
        read = {"logits_dev": (at(0), n * V * size), **{name: (at(i), 4 * n) for name, i in (("uniforms_dev", 1), ("temperature_dev", 2), ("top_p_dev", 3), ("min_p_dev", 4), ("top_k_dev", 5))}}
        for name, other, mine in (("tokens", "probs", 4 * n), ("probs", "tokens", 4 * n * V)):
            for what, (p, m) in {**read, other: (good[other], 4 * n * V if other == "probs" else 4 * n)}.items():
                for over in (p, p + m - 4, p - mine + 4):
                    assert launched(**dict(good, **{name: over})) == (RANGE, False), (dtype, name, what, over)
                for beside in (p + m, p - mine):
                    assert launched(**dict(good, **{name: beside})) == (RANGE, True), (dtype, name, what, beside)
        # rows of both in one array: logits, then probabilities, and a gap between; one row for all
        step = V * size + 4 * V + 64
        rows = dict(good, row_stride=step // size, stride=step // 4)
        assert launched(**dict(rows, probs=at(0) + V * size)) == (RANGE, True) and launched(**dict(rows, probs=at(0) + step - 4 * V)) == (RANGE, True)
        assert launched(**dict(rows, probs=at(0) + V * size - 4)) == (RANGE, False) and launched(**dict(rows, probs=at(0) + step - 4 * V + 4)) == (RANGE, False)
        assert launched(**dict(rows, probs=at(0) - 5 * step + V * size + 64)) == (RANGE, True)
        assert launched(**dict(rows, stride=step // 4 + 1, probs=at(0) + V * size)) == (RANGE, False)      # further on they meet
        assert launched(**dict(good, row_stride=0, probs=at(0) + V * size)) == (RANGE, True) and launched(**dict(good, row_stride=0, probs=at(0) - 4 * V + 4)) == (RANGE, False)
        assert launched(**dict(rows, tokens=at(0) + V * size + 32)) == (RANGE, False)
    none = dict(given, temperature_dev=None, top_p_dev=None, min_p_dev=None, top_k_dev=None, probs=None, logits_dev=at(0), row_stride=V)
    assert launched(**none) == (RANGE, True)


def test_a_large_batch_of_samples_takes_bounded_memory():
    """A workspace serves calls of any settings and of fewer rows, and does not grow past some thousand rows."""
    need = lambda **k: sna.lib().sna_sample_tokens_workspace_bytes(C.byref(sampling(**k)))  # noqa: E731
    assert 0 < need(n_rows=1, vocab=4097) < 128 << 10 and need(n_rows=100000, vocab=4096) == 0
    for vocab in (4097, 131072, 1 << 20):
        sizes = [need(n_rows=n, vocab=vocab) for n in (1, 7, 128, 4000, 8192, 8193, 65536, 1 << 24)]
        assert sizes == sorted(sizes) and sizes[4] == sizes[-1] < 1 << 30
        for k in (dict(temperature=0.0), dict(top_k=1), dict(top_k=9, top_p=0.5), dict(top_p_dev=AT, dtype=2)):
            assert need(n_rows=128, vocab=vocab, **k) == sizes[2]
