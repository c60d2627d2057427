"""What the serving operators refuse, without a GPU: the C entries check every argument before anything is enqueued."""
import ctypes as C

import pytest
import torch

import paper_2312_16733_amd as sna
from paper_2312_16733_amd import serving
from paper_2312_16733_amd.binding import PagedBatchC, PagedCacheC, RowsC

NULL, RANGE, ALIGN = -1, -3, -4
AT = 1 << 20                                                           # a made-up device address: never read by the host


def cache(**k):
    d = dict(k_pages_dev=AT, v_pages_dev=AT, k_page_stride=2 * 16 * 64, v_page_stride=2 * 16 * 64, n_pages=9, kv_heads=2, page_size=16, head_dim=64, dtype=1)
    return PagedCacheC(**{**d, **k})


def batch(**k):
    d = dict(starts_dev=AT, lens_dev=AT, page_table_dev=AT, table_stride=4, n_seqs=3, n_tokens=5, table_width=4, max_new=3, max_len=60)
    return PagedBatchC(**{**d, **k})


def rows(dev=AT, token_stride=512, head_stride=64):
    return RowsC(dev, token_stride, head_stride)


def attention(c=None, b=None, heads=4, q=None, out=None, scale=0.1, window=0, ws=AT, size=1 << 40):
    return sna.lib().sna_paged_attention(c or cache(), b or batch(), heads, q or rows(), out or rows(), scale, window, ws, size, None)


def append(c=None, b=None, heads=4, q=None, k=None, v=None, out=None, inv=AT, rot=64, qn=None, kn=None):
    return sna.lib().sna_kv_append(c or cache(), b or batch(), heads, q or rows(), k or rows(), v or rows(), out or rows(), inv, rot, 0, qn, kn, 1e-6, None)


CACHES = [(dict(k_pages_dev=None), NULL), (dict(v_pages_dev=None), NULL), (dict(dtype=0), RANGE), (dict(dtype=3), RANGE), (dict(head_dim=96), RANGE),
          (dict(page_size=8), RANGE), (dict(page_size=48), RANGE), (dict(page_size=2048), RANGE), (dict(n_pages=0), RANGE), (dict(kv_heads=0), RANGE),
          (dict(k_page_stride=2 * 16 * 64 - 8), RANGE), (dict(v_page_stride=0), RANGE), (dict(k_pages_dev=AT + 8), ALIGN), (dict(v_page_stride=2 * 16 * 64 + 4), ALIGN)]
BATCHES = [(dict(starts_dev=None), NULL), (dict(lens_dev=None), NULL), (dict(page_table_dev=None), NULL), (dict(n_seqs=-1), RANGE), (dict(n_tokens=-1), RANGE),
           (dict(table_width=0), RANGE), (dict(max_new=0), RANGE), (dict(max_new=6), RANGE), (dict(max_new=1), RANGE), (dict(max_len=2), RANGE), (dict(table_stride=-1), RANGE)]


@pytest.mark.parametrize("call", [append, attention])
def test_caches_and_batches_are_refused(call):
    for bad, status in CACHES:
        assert call(c=cache(**bad)) == status, bad
        assert sna.lib().sna_last_error()
    for bad, status in BATCHES:
        assert call(b=batch(**bad)) == status, bad
    for heads in (0, 3, -2, 130):
        assert call(heads=heads) == RANGE, heads
    assert call(b=batch(n_seqs=1 << 20, n_tokens=1 << 26, max_new=1 << 10, max_len=1 << 10), heads=128) == RANGE      # more blocks than a launch has


def test_rows_are_refused():
    for bad, status in ((rows(dev=None), NULL), (rows(dev=AT + 2), ALIGN), (rows(token_stride=511), ALIGN), (rows(head_stride=4), ALIGN)):
        assert attention(q=bad) == status and attention(out=bad) == status
        for name in ("q", "k", "v", "out"):
            assert append(**{name: bad}) == status, name
    assert attention(window=-1) == RANGE
    for scale in (0.0, -0.1, float("inf"), float("nan")):
        assert attention(scale=scale) == RANGE
    for rot in (-16, 8, 72, 80):
        assert append(rot=rot) == RANGE
    assert append(inv=None) == NULL
    assert append(qn=AT) == NULL and append(kn=AT) == NULL


def test_outputs_that_overlap_themselves_are_refused():
    """Rows of an expanded or windowed output would be written by several blocks."""
    one = dict(n_seqs=1, n_tokens=1, max_new=1)
    for bad in (rows(token_stride=0), rows(head_stride=0), rows(token_stride=248), rows(token_stride=-248), rows(head_stride=56, token_stride=1024),
                rows(token_stride=64, head_stride=64), rows(token_stride=64, head_stride=312), rows(token_stride=56, head_stride=1024), rows(token_stride=1 << 62, head_stride=0)):
        assert attention(out=bad) == RANGE and append(out=bad) == RANGE, bad
    assert attention(b=batch(**one), out=rows(head_stride=0)) == RANGE                               # one token, four heads
    # what does not overlap passes this check and fails at the next one, or at the launch that needs a GPU
    for good in (rows(), rows(token_stride=256), rows(token_stride=-256), rows(token_stride=64, head_stride=320), rows(token_stride=128, head_stride=640),
                 rows(token_stride=768, head_stride=128)):
        assert append(out=good, k=rows(dev=None)) == NULL, good
        assert attention(out=good, b=batch(max_len=100000), ws=None) == -7, good
    assert append(b=batch(**one), out=rows(token_stride=0), k=rows(dev=None)) == NULL


def test_scales_beyond_fp32_are_refused():
    """The kernels take powers of two: scale * log2(e) has to be a number, too."""
    for scale in (3e38, 2.4e38):
        assert attention(scale=scale) == RANGE, scale
    assert attention(scale=2.3e38, b=batch(max_len=100000), ws=None) == -7                          # passes, and fails at the next check


def test_steps_of_more_threads_than_a_launch_has_are_refused():
    c = cache(kv_heads=256, k_page_stride=256 * 16 * 64, v_page_stride=256 * 16 * 64)
    many, wide = dict(n_seqs=1 << 20, max_len=1 << 20), rows(token_stride=256 * 64)
    calls = [lambda: append(c=c, b=batch(**many, n_tokens=1 << 20, max_new=1), heads=256, out=wide), lambda: append(c=c, b=batch(**many, n_tokens=1 << 21, max_new=1 << 20), heads=256, out=wide),
             lambda: attention(c=c, b=batch(**many, n_tokens=1 << 21, max_new=1 << 20), heads=256, out=wide), lambda: verify(n=1 << 22)]
    for call in calls:
        assert call() == RANGE
        assert b"more blocks than a launch has" in sna.lib().sna_last_error()


def test_workspaces_are_refused():
    long = batch(max_len=100000)
    need = sna.lib().sna_paged_attention_workspace_bytes(cache(), long, 4, 0)
    assert need > 0
    for bad in (dict(ws=None), dict(ws=AT + 8), dict(size=need - 1)):
        assert attention(b=long, **bad) == -7, bad
    assert sna.lib().sna_paged_attention_workspace_bytes(cache(), batch(), 4, 0) == 0                # short: no parts
    assert sna.lib().sna_paged_attention_workspace_bytes(cache(), long, 4, 500) == 0
    assert sna.lib().sna_paged_attention_workspace_bytes(cache(dtype=0), long, 4, 0) == RANGE


def test_a_step_without_tokens_is_no_launch():
    for none in (dict(n_seqs=0, n_tokens=0), dict(n_tokens=0)):
        assert append(b=batch(**none)) == 0 and attention(b=batch(**none)) == 0


def test_tokens_without_sequences_are_refused():
    """Rows that belong to nobody would come back as the allocator left them."""
    for b in (batch(n_seqs=0), batch(n_seqs=0, n_tokens=1, max_new=1), batch(n_seqs=0, n_tokens=1, max_new=0, max_len=0)):
        assert append(b=b) == RANGE and attention(b=b) == RANGE
        assert sna.lib().sna_paged_attention_workspace_bytes(cache(), b, 4, 0) == RANGE


def test_tensors_are_refused():
    k, v = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(4, 2, 64, 16, dtype=torch.bfloat16)
    for bad in ((k[0], v), (k, k), (k, v.half()), (k.float(), v.float()), (k, v)):                   # the last: not on a GPU
        with pytest.raises(ValueError):
            sna.PagedCache(*bad)
    n = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        sna.PagedBatch(n, n[:2], torch.zeros(2, 4, dtype=torch.int32), 1, 1)                        # not on a GPU


def test_validate_finds_what_does_not_fit():
    def of(starts, lens, table, n_tokens=5, max_new=4, max_len=64):
        serving._validate(*(torch.tensor(x, dtype=torch.int32) for x in (starts, lens, table)), max_new, max_len, 16, 9, n_tokens)

    good = dict(starts=[0, 1, 1, 5], lens=[17, 0, 33], table=[[0, 8, -1, -1], [-1] * 4, [3, 4, 5, 99]])
    of(**good)
    for bad in (dict(starts=[1, 1, 1, 5]), dict(starts=[0, 2, 1, 5]), dict(starts=[0, 1, 1, 4]), dict(lens=[17, 0, 65]), dict(lens=[17, 0, 3]), dict(lens=[17, 16, 33]),
                dict(table=[[0, 9, -1, -1], [-1] * 4, [3, 4, 5, 99]]), dict(max_new=3), dict(max_len=32), dict(lens=[17, 0, 49])):
        with pytest.raises(ValueError):
            of(**{**good, **bad})
    with pytest.raises(ValueError):
        of([0, 1], [65], [[1, 2, 3, 4]], n_tokens=1, max_len=99)


def test_calls_are_refused():
    for call, args in ((sna.kv_append, 5), (sna.paged_attention, 3), (sna.verify_draft, 3)):
        with pytest.raises(TypeError):
            call(*[None] * (args - 1))
        with pytest.raises(TypeError):
            call(*[None] * args, nonsense=1)
        with pytest.raises(TypeError):
            call(*[None] * 13)
    with pytest.raises(TypeError):
        sna.kv_append(None, None, None, None, None)
    with pytest.raises(TypeError):
        sna.paged_attention(1, 2, 3, cache=1)
    with pytest.raises(ValueError):
        sna.verify_draft(None, None, None)


def verify(target=AT, draft=None, tokens=AT, token_bytes=4, uniforms=AT, counts=None, n=2, k=3, v=100, out=AT, accepted=AT, stride=400):
    return sna.lib().sna_verify_draft(target, stride, 100, draft, stride, 100, tokens, token_bytes, uniforms, counts, n, k, v, out, accepted, None)


def test_verification_is_refused():
    for bad in ("target", "tokens", "uniforms", "out", "accepted"):
        assert verify(**{bad: None}) == NULL, bad
    for bad in ("target", "draft", "tokens", "uniforms", "counts", "out", "accepted"):
        assert verify(**{bad: AT + 2}) == ALIGN, bad
    assert verify(tokens=AT + 4, token_bytes=8) == ALIGN
    for bad in (dict(n=-1), dict(k=-1), dict(v=0), dict(token_bytes=2), dict(stride=-1)):
        assert verify(**bad) == RANGE, bad
    assert verify(n=0) == 0
    t = torch.ones(2, 3, 10)
    with pytest.raises(ValueError):
        sna.verify_draft(t, torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, 3))                # not on a GPU
