"""Attention of trees of drafted tokens, the walk along the ones that stand, and moving and copying of their pages, on the GPU
against their definitions."""
import random

import pytest
import torch

import paged_launches as launches
import paged_reference as ref
import paper_2312_16733_amd as sna
import tree_reference as tree
from test_gpu_serving import parts, within

pytestmark = pytest.mark.gpu

# (slots after the step, new tokens) of every sequence
STEPS = {
    "one token": [(1, 1)],
    "one tree": [(40, 13)],
    "levels": [(300, 4), (16, 3), (17, 2), (5, 5), (64, 4), (65, 1), (129, 6)],
    "some idle": [(40, 0), (33, 5), (8, 0), (64, 0), (200, 20)],
    "two words": [(160, 77), (100, 100), (70, 64), (300, 1), (131, 65)],
    "large": [(700, 333), (50, 30), (611, 200)],
}
HEADS = [(12, 12, 64), (8, 1, 64), (9, 3, 64), (32, 8, 128), (7, 1, 128), (16, 16, 128)]


def attend(s, window=0, **k):
    return sna.tree_attention(*parts(s), s["q"], s["masks"], prefix=s["prefix"], positions=s["positions"], window=window, **k)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("step", STEPS)
@pytest.mark.parametrize("heads,page,window,kind", [(HEADS[0], 16, 0, "tree"), (HEADS[1], 32, 20, "tree"), (HEADS[2], 16, 0, "random"), (HEADS[3], 16, 100, "chain"),
                                                    (HEADS[4], 64, 0, "tree"), (HEADS[3], 128, 0, "random"), (HEADS[5], 16, 1, "tree"), ((64, 1, 128), 32, 0, "empty")])
def test_tree_attention(dtype, step, heads, page, window, kind):
    s = tree.make(STEPS[step], *heads, page, ref.DT[dtype], seed=7, kind=kind)
    want, err = tree.attention(s, window)
    within(attend(s, window), want, err, "out")


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,page,seqs,earlier,window,kind", [
    (HEADS[0], 16, [(300, 4), (12, 3), (77, 1)], 8, 0, "tree"), (HEADS[3], 64, [(200, 16), (90, 9)], 70, 0, "tree"), (HEADS[2], 16, [(90, 2), (300, 5)], 60, 33, "tree"),
    (HEADS[4], 32, [(150, 64), (129, 40)], 64, 0, "random"), (HEADS[1], 16, [(1500, 8), (2500, 8)], 30, 700, "chain"), (HEADS[3], 16, [(5000, 8), (900, 8)], 24, 0, "empty")])
def test_a_part_of_a_tree_behind_others(dtype, heads, page, seqs, earlier, window, kind):
    """Drafting goes level by level: the tree begins before the step's own tokens, and some of it is hidden from each."""
    s = tree.make(seqs, *heads, page, ref.DT[dtype], seed=8, earlier=earlier, kind=kind)
    want, err = tree.attention(s, window)
    within(attend(s, window), want, err, "out")


@pytest.mark.parametrize("heads,page,seqs,window", [
    ((32, 8, 128), 16, [(5000, 13), (30, 3), (9001, 32)], 0), ((32, 8, 128), 64, [(20011, 77)], 0), ((12, 12, 64), 16, [(4097, 8), (1500, 16)], 0),
    ((8, 1, 64), 32, [(30000, 9)], 0), ((32, 8, 128), 16, [(9000, 5), (100, 3), (7777, 2)], 3001), ((8, 2, 128), 64, [(6000, 300), (3000, 1), (50, 50)], 0),
    ((16, 4, 64), 16, [(2500, 200), (4100, 40), (900, 1), (1, 1)], 1000), ((7, 1, 128), 32, [(3001, 256)], 0)])
def test_tree_attention_over_long_caches(heads, page, seqs, window):
    s = tree.make(seqs, *heads, page, torch.bfloat16, seed=9)
    want, err = tree.attention(s, window)
    within(attend(s, window), want, err, "out")


@pytest.mark.parametrize("heads,page,seqs,window,kind", [
    ((32, 1, 128), 16, [(9000, 128)], 0, "tree"), ((32, 1, 64), 64, [(5000, 300), (2100, 17), (300, 300)], 0, "random"), ((28, 4, 128), 16, [(7000, 512)], 2000, "tree"),
    ((32, 1, 128), 16, [(600, 13), (90, 2), (333, 40)], 0, "random"), ((28, 4, 128), 16, [(600, 100)], 0, "empty"), ((8, 1, 64), 32, [(4000, 400)], 0, "chain"),
    ((8, 1, 64), 16, [(500, 500), (40, 7), (0, 0)], 0, "tree"), ((16, 16, 64), 16, [(700, 90), (650, 33)], 100, "random"), ((64, 1, 128), 16, [(20000, 160)], 0, "random")])
def test_many_rows_of_few_heads(heads, page, seqs, window, kind):
    """Planes by the dozen over few shares of the keys, and steps small enough for many tiles of few rows."""
    s = tree.make(seqs, *heads, page, torch.bfloat16, seed=31, kind=kind)
    want, err = tree.attention(s, window)
    within(attend(s, window), want, err, "out")


@pytest.mark.parametrize("i", range(len(launches.STEPS)))
def test_every_launch(i):
    """The steps that get each launch of attention, as trees of random masks over all of a chunk, 4096 tokens at most."""
    launch, _, dim, (heads, kv_heads, length, new, n, ragged, singles, window) = launches.STEPS[i]
    seqs = launches.seqs(length, new, n, ragged, singles)
    s = tree.make(seqs, heads, kv_heads, dim, 16, torch.bfloat16 if i % 2 else torch.float16, seed=20 + i, kind="random", spare=0)
    print(launch, flush=True)
    want, err = tree.attention(s, window)
    within(attend(s, window), want, err, "out")


def test_a_chain_is_causal_attention():
    s = tree.make([(700, 33), (90, 12), (1300, 20)], 16, 4, 128, 16, torch.bfloat16, seed=10, kind="chain")
    want, err = ref.attention(s)
    within(attend(s), want, err, "tree")
    within(sna.paged_attention(*parts(s), s["q"]), want, err, "causal")


def test_scale_strides_layers_and_spare_words():
    s = tree.make([(90, 4), (33, 33), (200, 1)], 8, 2, 128, 16, torch.bfloat16, seed=11, layers=3, words=3)
    want, err = tree.attention(s, scale=0.25)
    out = torch.full((8, s["q"].shape[0], 128), 7.0, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    assert attend(s, scale=0.25, out=out) is out
    within(out, want, err, "out")


def test_bits_behind_the_last_slot_name_nothing():
    """Masks full of ones: what lies behind a sequence's last slot (NaN, or no page at all) is not seen."""
    for seqs, heads in (([(100, 7), (64, 3)], (8, 2, 128)), ([(900, 90), (70, 70)], (16, 4, 64))):
        s = tree.make(seqs, *heads, 16, torch.bfloat16, seed=12, words=5)
        s["masks"].fill_(-1)
        s["bits"] = [torch.ones(n, 5 * 64, dtype=torch.bool) for _, n in seqs]
        want, err = tree.attention(s)
        within(attend(s), want, err, "out")


@pytest.mark.parametrize("heads,seqs", [((8, 2, 128), [(100, 7), (50, 5)]), ((32, 8, 128), [(4000, 90), (200, 60)]), ((12, 12, 64), [(3000, 20)]), ((4, 1, 64), [(40, 1)])])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_values_that_are_no_numbers_reach_only_those_that_see_them(heads, seqs, bad):
    s = tree.make(seqs, *heads, 16, torch.bfloat16, seed=13, kind="random")
    want, err = tree.attention(s)
    hit = torch.zeros(s["q"].shape[0], dtype=torch.bool, device="cuda")
    row = 0
    for b, (l, n) in enumerate(seqs):
        slot = l - n + n // 2
        page = int(s["table"][b, slot // 16])
        s["v_pages"][page, :, :, slot % 16] = bad
        s["k_pages"][page, :, slot % 16] = bad if b == 0 else s["k_pages"][page, :, slot % 16]
        hit[row: row + n] = tree.seen_of(s, b)[:, slot]
        row += n
    out = attend(s)
    assert not hit.all()
    within(out[~hit], want[~hit], err[~hit], "the others")
    if hit.any():
        assert not torch.isfinite(out[hit].float()).any()


@pytest.mark.parametrize("heads,seqs", [((8, 2, 128), [(100, 5), (60, 3)]), ((8, 2, 128), [(900, 90), (500, 1)]), ((32, 8, 128), [(4000, 70), (3000, 64)]), ((4, 4, 64), [(400, 60), (90, 9)])])
def test_arrays_that_do_not_fit(heads, seqs):
    """Pages that are none, lengths beyond the table, prefixes and positions of any value, masks full of ones: whatever comes back for
    those sequences, the last is right."""
    s = tree.make(seqs * 2 + [(70, 1), (200, 40)], *heads, 16, torch.bfloat16, seed=30, earlier=0)
    want, err = tree.attention(s)
    n = s["seqs"][-1][1]
    prefix = torch.tensor(s["base"], dtype=torch.int32, device="cuda")
    prefix[:4] = torch.tensor([-5, 2 ** 31 - 1, -2 ** 31, 17], dtype=torch.int32)
    s["positions"][:3] = torch.tensor([2 ** 31 - 1, -2 ** 31, -1], dtype=torch.int32)
    s["masks"][: -n] = -1
    s["table"][0, 1], s["table"][0, 2] = -5, 2 ** 31 - 1
    s["lens"][1], s["lens"][2], s["lens"][4] = 10 ** 9, -7, 0
    s["prefix"] = prefix
    for window in (0, 300):
        out = attend(s, window)
        torch.cuda.synchronize()
        within(out[-n:], want[-n:], err[-n:], "the last sequence")


def test_positions_of_the_tree():
    """kv_append rotates by the positions it is given and stores by slots."""
    s = tree.make([(40, 13), (100003, 7), (9, 0)], 9, 3, 64, 16, torch.float16, seed=14, junk=False)
    inv = (10000.0 ** (-torch.arange(0, 64, 2).double() / 64)).float().cuda()
    D, half = 64, 32
    a = s["positions"].double()[:, None, None] * inv.double()
    got = sna.kv_append(*parts(s), s["q"], s["k"], s["v"], inv_freq=inv, positions=s["positions"])
    where = [(b, l - n + i) for b, (l, n) in enumerate(s["seqs"]) for i in range(n)]
    stored = torch.stack([s["k_pages"][int(s["table"][b, p // 16]), :, p % 16] for b, p in where])
    for x, y, name in ((s["q"], got, "q"), (s["k"], stored, "k")):
        u, v = x[..., :half].double(), x[..., half:].double()
        want = torch.cat((u * a.cos() - v * a.sin(), u * a.sin() + v * a.cos()), -1)
        size = torch.cat((u.abs() + v.abs(),) * 2, -1)
        within(y, want, want.abs() * 2.0 ** -11 + size * (160 * 2.0 ** -24) + 2.0 ** -25, name)
    values = torch.stack([s["v_pages"][int(s["table"][b, p // 16]), :, :, p % 16] for b, p in where])
    assert torch.equal(values, s["v"])


# ---------------------------------------------------------------- the walk
def walked(sizes, max_new, sampled, tokens, parents):
    kept, counts, following, at = [], [], [], 0
    for n in sizes:
        s, t, p = (x[at: at + n] for x in (sampled, tokens, parents))
        path = [0] if n else []
        while path:
            c = path[-1]
            step = next((j for j in range(c + 1, n) if p[j] == c and s[c] >= 0 and t[j] == s[c]), None)
            if step is None:
                break
            path.append(step)
        kept.append(path + [-1] * (max_new - len(path)))
        counts.append(len(path))
        following.append(s[path[-1]] if path else -1)
        at += n
    return kept, counts, following


def batch_of(sizes, max_new=None):
    n = len(sizes)
    return sna.PagedBatch(torch.tensor([0] + sizes).cumsum(0).int().cuda(), torch.tensor(sizes, dtype=torch.int32).cuda(), torch.zeros(n, 1, dtype=torch.int32).cuda(), max_new or max(sizes), max(sizes))


@pytest.mark.parametrize("sizes", [[1], [13], [2, 1, 5], [0, 7, 0, 64], [65, 64, 3], [200, 77, 1], [4096, 5], [30] * 300])
@pytest.mark.parametrize("long", [False, True])
def test_walk(sizes, long):
    r = random.Random(len(sizes) * 1000 + sizes[0])
    tokens, sampled, parents = [], [], []
    for n in sizes:
        p = tree.parents(n, r.random()) if n else []
        t = [r.randrange(6) for _ in range(n)]                         # siblings with one token among them
        parents += p
        tokens += t
        children = {}
        for j in range(1, n):
            children.setdefault(p[j], []).append(j)
        sampled += [t[r.choice(children[i])] if i in children and r.random() < 0.9 else r.randrange(-1, 6) for i in range(n)]
    want = walked(sizes, max(sizes) + 3, sampled, tokens, parents)
    as_ints = lambda x: torch.tensor(x, dtype=torch.int64 if long else torch.int32).cuda()  # noqa: E731
    got = sna.verify_tree(batch_of(sizes, min(max(sizes) + 3, 4096)), torch.tensor(sampled, dtype=torch.int32).cuda(), as_ints(tokens), torch.tensor(parents, dtype=torch.int32).cuda())
    width = min(max(sizes) + 3, 4096)
    assert got[0].tolist() == [k[:width] for k in want[0]] and got[1].tolist() == want[1] and got[2].tolist() == want[2]


def test_walk_of_the_unusual():
    """A chain of 4096 that stands whole; parents that are none; a drafted -1 beside a sampled one; ids past 2^31."""
    n = 4096
    t = torch.arange(n) % 50257
    p = torch.arange(n, dtype=torch.int32) - 1
    kept, counts, following = sna.verify_tree(batch_of([n]), torch.roll(t, -1).cuda(), t.cuda(), p.cuda())
    assert kept[0].tolist() == list(range(n)) and counts.tolist() == [n] and following.tolist() == [0]
    sampled, tokens, parents = [5, 5, 5, -1, 9], [0, 5, 5, 5, -1], [7, 1, 2 ** 31 - 1, 0, 3]
    got = sna.verify_tree(batch_of([5]), *(torch.tensor(x, dtype=torch.int32).cuda() for x in (sampled, tokens, parents)))
    assert [x.tolist() for x in got] == [[[0, 3, -1, -1, -1]], [2], [-1]]
    big = 1 << 40
    got = sna.verify_tree(batch_of([2]), torch.tensor([big, 3]).cuda(), torch.tensor([0, big]).cuda(), torch.tensor([-1, 0], dtype=torch.int32).cuda())
    assert got[0].tolist() == [[0, 1]] and got[2].tolist() == [3]


# ---------------------------------------------------------------- moving and copying
def compacted(s, kept, counts):
    """The pools that come of it, and the lengths; everything by single slots."""
    k, v, page = s["k_pages"].clone(), s["v_pages"].clone(), s["page"]
    lens = []
    for b, (l, n) in enumerate(s["seqs"]):
        base = l - n
        at = lambda p: (int(s["table"][b, p // page]), p % page)  # noqa: E731
        for i in range(counts[b]):
            (p0, i0), (p1, i1) = at(base + kept[b][i]), at(base + i)
            k[p1, :, i1] = s["k_pages"][p0, :, i0]
            v[p1, :, :, i1] = s["v_pages"][p0, :, :, i0]
        lens.append(base + counts[b])
    return k, v, lens


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("seqs", [[(13, 13)], [(40, 13), (33, 1), (9, 0), (200, 64)], [(700, 300), (64, 17), (16, 16), (17, 16)]])
@pytest.mark.parametrize("kv_heads,dim,page", [(1, 64, 16), (3, 64, 32), (24, 128, 16), (8, 128, 64), (2, 64, 128), (100, 64, 16)])
def test_compaction(dtype, seqs, kv_heads, dim, page):
    s = ref.make(seqs, kv_heads, kv_heads, dim, page, ref.DT[dtype], seed=15, layers=2)
    r = random.Random(page + kv_heads)
    kept, counts = [], []
    for _, n in seqs:
        c = r.randint(0, n)
        kept.append(sorted(r.sample(range(n), c)))
        counts.append(c)
    width = max(max(counts), 1) + 1
    k, v, lens = compacted(s, kept, counts)
    got = sna.kv_compact(*parts(s), torch.tensor([x + [-1] * (width - len(x)) for x in kept], dtype=torch.int32).cuda(), torch.tensor(counts, dtype=torch.int32).cuda())
    assert got.tolist() == lens
    assert same_bits(s["k_pages"], k) and same_bits(s["v_pages"], v)


def test_compaction_of_what_does_not_fit():
    """Numbers that do not rise or are no token's, counts that are too large, pages that are none: nothing else changes."""
    seqs = [(40, 10), (50, 10), (60, 10), (30, 8)]
    s = ref.make(seqs, 2, 2, 64, 16, torch.bfloat16, seed=16)
    kept = torch.tensor([[0, 4, 2 ** 31 - 1, -2 ** 31, 9], [0, 2, 3, 5, 9], [1, 3, 4, 12, 99], [2, 3, 5, 7, 0]], dtype=torch.int32).cuda()
    counts = torch.tensor([5, 2 ** 31 - 1, -4, 4], dtype=torch.int32).cuda()
    s["table"][1, 3] = s["n_pages"]                                    # slots 48 and 49 of the second sequence
    k, v, page = s["k_pages"].clone(), s["v_pages"].clone(), 16
    for b, moves in ((0, [(4, 1), (9, 4)]), (1, [(2, 1), (3, 2), (5, 3)]), (3, [(2, 0), (3, 1), (5, 2), (7, 3)])):
        base = seqs[b][0] - seqs[b][1]
        for j, i in moves:
            (p0, i0), (p1, i1) = ((int(s["table"][b, (base + x) // page]), (base + x) % page) for x in (j, i))
            k[p1, :, i1], v[p1, :, :, i1] = s["k_pages"][p0, :, i0], s["v_pages"][p0, :, :, i0]
    got = sna.kv_compact(*parts(s), kept, counts)
    assert got.tolist() == [35, 45, 50, 26]
    assert same_bits(s["k_pages"], k) and same_bits(s["v_pages"], v)


def test_compaction_of_lengths_below_the_step():
    """A sequence shorter than its new tokens: slots below 0 are nobody's."""
    s = ref.make([(20, 20), (40, 5)], 2, 2, 64, 16, torch.bfloat16, seed=17)
    s["lens"][0] = 15                                                  # its step begins at slot -5
    k, v = s["k_pages"].clone(), s["v_pages"].clone()
    at = lambda p: (int(s["table"][0, p // 16]), p % 16)  # noqa: E731
    for j, i in ((6, 5), (9, 7)):                                      # places 0 and 3, 2 and 4 of slots: 6 - 5 -> 5 - 5, 9 - 5 -> 7 - 5
        (p0, i0), (p1, i1) = at(j - 5), at(i - 5)
        k[p1, :, i1], v[p1, :, :, i1] = s["k_pages"][p0, :, i0], s["v_pages"][p0, :, :, i0]
    kept = torch.tensor([[0, 1, 2, 3, 4, 6, 6, 9], [0, 1, 2, 3, 4, -1, -1, -1]], dtype=torch.int32).cuda()
    got = sna.kv_compact(*parts(s), kept, torch.tensor([8, 5], dtype=torch.int32).cuda())
    # place 6 stays where it is, and is read for place 5 before
    assert got.tolist() == [3, 40] and same_bits(s["k_pages"], k) and same_bits(s["v_pages"], v)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("kv_heads,dim,page,n", [(1, 64, 16, 1), (3, 64, 32, 7), (24, 128, 16, 20), (8, 128, 1024, 3), (5, 64, 128, 200)])
def test_copies(dtype, kv_heads, dim, page, n):
    """Other layers of the pool stay; pairs outside the pool are left out; several targets of one source."""
    g = torch.Generator().manual_seed(n)
    pool = 2 * n + 2
    k = torch.randn(pool, 3, kv_heads, page, dim, generator=g).to(ref.DT[dtype]).cuda()
    v = torch.randn(pool, 3, kv_heads, dim, page, generator=g).to(ref.DT[dtype]).cuda()
    order = torch.randperm(pool, generator=g).int()
    source, target = order[torch.randint(0, (n + 2) // 3, (n,), generator=g)], order[n: 2 * n].clone()
    wk, wv = k.clone(), v.clone()
    for a, b in zip(source.tolist(), target.tolist()):
        wk[b, 1], wv[b, 1] = k[a, 1], v[a, 1]
    bad = torch.tensor([-1, pool, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    source, target = torch.cat((source, bad, order[:4].clone())), torch.cat((target, order[-1:].repeat(4), bad))
    cache = sna.PagedCache(k[:, 1], v[:, 1])
    assert sna.copy_pages(cache, source.cuda(), target.cuda()) is None
    assert same_bits(k, wk) and same_bits(v, wv)
    sna.copy_pages(cache, source[:0].cuda(), target[:0].cuda())
    assert same_bits(k, wk) and same_bits(v, wv)


def test_pages_past_32_bit_offsets():
    """Copies and moves beyond 4 GiB of the pool."""
    page, H, D = 64, 8, 128
    n = (5 << 30) // (H * page * D * 2)
    k = torch.zeros(n, H, page, D, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros(n, H, D, page, dtype=torch.bfloat16, device="cuda")
    k[n - 1], v[n - 1] = torch.randn_like(k[0]), torch.randn_like(v[0])
    cache = sna.PagedCache(k, v)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    sna.copy_pages(cache, ints(n - 1), ints(n - 3))
    assert torch.equal(k[n - 3], k[n - 1]) and torch.equal(v[n - 3], v[n - 1]) and int((k[n - 2] != 0).sum()) == 0
    batch = sna.PagedBatch(ints(0, 9), ints(9), ints(n - 3)[None], 9, 9)
    assert sna.kv_compact(cache, batch, ints(0, 3, 8)[None], ints(3)).tolist() == [3]
    assert torch.equal(k[n - 3, :, 1:3], k[n - 1, :, [3, 8]]) and torch.equal(v[n - 3, :, :, 1:3], v[n - 1, :, :, [3, 8]])


# ---------------------------------------------------------------- together
def test_a_round_in_a_graph():
    """Append, attention, sampling, the walk and the moves of one round, captured once and replayed next to eager rounds from the same
    state: the same tokens, lengths and pages, bit for bit."""
    n, nodes, H, K, D, V = 3, 13, 8, 2, 64, 1000
    p = tree.parents(nodes, 3)
    masks, depths = sna.tree_masks(p)
    s = ref.make([(40 + 20 * b, nodes) for b in range(n)], H, K, D, 16, torch.bfloat16, seed=18, fill=0.0, junk=False)
    g = torch.Generator().manual_seed(4)
    head = (torch.randn(V, H * D, generator=g) * 0.3).to("cuda", torch.bfloat16)
    inv = (10000.0 ** (-torch.arange(0, 64, 2).double() / 64)).float().cuda()
    masks, depth, par = masks.repeat(n, 1).cuda(), torch.tensor(depths * n, dtype=torch.int32).cuda(), torch.tensor(p * n, dtype=torch.int32).cuda()
    tokens = torch.randint(0, V, (n * nodes,), generator=g).cuda()
    u = torch.rand(n * nodes, generator=g).cuda()
    rows = torch.arange(n * nodes, device="cuda") // nodes
    cache, batch = parts(s)

    def step():
        positions = (s["lens"] - nodes)[rows] + depth
        q = sna.kv_append(cache, batch, s["q"], s["k"], s["v"], inv_freq=inv, positions=positions)
        x = sna.tree_attention(cache, batch, q, masks, positions=positions)
        drawn = sna.sample_tokens(x.flatten(1) @ head.t(), u, temperature=0.7, top_k=40, top_p=0.9)
        t = torch.where(torch.arange(n * nodes, device="cuda") % 2 == 0, drawn[(rows * nodes + par.clamp(min=0))].long(), tokens)      # half of them as drawn
        kept, counts, following = sna.verify_tree(batch, drawn, t, par)
        return drawn, kept, counts, following, sna.kv_compact(cache, batch, kept, counts)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    k0, v0 = s["k_pages"].clone(), s["v_pages"].clone()
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    stood = 0
    for i in range(4):
        u.copy_(torch.rand(n * nodes, generator=g))
        s["k_pages"].copy_(k0)
        s["v_pages"].copy_(v0)
        eager = [x.clone() for x in step()]
        k1, v1 = s["k_pages"].clone(), s["v_pages"].clone()
        s["k_pages"].copy_(k0)
        s["v_pages"].copy_(v0)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, eager):
            assert torch.equal(a, b)
        assert same_bits(s["k_pages"], k1) and same_bits(s["v_pages"], v1)
        assert eager[4].tolist() == [l - nodes + c for (l, _), c in zip(s["seqs"], eager[2].tolist())]
        stood += int(eager[2].sum()) - n
    assert stood > 0


def test_calls_on_another_stream():
    s = tree.make([(700, 13), (90, 12)], 16, 4, 128, 16, torch.bfloat16, seed=19)
    want, zeros = attend(s), torch.zeros(25, dtype=torch.int32, device="cuda")
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    got = attend(s, stream=other)
    kept, counts, following = sna.verify_tree(parts(s)[1], zeros, zeros, zeros, stream=other.cuda_stream)
    torch.cuda.current_stream().wait_stream(other)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and counts.tolist() == [2, 2]        # the root, and of its children the first


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("seqs", [[(1, 1)], [(300, 1), (16, 1), (17, 1), (129, 1)], [(40, 0), (33, 1), (0, 0), (200, 1)], [(83, 83), (150, 37), (64, 64), (9, 1)], [(40, 13), (1000, 4), (21, 21)]])
@pytest.mark.parametrize("heads,page,rot,interleaved,norm", [
    ((12, 12, 64), 16, 64, False, False), ((9, 3, 64), 32, 32, True, True), ((32, 8, 128), 16, 128, True, False), ((7, 1, 128), 64, 48, False, True), ((40, 8, 128), 16, 64, True, True)])
def test_positions_of_any_number(dtype, seqs, heads, page, rot, interleaved, norm):
    """Every form of the append, single tokens a sequence among them, by positions that are no slots': rotation goes by them, the place
    in the cache by the slot."""
    s = ref.make(seqs, *heads, page, ref.DT[dtype], seed=19, layers=2)
    g = torch.Generator().manual_seed(6)
    T = s["q"].shape[0]
    positions = torch.randint(0, 200, (T,), generator=g, dtype=torch.int32)
    positions[::5] = torch.randint(0, 1 << 17, (len(positions[::5]),), generator=g, dtype=torch.int32)
    positions[3::7] = -3
    inv = (10000.0 ** (-torch.arange(0, rot, 2).double() / rot)).float().cuda()
    w = [torch.rand(heads[2], generator=g).cuda() + 0.5 if norm else None for _ in range(2)]
    (wq, eq), (wk, ek), wv = ref.append(dict(s, seqs=[(p + 1, 1) for p in positions.tolist()]), inv, interleaved, *w, eps=1e-5)
    old_k, old_v = s["k_pages"].clone(), s["v_pages"].clone()
    got = sna.kv_append(*parts(s), s["q"], s["k"], s["v"], inv_freq=inv, interleaved=interleaved, q_norm=w[0], k_norm=w[1], eps=1e-5, positions=positions.cuda())
    within(got, wq, eq, "q")
    where = [(b, l - n + i) for b, (l, n) in enumerate(seqs) for i in range(n)]
    pages, slots = torch.tensor([int(s["table"][b, p // page]) for b, p in where], device="cuda"), torch.tensor([p % page for _, p in where], device="cuda")
    within(s["k_pages"][pages, :, slots], wk, ek, "k")
    assert torch.equal(s["v_pages"][pages, :, :, slots], wv)
    old_k[pages, :, slots], old_v[pages, :, :, slots] = s["k_pages"][pages, :, slots], s["v_pages"][pages, :, :, slots]
    assert same_bits(old_k, s["k_pages"]) and same_bits(old_v, s["v_pages"])
