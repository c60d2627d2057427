"""Autoregressive serving operators on the GPU against their definitions in 64 bits."""
import pytest
import torch

import paper_2312_16733_amd as sna
import paged_launches as launches
import paged_reference as ref

pytestmark = pytest.mark.gpu


def parts(s):
    cache = sna.PagedCache(s["k_pages"], s["v_pages"])
    batch = sna.PagedBatch(s["starts"], s["lens"], s["table"], s["max_new"], s["max_len"])
    return cache, batch


def within(got, want, err, what):
    assert torch.isfinite(got.float()).all(), f"{what}: not finite"
    off = (got.double() - want).abs()
    worst = (off / err).nan_to_num(nan=0.0).max().item()               # an exact zero has no error allowed, and is 0 / 0
    print(f"{what}: {worst:.3f} of the bound", flush=True)
    assert (off <= err).all(), f"{what}: {worst} of the bound"


# (length, new tokens) of every sequence
STEPS = {
    "one token": [(1, 1)],
    "decode": [(300, 1), (16, 1), (17, 1), (1, 1), (64, 1), (65, 1), (129, 1)],
    "some idle": [(40, 0), (33, 1), (0, 0), (64, 0), (200, 1)],
    "drafts": [(77, 5), (5, 5), (130, 4), (64, 1), (100, 0), (16, 2)],
    "chunks": [(83, 83), (150, 37), (64, 64), (301, 17), (9, 1)],
    "long chunk": [(700, 333), (50, 1), (611, 20)],
}
HEADS = [(12, 12, 64), (8, 1, 64), (9, 3, 64), (32, 8, 128), (7, 1, 128), (16, 16, 128)]


# ---------------------------------------------------------------- append
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("step", STEPS)
@pytest.mark.parametrize("heads,page,rot,interleaved,norm", [
    ((12, 12, 64), 16, 64, False, False), ((9, 3, 64), 32, 32, True, True), ((32, 8, 128), 16, 128, True, False),
    ((7, 1, 128), 64, 48, False, True), ((40, 8, 128), 16, 64, False, True), ((8, 1, 64), 128, 0, False, True)])
def test_append(dtype, step, heads, page, rot, interleaved, norm):
    s = ref.make(STEPS[step], *heads, page, ref.DT[dtype], seed=3, layers=2)
    g = torch.Generator().manual_seed(5)
    D = heads[2]
    inv = (10000.0 ** (-torch.arange(0, rot, 2).double() / rot)).float().cuda() if rot else None
    w = [torch.rand(D, generator=g).cuda() + 0.5 if norm else None for _ in range(2)]
    (wq, eq), (wk, ek), wv = ref.append(s, inv, interleaved, *w, eps=1e-5)
    old_k, old_v = s["k_pages"].clone(), s["v_pages"].clone()
    cache, batch = parts(s)
    batch.validate(cache, s["q"].shape[0])
    q = sna.kv_append(cache, batch, s["q"], s["k"], s["v"], inv_freq=inv, interleaved=interleaved, q_norm=w[0], k_norm=w[1], eps=1e-5)
    within(q, wq, eq, "q")
    row, touched_k, touched_v = 0, torch.zeros_like(old_k, dtype=torch.bool), torch.zeros_like(old_v, dtype=torch.bool)
    for b, (l, n) in enumerate(s["seqs"]):
        pos = torch.arange(l - n, l, device="cuda")
        page_of, slot = s["table"][b, pos // page].long(), pos % page
        if n:
            within(s["k_pages"][page_of, :, slot], wk[row: row + n], ek[row: row + n], f"k of sequence {b}")
            assert torch.equal(s["v_pages"][page_of, :, :, slot], wv[row: row + n])
            touched_k[page_of, :, slot] = True
            touched_v[page_of, :, :, slot] = True
        row += n
    # nothing else in the pool has changed, bit for bit
    for new, old, touched in ((s["k_pages"], old_k, touched_k), (s["v_pages"], old_v, touched_v)):
        assert torch.equal(new.view(torch.int16)[~touched], old.view(torch.int16)[~touched])


def test_append_far_positions_and_in_place():
    """Angles of positions past 10^5, where a 32-bit product would be off by 1e-2 radians; q written over itself."""
    s = ref.make([(131071, 1), (131072, 3), (100003, 2)], 16, 2, 128, 64, torch.float16, seed=4, junk=False)
    inv = (10000.0 ** (-torch.arange(0, 128, 2).double() / 128)).float().cuda()
    (wq, eq), (wk, ek), _ = ref.append(s, inv)
    cache, batch = parts(s)
    q = sna.kv_append(cache, batch, s["q"], s["k"], s["v"], inv_freq=inv, out=s["q"])
    assert q is s["q"]
    within(q, wq, eq, "q")
    within(s["k_pages"][s["table"][1, 131071 // 64].long(), :, 131071 % 64], wk[3], ek[3], "k")


def test_append_without_a_page():
    """Tokens whose page is none of the pool's, or behind the table, leave the pool as it is; q is returned all the same."""
    s = ref.make([(40, 20), (33, 1), (50, 3)], 4, 2, 64, 16, torch.bfloat16, seed=6)
    s["table"][0, 1:3] = torch.tensor([-1, 2 ** 31 - 1], dtype=torch.int32)
    s["table"][1, 2] = s["n_pages"]
    s["lens"][2] = 10 ** 9
    old = s["k_pages"].clone(), s["v_pages"].clone()
    cache, batch = parts(s)
    q = sna.kv_append(cache, batch, s["q"], s["k"], s["v"])
    torch.cuda.synchronize()
    assert torch.equal(q, s["q"])
    assert torch.equal(s["k_pages"].view(torch.int16), old[0].view(torch.int16)) and torch.equal(s["v_pages"].view(torch.int16), old[1].view(torch.int16))


# ---------------------------------------------------------------- attention
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("step", STEPS)
@pytest.mark.parametrize("heads,page,window", [(HEADS[0], 16, 0), (HEADS[1], 32, 20), (HEADS[2], 16, 0), (HEADS[3], 16, 100), (HEADS[4], 64, 0),
                                               (HEADS[3], 128, 0), (HEADS[5], 16, 1), ((64, 1, 128), 32, 0)])
def test_attention(dtype, step, heads, page, window):
    s = ref.make(STEPS[step], *heads, page, ref.DT[dtype], seed=7)
    cache, batch = parts(s)
    want, err = ref.attention(s, window)
    within(sna.paged_attention(cache, batch, s["q"], window=window), want, err, "out")


@pytest.mark.parametrize("heads,page,seqs,window", [
    ((32, 8, 128), 16, [(5000, 1), (3, 1), (9001, 1)], 0), ((32, 8, 128), 64, [(20011, 1)], 0), ((12, 12, 64), 16, [(4097, 1), (1500, 1)], 0),
    ((8, 1, 64), 32, [(30000, 9)], 0), ((32, 8, 128), 16, [(9000, 5), (100, 3), (7777, 2)], 3001), ((8, 2, 128), 64, [(6000, 1200), (3000, 1), (50, 50)], 0),
    ((16, 4, 64), 16, [(2500, 600), (4100, 40), (900, 1), (1, 1)], 1000), ((7, 1, 128), 32, [(3001, 700)], 0)])
def test_attention_over_long_caches(heads, page, seqs, window):
    s = ref.make(seqs, *heads, page, torch.bfloat16, seed=8)
    cache, batch = parts(s)
    want, err = ref.attention(s, window)
    within(sna.paged_attention(cache, batch, s["q"], window=window), want, err, "out")


def test_attention_scale_strides_and_layers():
    """A scale of its own, rows of q inside a wider projection, an output with heads outside tokens, a pool whose layers take turns."""
    s = ref.make([(90, 4), (33, 33), (200, 1)], 8, 2, 128, 16, torch.bfloat16, seed=9, layers=3)
    cache, batch = parts(s)
    want, err = ref.attention(s, scale=0.25)
    out = torch.full((8, s["q"].shape[0], 128), 7.0, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    assert sna.paged_attention(cache, batch, s["q"], scale=0.25, out=out) is out
    within(out, want, err, "out")


def test_attention_of_large_scores():
    """Scores of several hundred: the running maximum has to keep every exponential in range, whichever tile it comes from."""
    s = ref.make([(700, 3), (1300, 1)], 8, 2, 64, 16, torch.float16, seed=10)
    cache, batch = parts(s)
    want, err = ref.attention(s, scale=20.0)
    within(sna.paged_attention(cache, batch, s["q"], scale=20.0), want, err, "out")


def test_attention_without_keys_and_unused_rows():
    """A sequence shorter than its new tokens: those of negative positions see nothing and give zeros; rows of no sequence stay."""
    s = ref.make([(40, 40), (30, 2)], 4, 2, 64, 16, torch.bfloat16, seed=11)
    s["lens"][0] = 25
    cache, batch = parts(s)
    out = torch.full_like(s["q"].contiguous(), 3.0)
    sna.paged_attention(cache, batch, s["q"], out=out)
    assert (out[:15] == 0).all()
    t = dict(s, seqs=[(25, 25), (30, 2)], q=s["q"][15:])
    want, err = ref.attention(t)
    within(out[15:], want, err, "the others")


def test_attention_of_chunks_without_keys():
    """The same where the many-rows kernel takes the step; and steps without tokens, or sequences."""
    s = ref.make([(1300, 1300), (700, 2), (0, 0)], 32, 8, 128, 16, torch.bfloat16, seed=19)
    s["lens"][0] = 1200
    cache, batch = parts(s)
    out = torch.full_like(s["q"].contiguous(), 3.0)
    sna.paged_attention(cache, batch, s["q"], out=out)
    assert (out[:100] == 0).all()
    t = dict(s, seqs=[(1200, 1200), (700, 2), (0, 0)], q=s["q"][100:])
    want, err = ref.attention(t)
    within(out[100:], want, err, "the others")
    none = s["starts"] * 0
    for b, n in ((sna.PagedBatch(none, s["lens"], s["table"], 1, 1300), 3), (sna.PagedBatch(none[:1], s["lens"][:0], s["table"][:0], 1, 1), 0)):
        assert b.n_seqs == n
        q = sna.kv_append(cache, b, s["q"][:0], s["k"][:0], s["v"][:0])
        assert q.shape == (0, 32, 128) and sna.paged_attention(cache, b, q).shape == (0, 32, 128)


@pytest.mark.parametrize("heads,seqs", [((8, 2, 128), [(100, 1), (60, 3)]), ((8, 2, 128), [(300, 90), (500, 1)])])
def test_attention_with_bad_pages(heads, seqs):
    """Pages that are none, lengths beyond the table: whatever comes back for those sequences, the others are right."""
    s = ref.make(seqs + [(70, 1)], *heads, 16, torch.bfloat16, seed=12)
    cache, batch = parts(s)
    want, err = ref.attention(s)
    s["table"][0, 1] = -5
    s["table"][0, 2] = 2 ** 31 - 1
    s["lens"][1] = 10 ** 9
    out = sna.paged_attention(cache, batch, s["q"])
    torch.cuda.synchronize()
    within(out[-1:], want[-1:], err[-1:], "the last sequence")


def test_attention_past_32_bit_offsets():
    """Pages beyond 4 GiB of the pool."""
    page, H, D = 64, 8, 128
    n = (5 << 30) // (H * page * D * 2)
    kp = torch.empty(n, H, page, D, dtype=torch.bfloat16, device="cuda")
    vp = torch.empty(n, H, D, page, dtype=torch.bfloat16, device="cuda")
    seqs = [(200, 1), (130, 7)]
    s = ref.make(seqs, 32, H, D, page, torch.bfloat16, seed=13)
    ids = [[n - 1, 1, n - 3, n - 2], [n - 5, 2, n - 4]]
    for b, row in enumerate(ids):
        old = s["table"][b, : len(row)].long()
        kp[row], vp[row] = s["k_pages"][old], s["v_pages"][old]
        s["table"][b, : len(row)] = torch.tensor(row, dtype=torch.int32, device="cuda")
    s["k_pages"], s["v_pages"] = kp, vp
    cache, batch = parts(s)
    (_, _), (wk, ek), wv = ref.append(s)
    sna.kv_append(cache, batch, s["q"], s["k"], s["v"])
    within(kp[n - 2, :, 199 - 192], wk[0], ek[0], "k")
    assert torch.equal(vp[n - 2, :, :, 199 - 192], wv[0])
    want, err = ref.attention(s)
    within(sna.paged_attention(cache, batch, s["q"]), want, err, "out")


def test_step_on_another_stream_and_in_a_graph():
    """Append and attention captured once and replayed as the sequences grow, between eager calls, against eager results."""
    s = ref.make([(100, 1), (37, 1), (64, 1)], 8, 2, 64, 16, torch.bfloat16, seed=14, fill=0.0, junk=False)
    for b in range(3):                                                 # room to grow
        s["table"][b, -2:] = torch.arange(2, device="cuda", dtype=torch.int32) + 2 * b
    s["k_pages"] = torch.cat((s["k_pages"], s["k_pages"])).contiguous()
    s["v_pages"] = torch.cat((s["v_pages"], s["v_pages"])).contiguous()
    s["table"][:, -2:] += s["n_pages"]
    for b, (l, _) in enumerate(s["seqs"]):
        first = -(-l // 16)
        s["table"][b, first: first + 2] = s["table"][b, -2:].clone()
    s["max_len"] = 120
    cache, batch = parts(s)
    inv = (10000.0 ** (-torch.arange(0, 64, 2).double() / 64)).float().cuda()

    def step():
        q = sna.kv_append(cache, batch, s["q"], s["k"], s["v"], inv_freq=inv)
        return q, sna.paged_attention(cache, batch, q)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gq, gout = step()
    for i in range(4):
        s["lens"] += 1
        k0, v0 = s["k_pages"].clone(), s["v_pages"].clone()
        q, out = step()
        q, out, k1, v1 = q.clone(), out.clone(), s["k_pages"].clone(), s["v_pages"].clone()
        s["k_pages"].copy_(k0)
        s["v_pages"].copy_(v0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(gq, q) and torch.equal(gout, out) and torch.equal(s["k_pages"], k1) and torch.equal(s["v_pages"], v1)
        t = dict(s, seqs=[(int(l), 1) for l in s["lens"].tolist()], q=q)
        want, err = ref.attention(t)
        within(out, want, err, f"step {i}")
        other = torch.cuda.Stream()
        other.wait_stream(torch.cuda.current_stream())
        again = sna.paged_attention(cache, batch, q, stream=other)
        torch.cuda.current_stream().wait_stream(other)
        assert torch.equal(again, out)


# ---------------------------------------------------------------- verification
def verified(target, tokens, u, draft=None, counts=None):
    """The definition, one sequence and token at a time in Python's 64-bit numbers; also whether no comparison was a close call."""
    n, K1, V = target.shape
    out, accepted, clear = [], [], True
    for b in range(n):
        c = K1 - 1 if counts is None else min(max(int(counts[b]), 0), K1 - 1)
        a = 0
        while a < c:
            x = int(tokens[b, a])
            if not 0 <= x < V or not float(u[b, a]) * (1.0 if draft is None else float(draft[b, a, x])) < float(target[b, a, x]):
                break
            a += 1
        p = target[b, a].double()
        w = p.clone()
        if a < c:
            if draft is not None:
                w = p - draft[b, a].double()
            elif 0 <= int(tokens[b, a]) < V:
                w[int(tokens[b, a])] = 0
        w = torch.where(w > 0, w, 0.0)
        if not w.sum() > 0:
            w = torch.where(p > 0, p, 0.0)
        up = w.cumsum(0)
        if up[-1] > 0:
            at = float(u[b, K1 - 1]) * float(up[-1])
            x = int((up <= at).sum())
            clear = clear and (float((up - at).abs().min()) > 1e-12 * float(up[-1]) or float(u[b, K1 - 1]) == 0)
        else:
            x = -1
        out.append([int(t) for t in tokens[b, :a]] + [x] + [-1] * (K1 - 1 - a))
        accepted.append(a)
    return out, accepted, clear


def probabilities(n, K, V, seed, draft):
    g = torch.Generator().manual_seed(seed)
    logits = torch.randn(n, K + 1, V, generator=g) * 2.5
    if draft:
        q = torch.softmax(logits[:, :K] + torch.randn(n, K, V, generator=g), -1)
        tokens = torch.multinomial(q.reshape(-1, V), 1, generator=g).view(n, K) if K else torch.zeros(n, 0, dtype=torch.long)
    else:
        q = None
        tokens = logits[:, :K].argmax(-1)
        logits[:, :K].scatter_add_(2, tokens[..., None], torch.full((n, K, 1), 3.0))
    return torch.softmax(logits, -1), tokens, torch.rand(n, K + 1, generator=g), q


@pytest.mark.parametrize("n,K,V", [(1, 1, 1), (3, 2, 2), (5, 4, 7), (40, 8, 63), (9, 5, 64), (7, 3, 65), (33, 4, 1000), (6, 0, 1001), (4, 70, 130), (12, 5, 4097), (5, 3, 50257), (3, 7, 131072)])
@pytest.mark.parametrize("draft", [True, False])
def test_verification(n, K, V, draft):
    p, tokens, u, q = probabilities(n, K, V, 20 + V % 97, draft)
    counts = torch.randint(-1, K + 2, (n,), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    for c, t in ((None, tokens.int()), (counts, tokens)):
        want, accepted, clear = verified(p, t, u, q, c)
        assert clear
        got, acc = sna.verify_draft(p.cuda(), t.cuda(), u.cuda(), draft_probs=None if q is None else q.cuda(), n_draft=None if c is None else c.cuda())
        assert acc.tolist() == accepted
        assert got.tolist() == want


def test_verification_at_its_borders():
    """Zeros before the draw, a difference that is nothing, uniforms of 0 and next to 1, drafts outside the vocabulary, empty and NaN rows, strided rows."""
    V = 300
    p = torch.zeros(8, 3, V)
    p[:, :, 100], p[:, :, 200] = 0.25, 0.75
    q = p[:, :2].clone()
    q[:, :, 100], q[:, :, 200] = 0.25, 0.75
    tokens = torch.full((8, 2), 200, dtype=torch.int32)
    u = torch.full((8, 3), 0.5)
    u[0, 2] = 0.0                                                      # all taken, the first token with a weight
    u[1, 2] = 1 - 2.0 ** -24                                           # the last
    u[2, 0] = 1.0                                                      # 1 * 0.75 < 0.75 is false; nothing left of p - q: drawn from p
    tokens[3, 1] = V                                                   # no such token
    tokens[4, 0] = -1
    p[5] = 0.0                                                         # nothing to accept or draw
    p[6, 0, 200] = float("nan")                                        # not accepted; the difference at 100 is 0, so p's 100 is drawn
    p[7, 0, 100], p[7, 0, 200], q[7, 0, 200] = 0.5, 0.25, 0.75         # refused at 0.5 * 0.75 >= 0.25: drawn from 0.25 at 100
    want = [[200, 200, 100], [200, 200, 200], [200, -1, -1], [200, 200, -1], [200, -1, -1], [-1, -1, -1], [100, -1, -1], [100, -1, -1]]
    wide = torch.full((8, 4, V + 5), float("nan"))
    wide[:, :3, 3: V + 3] = p
    wide_q = torch.full((8, 5, V + 2), float("nan"))
    wide_q[:, 2:4, :V] = q
    assert verified(p, tokens, u, q)[:2] == (want, [2, 2, 0, 1, 0, 0, 0, 0])
    for a, d in ((p.cuda(), q.cuda()), (wide.cuda()[:, :3, 3: V + 3], wide_q.cuda()[:, 2:4, :V])):
        got, acc = sna.verify_draft(a, tokens.cuda(), u.cuda(), draft_probs=d)
        assert got.tolist() == want and acc.tolist() == [2, 2, 0, 1, 0, 0, 0, 0]


def test_verification_follows_the_target():
    """Over many uniforms the tokens that come out are the target's distribution, whatever the draft's: 5 deviations of 20000 draws."""
    n, V = 20000, 11
    g = torch.Generator().manual_seed(30)
    p, q = (torch.softmax(torch.randn(V, generator=g) * 1.5, 0) for _ in range(2))
    tokens = torch.multinomial(q, n, replacement=True, generator=g).view(n, 1)
    u = torch.rand(n, 2, generator=g)
    got, _ = sna.verify_draft(p.expand(n, 2, V).contiguous().cuda(), tokens.cuda(), u.cuda(), draft_probs=q.expand(n, 1, V).contiguous().cuda())
    share = torch.bincount(got[:, 0].cpu(), minlength=V) / n
    assert ((share - p).abs() <= 5 * (p * (1 - p) / n).sqrt()).all()


@pytest.mark.parametrize("heads,page,seqs,window", [
    ((32, 8, 128), 16, [(1100 + 37 * i % 900, i % 4 != 3) for i in range(100)], 0),                  # shares that begin and end anywhere
    ((8, 1, 64), 32, [(5000, 1), (1, 1), (0, 0)] + [(64 * i + 1, 2) for i in range(1, 30)], 0),
    ((16, 2, 64), 16, [(900 + i, i % 2) for i in range(330)] + [(3000, 1)], 0),                       # more sequences than lanes
    ((4, 4, 128), 64, [(7000, 16), (4000, 3), (6999, 9)], 2000)])
def test_attention_of_keys_shared_out(heads, page, seqs, window):
    s = ref.make([(l, int(n)) for l, n in seqs], *heads, page, torch.bfloat16, seed=15)
    cache, batch = parts(s)
    want, err = ref.attention(s, window)
    workspace = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")                      # NaN wherever it is read as fp32
    a = sna.paged_attention(cache, batch, s["q"], window=window, workspace=workspace)
    within(a, want, err, "out")
    assert torch.equal(sna.paged_attention(cache, batch, s["q"], window=window), a)                 # the sums' order is fixed


@pytest.mark.parametrize("heads,page,seqs,window", [
    ((32, 8, 128), 16, [(3000, 600), (2500, 1), (1400, 4), (900, 5), (700, 0), (1300, 130)], 0),     # beside the chunks: single tokens, drafts, idle ones
    ((8, 1, 64), 32, [(5000, 2500)], 0), ((8, 2, 128), 64, [(6000, 3000), (4100, 1)], 0),            # keys of chunks in shares
    ((32, 8, 64), 16, [(200 + 5 * i, 20 + i % 10) for i in range(40)], 0),                           # many short chunks
    ((40, 8, 128), 128, [(1000, 450), (2000, 10)], 700), ((64, 2, 64), 16, [(700, 300), (1200, 2), (60, 60)], 0)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attention_of_mixed_steps(dtype, heads, page, seqs, window):
    s = ref.make(seqs, *heads, page, ref.DT[dtype], seed=16)
    cache, batch = parts(s)
    want, err = ref.attention(s, window)
    workspace = torch.full((256 << 20,), 255, dtype=torch.uint8, device="cuda")
    a = sna.paged_attention(cache, batch, s["q"], window=window, workspace=workspace)
    within(a, want, err, "out")
    assert torch.equal(sna.paged_attention(cache, batch, s["q"], window=window), a)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,seqs,window", [((8, 2, 128), [(100, 4), (70, 1)], 0), ((4, 4, 64), [(300, 16), (50, 50)], 9), ((8, 2, 64), [(90, 30)], 0),
                                               ((8, 1, 128), [(3000, 2500), (100, 64)], 0), ((32, 8, 64), [(2100, 2000)], 100), ((16, 16, 128), [(700, 600), (80, 2)], 0)])
def test_attention_of_values_that_are_no_numbers(dtype, heads, seqs, window):
    """Infinities and NaN in values and keys reach the tokens that see them, and no others."""
    s = ref.make(seqs, *heads, 16, ref.DT[dtype], seed=17)
    want, err = ref.attention(s, window)                               # as if they were not there
    bad = torch.zeros_like(want, dtype=torch.bool)
    row = 0
    for b, (l, n) in enumerate(seqs):
        for back, dim, value in ((2, 3, float("nan")), (n // 2 + 1, 17, float("inf")), (n - 1, 40, -float("inf")), (min(l - 1, n + 20), 41, float("inf"))):
            p = l - 1 - back                                           # its position
            if not 0 <= p < l:
                continue
            s["v_pages"][s["table"][b, p // 16].long(), 0, dim, p % 16] = value
            for i in range(n):
                q = l - n + i
                if p <= q and (not window or p > q - window):
                    bad[row + i, : heads[0] // heads[1], dim] = True
        row += n
    cache, batch = parts(s)
    out = sna.paged_attention(cache, batch, s["q"], window=window).double()
    assert not torch.isfinite(out[bad]).any()
    off = (out - want).abs()
    assert (off <= err)[~bad].all(), ((off > err) & ~bad).nonzero()[:5]
    for b, (l, n) in enumerate(seqs):                                  # a key of NaN: whole rows, of the tokens that see it
        s["k_pages"][s["table"][b, (l - 1) // 16].long(), 0, (l - 1) % 16, 5] = float("nan")
    out = sna.paged_attention(cache, batch, s["q"], window=window).double()
    ends = [sum(n for _, n in seqs[: b + 1]) - 1 for b in range(len(seqs)) if seqs[b][1]]
    assert torch.isnan(out[ends][:, : heads[0] // heads[1]]).all()
    rest = ~bad
    rest[ends, : heads[0] // heads[1]] = False
    assert ((out - want).abs() <= err)[rest].all()


# Whatever launch a step gets: 16, 32 or 64 rows a block; keys shared out or walked whole by 4 or 8 waves; chunks of 128 or 256 rows
# a block, their keys whole or in shares
LAUNCHES = {
    "16 rows": ((8, 2), [(300, 1), (65, 4), (1, 1)]), "16 rows, 8 waves": ((8, 2), [(900 + 7 * i, 1 + i % 4) for i in range(20)]),
    "16 rows, shared": ((8, 2), [(5000, 4), (2100, 1), (3, 2)]), "16 rows, many": ((4, 4), [(2100 + i, 1) for i in range(150)]),
    "32 rows": ((20, 2), [(300, 3), (65, 1), (70, 2)]), "32 rows, 8 waves": ((20, 2), [(990 + i, 3) for i in range(20)]), "32 rows, shared": ((20, 2), [(5000, 3), (2100, 1), (3, 2)]),
    "64 rows": ((40, 1), [(300, 3), (65, 1), (70, 2)]), "64 rows, 8 waves": ((64, 1), [(990 + i, 1) for i in range(40)]), "64 rows, shared": ((64, 1), [(5000, 3), (2100, 1), (3, 2)]),
    "several tiles": ((8, 2), [(300, 100), (40, 40), (200, 1)]), "several tiles, shared": ((8, 2), [(4200, 100), (40, 40), (2000, 1)]),
    "several tiles of 64 rows": ((16, 4), [(1500, 500), (900, 30)] + [(700, 1)] * 20), "128-row chunks": ((8, 2), [(4000 + i, 31) for i in range(32)]), "256-row chunks": ((16, 2), [(3000, 1500), (1200, 1200), (900, 100)]),
    "chunks, shared": ((4, 1), [(9000, 2000)]), "chunks and single tokens": ((16, 2), [(3000, 1500), (2500, 1), (1800, 2)])}


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("window", [0, 777])
@pytest.mark.parametrize("launch", LAUNCHES)
def test_attention_in_every_launch(launch, window, dim, dtype):
    heads, seqs = LAUNCHES[launch]
    s = ref.make(seqs, *heads, dim, 32, ref.DT[dtype], seed=18)
    cache, batch = parts(s)
    want, err = ref.attention(s, window)
    within(sna.paged_attention(cache, batch, s["q"], window=window), want, err, "out")


@pytest.mark.parametrize("heads,seqs", [((32, 8, 128), [(5000, 1), (3000, 1)]), ((8, 2, 64), [(4000, 5), (2500, 3)]), ((16, 2, 128), [(3000, 1500), (2500, 1)]), ((4, 1, 64), [(9000, 2000)])])
def test_shared_keys_in_a_graph(heads, seqs):
    """Launches that join parts, captured with their workspace and replayed between eager calls of the same step."""
    s = ref.make(seqs, *heads, 16, torch.bfloat16, seed=21)
    cache, batch = parts(s)
    q = s["q"].contiguous()
    eager = sna.paged_attention(cache, batch, q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = sna.paged_attention(cache, batch, q)
    for i in range(3):
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(i)).to(q))
        eager = sna.paged_attention(cache, batch, q)
        out.zero_()
        graph.replay()
        again = sna.paged_attention(cache, batch, q)
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(again, eager)
    want, err = ref.attention(dict(s, q=q))
    within(out, want, err, "the last replay")


def test_tensors_that_do_not_fit_are_refused():
    s = ref.make([(3000, 1), (40, 1)], 8, 2, 128, 16, torch.bfloat16, seed=22)
    cache, batch = parts(s)
    q, k, v = (s[n].contiguous() for n in "qkv")
    inv = torch.ones(64, device="cuda")
    bad = [lambda: sna.PagedCache(s["k_pages"], s["v_pages"].half()), lambda: sna.PagedCache(s["k_pages"][:, :, ::2], s["v_pages"][..., ::2]),
           lambda: sna.PagedCache(s["k_pages"].cpu(), s["v_pages"]), lambda: sna.PagedBatch(s["starts"][:-1], s["lens"], s["table"], 1, 3000),
           lambda: sna.PagedBatch(s["starts"].long(), s["lens"], s["table"], 1, 3000), lambda: sna.PagedBatch(s["starts"], s["lens"], s["table"].t(), 1, 3000),
           lambda: sna.PagedBatch(s["starts"], s["lens"], s["table"], -1, 3000), lambda: sna.paged_attention(cache, batch, q.half()),
           lambda: sna.paged_attention(cache, batch, q.cpu()), lambda: sna.paged_attention(cache, batch, q[..., :64]), lambda: sna.paged_attention(cache, batch, q[0]),
           lambda: sna.paged_attention(cache, batch, q.transpose(1, 2).contiguous().transpose(1, 2)), lambda: sna.paged_attention(cache, batch, q, out=q[:1]),
           lambda: sna.paged_attention(cache, batch, q, window=-1), lambda: sna.paged_attention(cache, batch, q, workspace=torch.empty(1 << 24, device="cuda")),
           lambda: sna.kv_append(cache, batch, q, k[:1], v), lambda: sna.kv_append(cache, batch, q, k, q), lambda: sna.kv_append(cache, batch, q, k, v, inv_freq=inv.double()),
           lambda: sna.kv_append(cache, batch, q, k, v, inv_freq=torch.ones(129, device="cuda")), lambda: sna.kv_append(cache, batch, q, k, v, q_norm=inv, k_norm=inv),
           lambda: sna.verify_draft(torch.ones(2, 3, 9, device="cuda"), torch.zeros(2, 2, device="cuda"), torch.ones(2, 3, device="cuda")),
           lambda: sna.verify_draft(torch.ones(2, 3, 9, device="cuda"), torch.zeros(2, 2, dtype=torch.int32, device="cuda"), torch.ones(2, 2, device="cuda")),
           lambda: sna.verify_draft(torch.ones(2, 3, 9, device="cuda"), torch.zeros(2, 2, dtype=torch.int32, device="cuda"), torch.ones(2, 3, device="cuda"), draft_probs=torch.ones(2, 3, 9, device="cuda"))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: sna.paged_attention(cache, batch, q, scale=-1.0), lambda: sna.paged_attention(cache, batch, q[:, :7]), lambda: sna.kv_append(cache, batch, q, k, v, inv_freq=inv[:3]),
                 lambda: sna.kv_append(cache, batch, q, k, v, inv_freq=torch.ones(65, device="cuda")), lambda: sna.kv_append(cache, batch, q, k, v, q_norm=torch.ones(128, device="cuda"))):
        with pytest.raises(sna.SnaError):
            call()
    want, err = ref.attention(dict(s, q=q))
    within(sna.paged_attention(cache, batch, q), want, err, "and what fits still runs")


def test_tensors_that_were_replaced_in_place_are_refused():
    """A cache or batch whose tensors were resized, or given other memory, since it was made: an error, and no launch."""
    s = ref.make([(300, 2), (40, 1)], 8, 2, 64, 16, torch.bfloat16, seed=23)
    q, k, v = (s[n].contiguous() for n in "qkv")

    def refused(cache, batch):
        for call in (lambda: sna.paged_attention(cache, batch, q), lambda: sna.kv_append(cache, batch, q, k, v)):
            with pytest.raises(ValueError, match="in place|needed"):
                call()

    def grow(t):
        t.resize_(t.shape[0] + 5, *t.shape[1:])

    def swap(t):
        t.data = t.clone()

    def reset(t):
        t.set_(torch.zeros_like(t))

    def view(t):
        t.data = t.cpu()

    for change in (grow, swap, reset, view):
        for name in ("k_pages", "v_pages"):
            t = dict(s, k_pages=s["k_pages"].clone(), v_pages=s["v_pages"].clone())
            cache, batch = parts(t)
            change(t[name])
            refused(cache, batch)
        for name in ("starts", "lens", "table"):
            t = dict(s, **{name: s[name].clone()})
            cache, batch = parts(t)
            change(t[name])
            refused(cache, batch)
    t = dict(s, table=s["table"].clone())
    cache, batch = parts(t)
    t["table"].resize_(2, t["table"].shape[1] - 1)                      # smaller: the memory stays
    refused(cache, batch)
    cache, batch = parts(s)
    s["table"].add_(0)                                                  # other contents are no other tensor
    want, err = ref.attention(dict(s, q=q))
    within(sna.paged_attention(cache, batch, q), want, err, "and what has not changed still runs")


def test_expanded_outputs_are_refused():
    s = ref.make([(300, 3), (40, 1)], 8, 2, 64, 16, torch.bfloat16, seed=24)
    cache, batch = parts(s)
    q, k, v = (s[n].contiguous() for n in "qkv")
    one = torch.zeros(1, 8, 64, dtype=torch.bfloat16, device="cuda")
    for out in (one.expand(4, 8, 64), one[:, :1].expand(4, 8, 64), torch.zeros(4, 1, 64, dtype=torch.bfloat16, device="cuda").expand(4, 8, 64),
                torch.zeros(4096, dtype=torch.bfloat16, device="cuda").as_strided((4, 8, 64), (64, 64, 1))):
        for call in (lambda: sna.paged_attention(cache, batch, q, out=out), lambda: sna.kv_append(cache, batch, q, k, v, out=out)):
            with pytest.raises(sna.SnaError):
                call()
        assert (out == 0).all()
    want, err = ref.attention(dict(s, q=q))
    out = torch.zeros(3, 8, 4, 192, dtype=torch.bfloat16, device="cuda").permute(0, 2, 1, 3)[1, :, :, 64:128]       # heads outside tokens, inside more
    within(sna.paged_attention(cache, batch, q, out=out), want, err, "an output inside a larger tensor")


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,seqs,window", [((8, 2, 128), [(300, 4), (70, 2)], 0), ((4, 4, 64), [(500, 16), (90, 7)], 100), ((8, 2, 128), [(5000, 4), (2100, 3)], 0),
                                               ((20, 2, 64), [(400, 3)], 0), ((40, 1, 128), [(300, 3)], 0), ((8, 2, 64), [(300, 100)], 0)])
def test_no_number_in_one_tokens_sight_leaves_the_others_bit_for_bit(dtype, heads, seqs, window):
    """Where some token of a block sees an infinity or NaN, the keys are walked a second time: what the others get has to be
    what they get without it, to the last bit."""
    s = ref.make(seqs, *heads, 16, ref.DT[dtype], seed=25)
    cache, batch = parts(s)
    plain = sna.paged_attention(cache, batch, s["q"], window=window)
    seen = torch.zeros_like(plain, dtype=torch.bool)
    row = 0
    for b, (l, n) in enumerate(seqs):
        for back, dim, value in ((0, 3, float("nan")), (1, 17, float("inf"))):
            s["v_pages"][s["table"][b, (l - 1 - back) // 16].long(), 0, dim, (l - 1 - back) % 16] = value
            seen[row + n - 1 - back: row + n, : heads[0] // heads[1], dim] = True                  # by the last token, or the last two
        row += n
    got = sna.paged_attention(cache, batch, s["q"], window=window)
    assert not torch.isfinite(got[seen]).any()
    assert torch.equal(got[~seen], plain[~seen])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,seqs,window", [((8, 2, 128), [(900, 1), (70, 1)], 0), ((32, 8, 128), [(4000, 5), (3000, 5), (2100, 3)], 0), ((32, 8, 128), [(700, 5)] * 4, 0),
                                               ((16, 2, 64), [(2000, 4), (1500, 2)] * 4, 0), ((16, 2, 64), [(900, 4)] * 3, 300), ((20, 1, 128), [(3000, 1)] * 5, 0),
                                               ((24, 1, 64), [(5000, 1), (300, 1)], 0), ((8, 1, 128), [(9000, 4)], 0)])
def test_single_and_drafted_tokens_are_off_by_their_own_rounding(dtype, heads, seqs, window):
    """Up to 32 rows per key / value head: the error is that of rounding the 64-bit result once.  fp32 scores and sums are off by
    a few hundred steps of 2^-24 at most, less than a hundredth of half a step of either type in the norm; a tenth is allowed."""
    s = ref.make(seqs, *heads, 32, ref.DT[dtype], seed=26)
    cache, batch = parts(s)
    want, _ = ref.attention(s, window)
    off = (sna.paged_attention(cache, batch, s["q"], window=window).double() - want).norm()
    own = (want.to(ref.DT[dtype]).double() - want).norm()
    print(f"{float(off / own):.3f} of the result's own rounding", flush=True)
    assert off <= 1.1 * own


def test_bounds_that_are_loose():
    """max_new and max_len are bounds: a server may keep the same ones for every step, however few rows a step has."""
    s = ref.make([(30, 4), (9, 1)], 8, 2, 64, 16, torch.bfloat16, seed=27)
    cache = sna.PagedCache(s["k_pages"], s["v_pages"])
    want, err = ref.attention(s)
    (wq, eq), _, _ = ref.append(s)
    bounds = [sna.PagedBatch(s["starts"], s["lens"], s["table"], *b) for b in ((4, 30), (5, 30), (8, 30), (64, 40), (4096, 131072), (4096, 30))]
    for batch in bounds:
        within(sna.paged_attention(cache, batch, s["q"]), want, err, f"out, bounds {batch.max_new} and {batch.max_len}")
    for batch in bounds:
        within(sna.kv_append(cache, batch, s["q"], s["k"], s["v"]), wq, eq, f"q, bounds {batch.max_new} and {batch.max_len}")
    for max_new in (0, 2):                                              # no bounds of five tokens of two sequences
        with pytest.raises(sna.SnaError):
            sna.paged_attention(cache, sna.PagedBatch(s["starts"], s["lens"], s["table"], max_new, 30), s["q"])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("launch,several,dim,step", launches.STEPS)
def test_attention_in_each_launch_by_its_plan(launch, several, dim, step, dtype):
    """What test_paged_plan_host.py finds these steps to be launched as, unused slots full of NaN and workspaces, too."""
    heads, kv_heads, length, new, n, ragged, singles, window = step
    s = ref.make(launches.seqs(length, new, n, ragged, singles), heads, kv_heads, dim, 16, ref.DT[dtype], seed=28)
    cache, batch = parts(s)
    want, err = ref.attention(s, window)
    workspace = torch.full((256 << 20,), 255, dtype=torch.uint8, device="cuda")
    within(sna.paged_attention(cache, batch, s["q"], window=window, workspace=workspace), want, err, "out")
