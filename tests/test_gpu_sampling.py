"""Drawing tokens from filtered logits on the GPU against the definition in 64 bits, row by row."""
import math

import pytest
import torch

import paper_2312_16733_amd as sna

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def drawn(row, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, probabilities, whether no cut and no draw was a close call) of one row; settings as Python numbers, which the operator
    takes in fp32."""
    temperature, top_p, min_p = (float(torch.tensor(v, dtype=torch.float32)) for v in (temperature, top_p, min_p))
    x = row.double()
    x = torch.where(x.isnan(), -math.inf, x)
    V, top = x.numel(), x.max()
    if top == -math.inf:
        return -1, torch.zeros(V, dtype=torch.float64), True
    w = torch.exp((x - top) / temperature) if temperature > 0 else torch.zeros(V, dtype=torch.float64)
    w = torch.where(x == top, 1.0, torch.where(x == -math.inf, 0.0, w))
    order = torch.sort(x, descending=True, stable=True).indices
    s, clear = w[order].clone(), True
    k = top_k if temperature > 0 else 1
    if k > 0:
        s[k:] = 0
    kept = s > 0
    if top_p < 1:
        up = s.cumsum(0)
        at = top_p * up[-1]
        clear = clear and float((up - at).abs().min()) > 1e-10 * float(up[-1])
        kept &= up - s < at
        kept[0] = True
    if min_p > 0:
        clear = clear and float((s - min_p).abs().min()) > 1e-10
        kept &= s >= min_p
    w = torch.zeros(V, dtype=torch.float64).scatter_(0, order, torch.where(kept, s, 0.0))
    up = w.cumsum(0)
    at = u * float(up[-1])
    clear = clear and (u == 0 or float((up - at).abs().min()) > 1e-10 * float(up[-1]))
    return int((up <= at).sum()), w / up[-1], clear


def checked(logits, u, close=False, **settings):
    """Both forms of the call, with and without probabilities, against the definition."""
    n, V = logits.shape
    rows = lambda name: settings[name].tolist() if torch.is_tensor(settings.get(name)) else [settings[name]] * n if name in settings else None  # noqa: E731
    of = {name: rows(name) for name in ("temperature", "top_k", "top_p", "min_p")}
    want = [drawn(logits[i].cpu(), float(u[i]), **{name: v[i] for name, v in of.items() if v}) for i in range(n)]
    assert close or all(c for _, _, c in want), "a close call: take another seed"
    on = {name: v.cuda() if torch.is_tensor(v) else v for name, v in settings.items()}
    tokens, probs = sna.sample_tokens(logits, u.cuda(), probs=True, **on)
    alone = sna.sample_tokens(logits, u.cuda(), **on)
    assert tokens.dtype == torch.int32 and probs.dtype == torch.float32
    assert tokens.tolist() == [t for t, _, _ in want]
    assert alone.tolist() == tokens.tolist()
    p = torch.stack([q for _, q, _ in want])
    off = (probs.cpu().double() - p).abs()
    # one rounding to fp32; the sum of V weights is off by half a step of 2^-44 each, and is 1 or more
    assert (off <= p * (2.0 ** -24 + V * 2.0 ** -45 + 1e-12) + 2.0 ** -126).all(), float((off / p.clamp(min=1e-30)).max())
    assert ((probs.cpu() > 0) == (p > 2.0 ** -126)).all()
    return tokens, probs


def logits_of(n, V, dtype, seed, scale=2.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(n, V, generator=g) * scale).to(DT[dtype]).cuda(), torch.rand(n, generator=g)


SETTINGS = [{}, {"temperature": 0.7}, {"top_k": 5}, {"top_k": 1}, {"top_k": 200, "temperature": 1.3}, {"top_p": 0.9}, {"top_p": 0.5, "temperature": 0.6}, {"min_p": 0.07},
            {"top_k": 50, "top_p": 0.8}, {"top_k": 3000, "top_p": 0.95}, {"top_k": 40, "top_p": 0.93, "min_p": 0.02, "temperature": 0.9}, {"temperature": 0.0}, {"top_k": 3000}]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n,V", [(1, 1), (3, 2), (5, 7), (9, 63), (9, 64), (7, 65), (17, 1000), (6, 1001), (5, 4097), (4, 8191), (3, 16385), (3, 50257), (2, 131072), (1, 262145)])
def test_tokens_and_probabilities(dtype, n, V):
    for i, settings in enumerate(SETTINGS):
        for seed in range(10):                                         # borders are not where a rounding would decide
            logits, u = logits_of(n, V, dtype, 100 * i + seed)
            if all(drawn(logits[j].cpu(), float(u[j]), **settings)[2] for j in range(n)):
                break
        print(settings, flush=True)
        checked(logits, u, **settings)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [700, 5003, 100003])
def test_settings_of_each_row(dtype, V):
    n = 24
    t = torch.tensor([0.0, 0.5, 1.0, 1.7] * 6)
    k = torch.tensor([0, 1, 30, V, -3, 10 ** 9] * 4, dtype=torch.int32)
    p = torch.tensor([1.0, 0.9, 0.3] * 8)
    m = torch.tensor([0.0] * 8 + [0.1] * 8 + [1.0] * 8)
    logits, u = logits_of(n, V, dtype, 7)
    checked(logits, u, close=True, temperature=t, top_k=k, top_p=p, min_p=m)
    checked(logits, u, close=True, temperature=t, top_k=20, top_p=p)


@pytest.mark.parametrize("V", [40, 3000, 70001])
def test_equal_logits_go_by_their_number(V):
    """All equal; halves; both zeros; what is kept is the lowest numbers, and the draw runs over them in order."""
    u = torch.tensor([0.0, 0.3, 0.6, 1 - 2.0 ** -24])
    same = torch.full((4, V), -3.25, device="cuda")
    for settings in ({}, {"top_k": 7}, {"top_p": 0.5}, {"top_k": 30, "top_p": 0.25}, {"min_p": 1.0}, {"top_k": V - 1}):
        checked(same, u, close=True, **settings)
    zeros = torch.zeros(4, V, device="cuda")
    zeros[:, 1::2] = -0.0
    zeros[2:, V // 2] = 5.0
    checked(zeros, u, close=True, top_k=9)
    some = torch.where(torch.arange(V, device="cuda") % 3 == 0, 1.0, 0.5).repeat(4, 1).to(torch.bfloat16)
    checked(some, u, close=True, top_k=V // 2)
    assert sna.sample_tokens(same, u.cuda(), top_k=7).tolist() == [0, 2, 4, 6]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("V", [90, 20011])
def test_masks_infinities_and_nan(dtype, V):
    """Rows with most of the vocabulary masked by -inf or the lowest value; NaN; nothing left; +inf; levels far from each other."""
    logits, u = logits_of(12, V, dtype, 11)
    low = torch.finfo(DT[dtype]).min
    hide = torch.rand(12, V, generator=torch.Generator().manual_seed(2)).cuda() < 0.97
    logits[0] = torch.where(hide[0], -math.inf, logits[0])
    logits[1] = torch.where(hide[1], low, logits[1])
    logits[2] = torch.where(hide[2], math.nan, logits[2])
    logits[3] = -math.inf
    logits[4] = math.nan
    logits[5] = -math.inf
    logits[5, V - 1] = low                                             # one token left
    logits[6] = low
    logits[7, 3::20] = math.inf
    logits[8, 5] = math.inf
    logits[9, V // 3] = 3e4                                            # all others lie far below
    logits[10] = logits[10] * 1e-3 - 20
    logits[10, 0] = 20
    logits[11, ::2] = -math.inf
    for settings in ({}, {"top_k": 4}, {"top_p": 0.9}, {"top_k": 20, "top_p": 0.7, "min_p": 0.01}, {"temperature": 0.0}, {"temperature": 1e-30}, {"temperature": 1e30}, {"min_p": 0.5}):
        print(settings, flush=True)
        tokens, probs = checked(logits, u, close=True, **settings)
        assert tokens[3] == -1 and tokens[4] == -1 and (probs[3:5] == 0).all() and tokens[5] == V - 1


def test_a_large_nucleus_and_outliers():
    """A cut among tens of thousands of tokens that lie within a thousandth of each other, far below one that does not."""
    V = 60000
    g = torch.Generator().manual_seed(5)
    logits = (torch.rand(4, V, generator=g) * 1e-3 - 900).cuda()
    logits[:2, 77] = 100.0
    u = torch.rand(4, generator=g)
    for settings in ({"top_k": 20000}, {"top_k": 20001, "temperature": 300.0, "top_p": 0.999}, {"top_p": 0.37}, {"top_p": 0.9999, "temperature": 400.0}):
        checked(logits, u, close=True, **settings)


@pytest.mark.parametrize("dtype,V,scale", [("fp32", 50257, 0.05), ("fp32", 131072, 0.02), ("bf16", 16385, 0.3), ("bf16", 131072, 1.0), ("fp32", 30000, 3.0), ("fp16", 65536, 1e-4)])
def test_lists_of_every_length(dtype, V, scale):
    """Cuts whose lists a block holds, reads twice, or does not have: large counts, flat rows, ties by the thousand, one logit far below."""
    logits, u = logits_of(3, V, dtype, V + 7, scale)
    logits[2, 5] = -60000.0
    for settings in ({"top_p": 0.9}, {"top_p": 0.4, "min_p": 0.9}, {"top_k": 1500}, {"top_k": 2048}, {"top_k": 2049, "top_p": 0.5}, {"top_k": 4096}, {"top_k": 4097}, {"top_k": 12000, "top_p": 0.7},
                     {"top_k": 3500, "top_p": 0.999, "min_p": 0.5}, {"temperature": 50.0, "top_p": 0.97}, {"temperature": 0.0}):
        checked(logits, u, close=True, **settings)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n,V", [(70, 4097), (9, 50257), (3, 131072), (1, 300001)])
def test_the_best(dtype, n, V):
    """One logit that is kept: the first of several, anywhere in a row, behind NaN, infinite, both zeros, alone, or none."""
    logits, u = logits_of(n, V, dtype, V + n, 0.5)
    g = torch.Generator().manual_seed(3)
    for row in range(n):
        at = torch.randint(0, V, (3,), generator=g).tolist()
        logits[row, at] = [20.0, math.inf, 19.0, 20.0][row % 4]
        if row % 5 == 1:
            logits[row] = -math.inf
            logits[row, V - 1 - row] = -7.0
        if row % 5 == 2:
            logits[row, : V // 2] = math.nan
            logits[row, V // 2:] = torch.where(torch.arange(V - V // 2, device="cuda") % 3 == 2, 0.0, -0.0).to(logits.dtype)
        if row % 7 == 6:
            logits[row] = [-math.inf, math.nan][row % 2]
    per_row = torch.where(torch.arange(n) % 3 == 0, 0.0, -1.0)
    for settings in ({"temperature": 0.0}, {"top_k": 1}, {"temperature": 0.0, "top_p": 0.3, "min_p": 1.0, "top_k": 9}, {"top_k": 1, "temperature": 3.0, "top_p": 0.0}):
        tokens, _ = checked(logits, u, close=True, **settings)
        alike = sna.sample_tokens(logits, u.cuda(), temperature=per_row.cuda(), top_k=torch.full((n,), 40, dtype=torch.int32, device="cuda"))
        assert alike.tolist() == tokens.tolist()


def test_the_borders_of_the_draw():
    """u of 0 gives the first token that is kept, the largest u the last; what lies outside [0, 1) counts as its end."""
    logits, _ = logits_of(6, 5000, "fp32", 3)
    u = torch.tensor([0.0, 1 - 2.0 ** -24, 1.0, -1.0, 7.0, math.nan])
    tokens = sna.sample_tokens(logits, u.cuda(), top_k=25)
    kept = [torch.topk(logits[i], 25).indices.sort().values.tolist() for i in range(6)]
    assert tokens.tolist() == [kept[0][0], kept[1][-1], kept[2][-1], kept[3][0], kept[4][-1], kept[5][0]]


def test_settings_that_are_no_numbers():
    """Per-row settings are the device's: a temperature that is not positive is 0, what is no number cuts nothing, the best stays."""
    logits, u = logits_of(6, 3000, "fp32", 9)
    nan, best = math.nan, logits.argmax(1).tolist()
    f = lambda *x: torch.tensor(x).cuda()  # noqa: E731
    whole = sna.sample_tokens(logits, u.cuda()).tolist()
    assert sna.sample_tokens(logits, u.cuda(), temperature=f(nan, -1.0, 0.0, -0.0, -math.inf, 1.0)).tolist() == best[:5] + whole[5:]
    assert sna.sample_tokens(logits, u.cuda(), top_p=f(nan, 2.0, 1.0, -1.0, 0.0, -math.inf)).tolist() == whole[:3] + best[3:]
    assert sna.sample_tokens(logits, u.cuda(), min_p=f(nan, -1.0, 0.0, 2.0, 1.0, math.inf)).tolist() == whole[:3] + best[3:]
    flat = sna.sample_tokens(logits, f(0.5, 0.5, 0.5, 0.5, 0.5, 0.5), temperature=f(*[math.inf] * 6)).tolist()
    assert all(abs(t - 1500) < 3 for t in flat)                        # nearly all the same


def test_rows_of_any_stride_and_given_outputs():
    wide = torch.randn(9, 3011, device="cuda")
    u = torch.rand(9)
    out, probs = torch.full((9,), -7, dtype=torch.int32, device="cuda"), torch.full((9, 3001), 7.0, device="cuda")
    for logits in (wide[:, 3: 3003], wide[:1, 5: 3005].expand(9, 3000), wide[::2, 1: 3001]):
        n = logits.shape[0]
        want, p = sna.sample_tokens(logits.contiguous(), u[:n].cuda(), top_p=0.8, probs=True)
        got = sna.sample_tokens(logits, u[:n].cuda(), top_p=0.8, probs=probs[:n, :3000], out=out[:n])
        assert got[0].data_ptr() == out.data_ptr() and got[1].data_ptr() == probs.data_ptr()
        assert torch.equal(got[0], want) and torch.equal(got[1], p)
        assert (probs[:, 3000] == 7).all()


def test_rows_past_32_bit_offsets():
    V = 1 << 20
    pool = torch.empty((1 << 32) // 2 + V, dtype=torch.float16, device="cuda")
    logits = pool.as_strided((2, V), (1 << 31, 1))
    for i in range(2):
        logits[i] = torch.randn(V, device="cuda").half()
    checked(logits, torch.tensor([0.4, 0.7]), close=True, top_p=0.9)
    checked(logits, torch.tensor([0.2, 0.9]), close=True, top_k=100)


def test_nothing_to_draw():
    t, p = sna.sample_tokens(torch.zeros(0, 50, device="cuda"), torch.zeros(0, device="cuda"), probs=True)
    assert t.shape == (0,) and p.shape == (0, 50)


@pytest.mark.parametrize("n,V", [(3, 1000), (40, 50257), (5, 131072)])
def test_runs_are_the_same_and_graphs_replay(n, V):
    """The same bits every time, captured and on another stream; two graphs take turns."""
    logits, u = logits_of(n, V, "bf16", 21)
    u = u.cuda()
    settings = [dict(top_p=0.9, probs=True), dict(top_k=30, top_p=0.8, probs=True)]
    graphs, outs = [], []
    for k in settings:
        sna.sample_tokens(logits, u, **k)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(sna.sample_tokens(logits, u, **k))
        graphs.append(g)
    for i in range(4):
        logits.copy_(logits_of(n, V, "bf16", 30 + i)[0])
        u.copy_(torch.rand(n))
        want = [[x.clone() for x in sna.sample_tokens(logits, u, **k)] for k in settings]
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, outs):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        other = torch.cuda.Stream()
        other.wait_stream(torch.cuda.current_stream())
        again = sna.sample_tokens(logits, u, stream=other, **settings[0])
        torch.cuda.current_stream().wait_stream(other)
        assert torch.equal(again[0], want[0][0]) and torch.equal(again[1], want[0][1])


def test_a_sampled_token_is_what_verification_takes():
    """Probabilities of both models go from sampling into verify_draft: with the same model for both every draft stands."""
    n, K, V = 6, 3, 4000
    g = torch.Generator().manual_seed(8)
    logits = torch.randn(n * K, V, generator=g).cuda() * 2
    u = torch.rand(n * K, generator=g).cuda()
    tokens, probs = sna.sample_tokens(logits, u, top_k=50, top_p=0.9, probs=True)
    target = torch.cat((probs.view(n, K, V), probs.view(n, K, V)[:, :1]), 1)
    out, accepted = sna.verify_draft(target, tokens.view(n, K), torch.rand(n, K + 1, generator=g).cuda(), draft_probs=probs.view(n, K, V).contiguous())
    assert accepted.tolist() == [K] * n and torch.equal(out[:, :K], tokens.view(n, K))


@pytest.mark.parametrize("V", [1000, 5003])
def test_results_beside_what_is_read(V):
    """Probabilities in the gaps between the logits' rows are written there; what would be written over what is read is refused."""
    n = 7
    both = torch.full((n, 2 * V + 5), 3.0, device="cuda")
    logits, u = logits_of(n, V, "fp32", 12)
    both[:, :V] = logits
    u = u.cuda()
    want, p = sna.sample_tokens(logits, u, top_p=0.8, probs=True)
    got = sna.sample_tokens(both[:, :V], u, top_p=0.8, probs=both[:, V + 2: 2 * V + 2])
    assert torch.equal(got[0], want) and torch.equal(both[:, V + 2: 2 * V + 2], p)
    assert torch.equal(both[:, :V], logits) and (both[:, V: V + 2] == 3).all() and (both[:, 2 * V + 2:] == 3).all()
    k = torch.full((n,), 9, dtype=torch.int32, device="cuda")
    for bad in (dict(probs=both[:, V - 1: 2 * V - 1]), dict(probs=both[:, :V]), dict(out=k, top_k=k), dict(out=u.view(torch.int32)), dict(out=both.view(torch.int32)[1, :n]),
                dict(out=p.view(torch.int32)[2, :n], probs=p), dict(probs=torch.zeros(n * V, device="cuda").as_strided((n, V), (1, 1)))):
        with pytest.raises(sna.SnaError):
            sna.sample_tokens(both[:, :V], u, **bad)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_batches_of_thousands(dtype):
    """Rows that do not fit one workspace's worth: the same bits as in small calls, whatever their settings."""
    n, V = 8192 + 5, 4099
    g = torch.Generator(device="cuda").manual_seed(17)
    logits, u = (torch.randn(n, V + 1, generator=g, device="cuda") * 2).to(DT[dtype])[:, 1:], torch.rand(n, generator=g, device="cuda")
    logits[8193] = -math.inf
    pick = lambda *x: torch.tensor(x, device="cuda")[torch.randint(0, len(x), (n,), generator=g, device="cuda")]  # noqa: E731
    rows = {"temperature": pick(0.0, 0.7, 1.0), "top_k": pick(0, 1, 40, 2000).int(), "top_p": pick(1.0, 0.9), "min_p": pick(0.0, 0.1)}
    for settings in ({}, {"temperature": 0.0}, {"top_k": 1, "min_p": 0.5}, {"top_k": 60}, {"top_p": 0.9}, rows, {"temperature": rows["temperature"]}):
        tokens, probs = sna.sample_tokens(logits, u, probs=True, **settings)
        assert torch.equal(sna.sample_tokens(logits, u, **settings), tokens)
        for a in range(0, n, 1000):
            part = {k: v[a: a + 1000] if torch.is_tensor(v) else v for k, v in settings.items()}
            t, p = sna.sample_tokens(logits[a: a + 1000], u[a: a + 1000], probs=True, **part)
            assert torch.equal(t, tokens[a: a + 1000]) and torch.equal(p, probs[a: a + 1000]), (list(settings), a)
        assert tokens[8193] == -1
