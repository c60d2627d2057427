"""Cases and plain forms of the autoregressive serving operators: appending to a paged key / value cache (per-head norm and
position rotation on the way), attention of new tokens over that cache, verification of drafted tokens.

`run` computes an operator in elementary torch operations, or through the package's own entry points where `own` is true.

Layouts: key pages [pages][kv_heads][page_size][head_dim], value pages [pages][kv_heads][head_dim][page_size].  Sequence b of a
step has rows starts[b] .. starts[b + 1] - 1 of q, k and v; lens[b] tokens of it are cached once these are in, so its new token
i has position lens[b] - (its number of new tokens) + i; position p lies in page page_table[b][p // page_size].
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # One request of the 12 x 64-head transformer decodes a token: nothing but launch and latency.
        {"name": "append one token", "op": "append", "dtype": "bf16", "seqs": 1, "chunks": 0, "new": 1, "length": 128, "ragged": 0,
         "heads": 12, "kv_heads": 12, "head_dim": 64, "page": 16, "rot": 64, "interleaved": False, "norm": False},
        # A decode step of a large serving batch, grouped heads with norms, positions far apart.
        {"name": "append 256 decoding", "op": "append", "dtype": "fp16", "seqs": 256, "chunks": 0, "new": 1, "length": 2048, "ragged": 3,
         "heads": 32, "kv_heads": 8, "head_dim": 128, "page": 16, "rot": 128, "interleaved": False, "norm": True},
        # Chunks of four prompts enter the cache, their ends inside pages.
        {"name": "append four prompts", "op": "append", "dtype": "bf16", "seqs": 4, "chunks": 4, "new": 4093, "length": 6001, "ragged": 5,
         "heads": 32, "kv_heads": 8, "head_dim": 128, "page": 64, "rot": 64, "interleaved": True, "norm": True},
        # One request of the 12 x 64-head transformer decodes over a short context.
        {"name": "decode one short", "op": "attention", "dtype": "bf16", "seqs": 1, "chunks": 0, "new": 1, "length": 300, "ragged": 0,
         "heads": 12, "kv_heads": 12, "head_dim": 64, "page": 16, "window": 0},
        # The usual decode step: 64 requests of lengths up to 8192.
        {"name": "decode 64 ragged", "op": "attention", "dtype": "bf16", "seqs": 64, "chunks": 0, "new": 1, "length": 8192, "ragged": 7,
         "heads": 32, "kv_heads": 8, "head_dim": 128, "page": 16, "window": 0},
        # One very long context, where a single row of queries has to fill the chip.
        {"name": "decode one long", "op": "attention", "dtype": "bf16", "seqs": 1, "chunks": 0, "new": 1, "length": 131071, "ragged": 0,
         "heads": 32, "kv_heads": 8, "head_dim": 128, "page": 64, "window": 0},
        # Target pass of speculative decoding: four drafted tokens and the one before them for each of 16 requests.
        {"name": "verify pass 16 x 5", "op": "attention", "dtype": "fp16", "seqs": 16, "chunks": 16, "new": 5, "length": 4096, "ragged": 11,
         "heads": 32, "kv_heads": 8, "head_dim": 128, "page": 32, "window": 0},
        # Chunked prefill beside decoding requests, sliding window, heads of 64.
        {"name": "mixed step, window", "op": "attention", "dtype": "bf16", "seqs": 8, "chunks": 1, "new": 509, "length": 4000, "ragged": 13,
         "heads": 16, "kv_heads": 4, "head_dim": 64, "page": 16, "window": 1000},
        # The second half of a long prompt over the first.
        {"name": "prefill 4096 over 8192", "op": "attention", "dtype": "bf16", "seqs": 1, "chunks": 1, "new": 4096, "length": 8192, "ragged": 0,
         "heads": 32, "kv_heads": 8, "head_dim": 128, "page": 64, "window": 0},
        # One request, the framework's 1000 classes.
        {"name": "verify one of 1000", "op": "verify", "seqs": 1, "drafts": 4, "vocab": 1000, "draft_probs": True, "ragged": 0},
        # A serving batch with the vocabulary of a large model and drafts of different lengths.
        {"name": "verify 64 of 50257", "op": "verify", "seqs": 64, "drafts": 5, "vocab": 50257, "draft_probs": True, "ragged": 17},
        # The largest vocabularies, drafts taken greedily (no draft probabilities).
        {"name": "verify 128 of 131072", "op": "verify", "seqs": 128, "drafts": 7, "vocab": 131072, "draft_probs": False, "ragged": 19},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


HEADS = [(12, 12, 64), (16, 4, 64), (8, 1, 64), (9, 3, 64), (32, 8, 128), (16, 2, 128), (16, 16, 128), (7, 1, 128), (40, 8, 128)]


def draw(rng):
    op = rng.choice(["append", "attention", "attention", "verify"])
    if op == "verify":
        vocab, drafts = _log_int(rng, 1000, 131072), rng.randint(1, 8)
        return {"op": op, "seqs": _log_int(rng, 1, max(1, min(256, (1 << 27) // (vocab * (drafts + 1))))), "drafts": drafts, "vocab": vocab,
                "draft_probs": rng.random() < 0.6, "ragged": rng.randint(1, 999)}
    heads, kv_heads, head_dim = rng.choice(HEADS)
    case = {"op": op, "dtype": rng.choice(["bf16", "fp16"]), "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "page": rng.choice([16, 32, 64, 128]), "ragged": rng.randint(1, 999)}
    kind = rng.choice(["decode", "verify", "chunk", "mixed"])
    length = _log_int(rng, 16, 32768)
    new = 1 if kind == "decode" else rng.randint(2, min(9, length)) if kind == "verify" else _log_int(rng, 16, min(length, 4096, (3 << 28) // (heads * length)))
    # what the cache holds, what the plain form lays out for scores, and rows of q / k / v stay within the listed cases'
    seqs = min(256, (1 << 26) // (length * kv_heads * head_dim) if op == "append" else (1 << 29) // (length * kv_heads * head_dim))
    if op == "append":
        seqs = min(seqs, 16384 // new if kind != "mixed" else 256)
    else:
        seqs = min(seqs, (3 << 28) // (heads * new * length))
    seqs = _log_int(rng, 1, max(1, seqs))
    chunks = 0 if kind == "decode" else seqs if kind != "mixed" else max(1, seqs // 8)
    if op == "append":
        chunks = min(chunks, max(1, 16384 // new)) if chunks else 0
        case.update(rot=rng.choice([head_dim, head_dim // 2]), interleaved=rng.random() < 0.5, norm=rng.random() < 0.5)
    else:
        case.update(window=rng.choice([0, 0, _log_int(rng, 1, length)]))
    case.update(seqs=seqs, chunks=chunks, new=new, length=length)
    return case


def _steps(case):
    """(length after the step, new tokens) of every sequence: the first `chunks` bring up to `new` tokens, the others one."""
    r = random.Random(case["ragged"])
    fewest = lambda most: most if not case["ragged"] else r.randint((most + 1) // 2, most)  # noqa: E731
    news = [case["new"] if b == 0 and case["chunks"] else fewest(case["new"]) if b < case["chunks"] else 1 for b in range(case["seqs"])]
    lens = [case["length"] if b == 0 or not case["ragged"] else r.randint(max(n, case["length"] // 8), case["length"]) for b, n in enumerate(news)]
    return list(zip(lens, news))


def _counts(case):
    """Drafted tokens of every sequence."""
    r = random.Random(case["ragged"])
    return [case["drafts"] if b == 0 or not case["ragged"] else r.randint(0, case["drafts"]) for b in range(case["seqs"])]


def _prepare_verify(case, seed, gen):
    B, K, V = case["seqs"], case["drafts"], case["vocab"]
    rand = lambda *shape: torch.rand(*shape, generator=gen, device="cuda")  # noqa: E731
    logits = torch.randn(B, K + 1, V, generator=gen, device="cuda").mul_(2.5)
    if case["draft_probs"]:                                            # a smaller model's idea of the same distribution
        guess = logits[:, :K] + torch.randn(B, K, V, generator=gen, device="cuda")
        draft_probs = torch.softmax(guess, -1)
        tokens = torch.argmax(guess - torch.log(-torch.log(rand(B, K, V).clamp_(1e-9, 1 - 1e-7))), -1)
    else:
        draft_probs = None
        tokens = torch.argmax(logits[:, :K], -1)
        logits[:, :K].scatter_add_(2, tokens[..., None], torch.full((B, K, 1), 4.0, device="cuda"))
    return {"case": case, "target": torch.softmax(logits, -1), "draft_probs": draft_probs, "tokens": tokens.int(),
            "uniforms": rand(B, K + 1), "counts": torch.tensor(_counts(case), dtype=torch.int32, device="cuda")}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "verify":
        return _prepare_verify(case, seed, gen)
    dtype, Hq, Hk, D, ps = DTYPES[case["dtype"]], case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    steps = _steps(case)
    T, width = sum(n for _, n in steps), -(-max(l for l, _ in steps) // ps)
    used = torch.tensor([-(-l // ps) for l, _ in steps], device="cuda")
    n_pages = sum(-(-l // ps) for l, _ in steps) + 1
    # every sequence's pages lie anywhere in the pool; entries behind its last page name page 0, which is nobody's
    order = torch.randperm(n_pages - 1, generator=gen, device="cuda") + 1
    at = (torch.cumsum(used, 0) - used)[:, None] + torch.arange(width, device="cuda")
    inside = torch.arange(width, device="cuda") < used[:, None]
    page_table = torch.where(inside, order[at.clamp_(max=n_pages - 2)], 0).int()
    starts = torch.tensor([0] + [n for _, n in steps], device="cuda").cumsum(0).int()
    randn = lambda *shape: torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)  # noqa: E731
    state = {"case": case, "starts": starts, "lens": torch.tensor([l for l, _ in steps], dtype=torch.int32, device="cuda"),
             "page_table": page_table, "max_new": max(n for _, n in steps), "max_len": max(l for l, _ in steps),
             "k_pages": randn(n_pages, Hk, ps, D), "v_pages": randn(n_pages, Hk, D, ps)}
    if case["op"] == "attention":
        state["q"] = randn(T, Hq, D)
        return state
    qkv = randn(T, (Hq + 2 * Hk) * D)                                  # one projection's output, read in place
    state["q"], state["k"], state["v"] = (x.unflatten(1, (-1, D)) for x in qkv.split([Hq * D, Hk * D, Hk * D], 1))
    r = torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / case["rot"]
    state["inv_freq"] = (10000.0 ** -r).float()
    for name in ("q_norm", "k_norm"):
        state[name] = torch.rand(D, generator=gen, device="cuda") + 0.5 if case["norm"] else None
    return state


# ---- plain forms -----------------------------------------------------------------------------------------------------------
def _tokens(s):
    """Sequence and position of every new token, int64."""
    starts, lens = s["starts"].long(), s["lens"].long()
    t = torch.arange(s["q"].shape[0], device="cuda")
    seq = torch.searchsorted(starts, t, right=True) - 1
    return seq, lens[seq] - starts[seq + 1] + t


def _normed(x, weight):
    x = x.float()
    return x if weight is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * weight


def _rotated(x, cos, sin, interleaved):
    """x [T][heads][head_dim] with its leading 2 * cos.shape[-1] elements rotated in pairs."""
    half = cos.shape[-1]
    r = x[..., : 2 * half]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :half], r[..., half:])
    u, v = a * cos - b * sin, a * sin + b * cos
    r = torch.stack((u, v), -1).flatten(-2) if interleaved else torch.cat((u, v), -1)
    return torch.cat((r, x[..., 2 * half:]), -1)


def _append(s):
    c, dtype, ps = s["case"], s["q"].dtype, s["case"]["page"]
    seq, pos = _tokens(s)
    angle = pos.double()[:, None, None] * s["inv_freq"].double()       # far positions: the angle itself needs 64 bits
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    q = _rotated(_normed(s["q"], s["q_norm"]), cos, sin, c["interleaved"]).to(dtype)
    k = _rotated(_normed(s["k"], s["k_norm"]), cos, sin, c["interleaved"]).to(dtype)
    page, slot = s["page_table"][seq, pos // ps].long(), pos % ps
    s["k_pages"][page, :, slot] = k
    s["v_pages"][page, :, :, slot] = s["v"]
    return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _attention(s):
    c, q = s["case"], s["q"]
    Hk, D, G, ps, N = c["kv_heads"], c["head_dim"], c["heads"] // c["kv_heads"], c["page"], s["max_new"]
    B, width = s["page_table"].shape
    pages, starts, lens = s["page_table"].long(), s["starts"].long(), s["lens"].long()
    k = s["k_pages"][pages].permute(0, 2, 4, 1, 3).reshape(B, Hk, D, width * ps).float()
    v = s["v_pages"][pages].permute(0, 2, 1, 4, 3).reshape(B, Hk, width * ps, D).float()
    new = torch.arange(N, device="cuda")
    rows = (starts[:-1, None] + new).clamp(max=q.shape[0] - 1)
    qs = q[rows].view(B, N, Hk, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * N, D).float()
    scores = torch.matmul(qs * D ** -0.5, k).view(B, Hk, G, N, width * ps)
    q_pos = ((lens - starts[1:] + starts[:-1])[:, None] + new)[:, :, None]
    k_pos = torch.arange(width * ps, device="cuda")
    hidden = k_pos > q_pos
    if c["window"]:
        hidden |= k_pos <= q_pos - c["window"]
    scores.masked_fill_(hidden[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    scores = scores.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = scores.sum(-1, keepdim=True)
    out = torch.matmul(scores.view(B, Hk, G * N, width * ps), v).view(B, Hk, G, N, D)
    out = out / torch.where(total == 0, 1.0, total)
    seq, _ = _tokens(s)
    i = torch.arange(q.shape[0], device="cuda") - starts[seq]
    return {"out": out[seq, :, :, i].reshape(q.shape).to(q.dtype)}


def _verify(s):
    target, tokens, u, counts = s["target"], s["tokens"].long(), s["uniforms"].double(), s["counts"].long()
    B, K = tokens.shape
    b, i = torch.arange(B, device="cuda"), torch.arange(K, device="cuda")
    p = target[b[:, None], i, tokens].double()
    q = torch.ones_like(p) if s["draft_probs"] is None else s["draft_probs"][b[:, None], i, tokens].double()
    taken = (u[:, :K] * q < p) & (i < counts[:, None])
    accepted = torch.cumprod(taken.long(), 1).sum(1)
    row = target[b, accepted].double()                                 # 64 bits: a draw may fall next to a border
    at = accepted.clamp(max=K - 1)
    if s["draft_probs"] is None:
        away = torch.zeros_like(row).scatter_(1, tokens[b, at][:, None], math.inf)
    else:
        away = s["draft_probs"][b, at].double()
    rest = torch.where((accepted < counts)[:, None], row - away, row).clamp_(min=0.0)
    rest = torch.where((rest.sum(1) > 0)[:, None], rest, row)
    up_to = rest.cumsum(1)
    drawn = (up_to <= u[:, K:] * up_to[:, -1:]).sum(1)
    place = torch.arange(K + 1, device="cuda")
    out = torch.where(place < accepted[:, None], torch.cat((tokens, tokens[:, :1]), 1), -1)
    out = torch.where(place == accepted[:, None], drawn[:, None], out)
    return {"tokens": out.int(), "accepted": accepted.int()}


def run(state):
    if own:
        return _run_own(state)
    return {"append": _append, "attention": _attention, "verify": _verify}[state["case"]["op"]](state)


# ---- the package's operators -----------------------------------------------------------------------------------------------
def _run_own(s):
    import paper_2312_16733_amd as sna
    c = s["case"]
    if c["op"] == "verify":
        tokens, accepted = sna.verify_draft(s["target"], s["tokens"], s["uniforms"], draft_probs=s["draft_probs"], n_draft=s["counts"])
        return {"tokens": tokens, "accepted": accepted}
    cache = sna.PagedCache(s["k_pages"], s["v_pages"])
    batch = sna.PagedBatch(s["starts"], s["lens"], s["page_table"], s["max_new"], s["max_len"])
    if c["op"] == "attention":
        return {"out": sna.paged_attention(cache, batch, s["q"], window=c["window"])}
    q = sna.kv_append(cache, batch, s["q"], s["k"], s["v"], inv_freq=s["inv_freq"], interleaved=c["interleaved"],
                      q_norm=s["q_norm"], k_norm=s["k_norm"], eps=1e-6)
    return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


# ---- what a pass cannot do without, and what it returns in 64 bits ------------------------------------------------------------
def work(case):
    if case["op"] == "verify":
        rows = case["seqs"] * (2 if case["draft_probs"] else 1)        # the row drawn from, and the draft's
        return {"bytes": 4 * rows * case["vocab"] + 20 * case["seqs"] * case["drafts"], "flops": 2 * rows * case["vocab"]}
    Hq, Hk, D = case["heads"], case["kv_heads"], case["head_dim"]
    steps = _steps(case)
    T = sum(n for _, n in steps)
    if case["op"] == "append":
        return {"bytes": 4 * T * (Hq + 2 * Hk) * D, "flops": T * (Hq + Hk) * (3 * case["rot"] + (4 * D if case["norm"] else 0))}
    W = case["window"] or case["length"]
    seen = sum(min(l, n + W - 1) for l, n in steps)                    # keys that some new token of the sequence sees
    pairs = sum(sum(min(W, l - n + 1 + i) for i in range(n)) for l, n in steps)
    return {"bytes": 4 * seen * Hk * D + 4 * T * Hq * D, "flops": 4 * D * Hq * pairs}


def _exact_append(s):
    c, ps = s["case"], s["case"]["page"]
    out = {"q": s["q"].double(), "k_pages": s["k_pages"].double(), "v_pages": s["v_pages"].double()}
    table, half = s["page_table"].long(), c["rot"] // 2
    row = 0
    for b, (length, n) in enumerate(_steps(c)):
        pos = torch.arange(length - n, length, device="cuda")
        turn = torch.polar(torch.ones(n, half, dtype=torch.float64, device="cuda"), pos.double()[:, None] * s["inv_freq"].double())
        for name, weight in (("q", s["q_norm"]), ("k", s["k_norm"])):
            x = s[name][row: row + n].double()
            if weight is not None:
                x = x / (x.pow(2).mean(2, keepdim=True) + 1e-6).sqrt() * weight.double()
            r = x[:, :, : 2 * half]
            pairs = r.reshape(n, -1, half, 2) if c["interleaved"] else r.reshape(n, -1, 2, half).transpose(2, 3)
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None])
            x[:, :, : 2 * half] = (z if c["interleaved"] else z.transpose(2, 3)).reshape(r.shape)
            if name == "q":
                out["q"][row: row + n] = x
            else:
                out["k_pages"][table[b, pos // ps], :, pos % ps] = x
        out["v_pages"][table[b, pos // ps], :, :, pos % ps] = s["v"][row: row + n].double()
        row += n
    return out


def _exact_attention(s):
    c = s["case"]
    G, D = c["heads"] // c["kv_heads"], c["head_dim"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    row = 0
    for b, (length, n) in enumerate(_steps(c)):
        pages = s["page_table"][b, : -(-length // c["page"])].long()
        pos = torch.arange(length - n, length, device="cuda")[:, None]
        key = torch.arange(length, device="cuda")[None, :]
        seen = (key <= pos) & (key > pos - (c["window"] or length))
        for h in range(c["kv_heads"]):
            k = s["k_pages"][pages, h].reshape(-1, D)[:length].double()
            v = s["v_pages"][pages, h].transpose(1, 2).reshape(-1, D)[:length].double()
            for g in range(G):
                x = s["q"][row: row + n, h * G + g].double() @ k.t() / math.sqrt(D)
                out[row: row + n, h * G + g] = torch.softmax(x.masked_fill(~seen, -math.inf), 1) @ v
        row += n
    return {"out": out}


def exact(case, seed):
    if case["op"] == "verify":
        return None                                                    # whole numbers
    s = prepare(case, seed)
    return _exact_append(s) if case["op"] == "append" else _exact_attention(s)
