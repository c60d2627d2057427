"""Cases and plain forms of the operators that sampling and trees of drafted tokens need beside a paged cache: drawing tokens from
filtered logits, attention of a tree's tokens over the cache, the walk along the tokens that stand, moving their keys and values up,
and copying pages for sequences that part.

`run` computes an operator in elementary torch operations, or through the package's own entry points where `own` is true.

Layouts: key pages [pages][kv_heads][page_size][head_dim], value pages [pages][kv_heads][head_dim][page_size].  Sequence b of a
step has rows starts[b] .. starts[b + 1] - 1; lens[b] slots of it are cached once these are in, the last ones theirs.  A tree's
token sees the first `prefix` slots (all but the step's own, if none is given) and those of the following that its mask names:
bit j of word w is slot prefix + 64 w + j.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # Drafting: the second level of one request's tree, over a short context of the 12 x 64-head transformer.  Latency.
        {"name": "tree level of 4, one short", "op": "tree", "dtype": "bf16", "seqs": 1, "nodes": 4, "earlier": 5, "length": 300, "ragged": 0,
         "heads": 12, "kv_heads": 12, "head_dim": 64, "page": 16, "window": 0},
        # The target's pass over the trees of a serving batch.
        {"name": "trees of 32, 16 ragged", "op": "tree", "dtype": "fp16", "seqs": 16, "nodes": 32, "earlier": 0, "length": 4096, "ragged": 3,
         "heads": 32, "kv_heads": 8, "head_dim": 128, "page": 16, "window": 0},
        # One request with a long context and a large tree, whose masks take two words.
        {"name": "tree of 77, one long", "op": "tree", "dtype": "bf16", "seqs": 1, "nodes": 77, "earlier": 0, "length": 65519, "ragged": 0,
         "heads": 32, "kv_heads": 8, "head_dim": 128, "page": 64, "window": 0},
        # One request, the framework's 1000 classes.
        {"name": "sample one of 1000", "op": "sample", "dtype": "fp32", "rows": 1, "vocab": 1000, "temperature": 0.8, "top_k": 50, "top_p": 0.9, "min_p": 0.0,
         "mixed": 0, "probs": False},
        # A serving batch whose requests each have their own settings, greedy ones among them, probabilities for a verification.
        {"name": "sample 64 of 50257, mixed", "op": "sample", "dtype": "bf16", "rows": 64, "vocab": 50257, "temperature": 1.0, "top_k": 0, "top_p": 1.0, "min_p": 0.0,
         "mixed": 5, "probs": True},
        # The largest vocabularies, a nucleus of thousands of tokens.
        {"name": "sample 128 of 131072", "op": "sample", "dtype": "fp32", "rows": 128, "vocab": 131072, "temperature": 1.0, "top_k": 0, "top_p": 0.95, "min_p": 0.0,
         "mixed": 0, "probs": False},
        # Which of one request's drafted tokens stand.
        {"name": "walk one tree of 13", "op": "walk", "seqs": 1, "nodes": 13, "vocab": 1000, "ragged": 0},
        # The same for a large batch of large trees.
        {"name": "walk 256 trees of 64", "op": "walk", "seqs": 256, "nodes": 64, "vocab": 50257, "ragged": 7},
        # One request's accepted tokens move up, six layers of 4 heads.
        {"name": "compact one of 13", "op": "compact", "dtype": "bf16", "seqs": 1, "nodes": 13, "kept": 4, "length": 150, "ragged": 0, "kv_heads": 24, "head_dim": 64, "page": 16},
        # A serving batch, the layers of a page next to each other: 32 layers of 8 heads.
        {"name": "compact 64 of 32", "op": "compact", "dtype": "fp16", "seqs": 64, "nodes": 32, "kept": 8, "length": 80, "ragged": 11, "kv_heads": 256, "head_dim": 128, "page": 16},
        # One request parts in two: its last page in six layers of 4 heads.
        {"name": "copy one page", "op": "copy", "dtype": "bf16", "pairs": 1, "kv_heads": 24, "head_dim": 64, "page": 16},
        # A batch of prompts, four continuations each, 32 layers of 8 heads.
        {"name": "copy 192 pages", "op": "copy", "dtype": "bf16", "pairs": 192, "kv_heads": 256, "head_dim": 128, "page": 16},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


HEADS = [(12, 12, 64), (16, 4, 64), (8, 1, 64), (9, 3, 64), (32, 8, 128), (16, 2, 128), (16, 16, 128), (7, 1, 128), (40, 8, 128)]


def draw(rng):
    op = rng.choice(["tree", "tree", "sample", "sample", "walk", "compact", "copy"])
    if op == "sample":
        vocab = _log_int(rng, 1000, 131072)
        return {"op": op, "dtype": rng.choice(["fp32", "bf16", "fp16"]), "rows": _log_int(rng, 1, max(1, min(512, (1 << 24) // vocab))), "vocab": vocab,
                "temperature": round(rng.uniform(0.3, 1.5), 2), "top_k": rng.choice([0, 0, _log_int(rng, 1, 1000)]), "top_p": rng.choice([1.0, round(rng.uniform(0.3, 0.99), 2)]),
                "min_p": rng.choice([0.0, 0.0, round(rng.uniform(0.01, 0.2), 2)]), "mixed": rng.choice([0, rng.randint(1, 999)]), "probs": rng.random() < 0.4}
    if op == "walk":
        return {"op": op, "seqs": _log_int(rng, 1, 256), "nodes": _log_int(rng, 2, 200), "vocab": _log_int(rng, 1000, 131072), "ragged": rng.randint(1, 999)}
    heads, kv_heads, head_dim = rng.choice(HEADS)
    case = {"op": op, "dtype": rng.choice(["bf16", "fp16"]), "head_dim": head_dim, "page": rng.choice([16, 32, 64, 128])}
    if op != "tree":
        kv_heads *= rng.choice([1, 4, 16])                             # of several layers
        page_size = kv_heads * head_dim * case["page"]
        case.update(kv_heads=kv_heads)
        if op == "copy":
            return {**case, "pairs": _log_int(rng, 1, max(1, min(400, (96 << 20) // page_size)))}
        nodes, length = _log_int(rng, 2, 64), _log_int(rng, 1, 200)
        pages = -(-(nodes + length) // case["page"])
        return {**case, "nodes": nodes, "kept": rng.randint(1, max(1, min(8, nodes // 2))), "length": nodes + length,
                "seqs": _log_int(rng, 1, max(1, min(64, (150 << 20) // (page_size * pages)))), "ragged": rng.randint(1, 999)}
    nodes, earlier, length = _log_int(rng, 1, 200), rng.choice([0, 0, _log_int(rng, 1, 60)]), _log_int(rng, 16, 32768)
    length += nodes + earlier
    # what the cache holds and what the plain form lays out for scores stay within the listed cases'
    seqs = _log_int(rng, 1, max(1, min(64, (1 << 29) // (length * kv_heads * head_dim), (1 << 27) // (heads * nodes * length))))
    return {**case, "heads": heads, "kv_heads": kv_heads, "nodes": nodes, "earlier": earlier, "length": length, "seqs": seqs,
            "window": rng.choice([0, 0, _log_int(rng, 64, length + 64)]), "ragged": rng.randint(1, 999)}


def _steps(case):
    """(slots after the step, new tokens) of every sequence."""
    r = random.Random(case["ragged"])
    out = []
    for b in range(case["seqs"]):
        new = case["nodes"] if b == 0 or not case["ragged"] else r.randint((case["nodes"] + 1) // 2, case["nodes"])
        least = new + case.get("earlier", 0)
        out.append((case["length"] if b == 0 or not case["ragged"] else r.randint(max(least, case["length"] // 4), case["length"]), new))
    return out


def _tree(r, n):
    """Parents of n tokens, the first of them the root: each draws its parent among the latest few, as trees grow level by level."""
    return [-1] + [r.randint(max(0, i // 3 - 1), min(i - 1, i // 2)) for i in range(1, n)]


def _masks(parents):
    seen, depth = [], []
    for i, p in enumerate(parents):
        seen.append(1 << i | (seen[p] if i else 0))
        depth.append(depth[p] + 1 if i else 0)
    return seen, depth


def _kept(case, seed):
    """The accepted path of every sequence: rising, beginning with the root, and behind the slots that it moves to, so that a second
    pass moves the same tokens."""
    r = random.Random(seed)
    kept, counts = [], []
    for _, new in _steps(case):
        n = r.randint(1, max(1, min(case["kept"], new // 2)))
        kept.append([0] + sorted(r.sample(range(n, new), n - 1)) if n > 1 else [0])
        counts.append(n)
    if not case["ragged"]:
        new = case["nodes"]
        counts = [case["kept"]] * len(kept)
        kept = [[0] + sorted(r.sample(range(case["kept"], new), case["kept"] - 1)) for _ in kept]
    return kept, counts


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _paged(case, gen):
    """The step's sequences and pages full of numbers; every sequence's pages lie anywhere in the pool, page 0 is nobody's."""
    ps, steps = case["page"], _steps(case)
    used = torch.tensor([-(-l // ps) for l, _ in steps], device="cuda")
    n_pages, width = sum(-(-l // ps) for l, _ in steps) + 1, -(-max(l for l, _ in steps) // ps)
    order = torch.randperm(n_pages - 1, generator=gen, device="cuda") + 1
    at = (torch.cumsum(used, 0) - used)[:, None] + torch.arange(width, device="cuda")
    inside = torch.arange(width, device="cuda") < used[:, None]
    rand = lambda *shape: torch.randn(*shape, generator=gen, device="cuda", dtype=DTYPES[case["dtype"]])  # noqa: E731
    return {"case": case, "page_table": torch.where(inside, order[at.clamp_(max=n_pages - 2)], 0).int(), "starts": _ints([0] + [n for _, n in steps]).cumsum(0).int(),
            "lens": _ints([l for l, _ in steps]), "max_new": max(n for _, n in steps), "max_len": max(l for l, _ in steps),
            "k_pages": rand(n_pages, case["kv_heads"], ps, case["head_dim"]), "v_pages": rand(n_pages, case["kv_heads"], case["head_dim"], ps)}


def _prepare_tree(case, seed, gen):
    s = _paged(case, gen)
    r, steps, e = random.Random(seed), _steps(case), case["earlier"]
    words = -(-(e + s["max_new"]) // 64)
    masks, positions = [], []
    for length, new in steps:
        seen, depth = _masks(_tree(r, e + new))
        for m, d in zip(seen[e:], depth[e:]):
            masks.append([(m >> 64 * w & (1 << 64) - 1) - (1 << 64) * (m >> 64 * w + 63 & 1) for w in range(words)])
            positions.append(length - new - e + d)
    s["masks"], s["positions"] = torch.tensor(masks, dtype=torch.int64, device="cuda"), _ints(positions)
    s["prefix"] = _ints([l - n - e for l, n in steps]) if e else None
    s["q"] = torch.randn(len(masks), case["heads"], case["head_dim"], generator=gen, device="cuda", dtype=DTYPES[case["dtype"]])
    return s


def _prepare_sample(case, seed, gen):
    n, V = case["rows"], case["vocab"]
    logits = torch.randn(n, V, generator=gen, device="cuda").mul_(2.0)
    # a handful of likely tokens, more of them in some rows than in others
    likely = torch.randint(0, V, (n, 8), generator=gen, device="cuda")
    logits.scatter_add_(1, likely, torch.rand(n, 8, generator=gen, device="cuda") * torch.rand(n, 1, generator=gen, device="cuda") * 12)
    s = {"case": case, "logits": logits.to(DTYPES[case["dtype"]]), "uniforms": torch.rand(n, generator=gen, device="cuda")}
    for name, choices in (("temperature", [0.0, 0.6, 0.8, 1.0, 1.2]), ("top_k", [0, 1, 40, 50, 200]), ("top_p", [1.0, 0.8, 0.9, 0.95]), ("min_p", [0.0, 0.0, 0.05, 0.1])):
        if case["mixed"]:
            r = random.Random(f"{name} {case['mixed']}")
            rows = [r.choice(choices) for _ in range(n)]
            s[name] = _ints(rows) if name == "top_k" else torch.tensor(rows, device="cuda")
        else:
            s[name] = case[name]
    return s


def _prepare_walk(case, seed, gen):
    r, V = random.Random(seed), case["vocab"]
    sizes = [n for _, n in _steps({**case, "length": case["nodes"]})]
    parents, tokens, sampled = [], [], []
    for n in sizes:
        p = _tree(r, n)
        t = [r.randrange(V) for _ in range(n)]
        children = [[] for _ in range(n)]
        for j in range(1, n):
            children[p[j]].append(j)
        parents += p
        tokens += t
        sampled += [t[r.choice(c)] if c and r.random() < 0.75 else r.randrange(V) for c in children]
    n = len(sizes)
    return {"case": case, "starts": _ints([0] + sizes).cumsum(0).int(), "lens": _ints(sizes), "page_table": torch.zeros(n, -(-max(sizes) // 16), dtype=torch.int32, device="cuda"),
            "max_new": max(sizes), "max_len": max(sizes), "parents": _ints(parents), "tokens": _ints(tokens), "sampled": _ints(sampled)}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "tree":
        return _prepare_tree(case, seed, gen)
    if case["op"] == "sample":
        return _prepare_sample(case, seed, gen)
    if case["op"] == "walk":
        return _prepare_walk(case, seed, gen)
    if case["op"] == "compact":
        s = _paged(case, gen)
        kept, counts = _kept(case, seed)
        width = max(counts)
        s["kept"], s["counts"] = _ints([k + [-1] * (width - len(k)) for k in kept]), _ints(counts)
        return s
    n, shape = 2 * case["pairs"] + 3, (case["kv_heads"], case["page"], case["head_dim"])
    order = torch.randperm(n, generator=gen, device="cuda").int()
    # several continuations part from one page
    source = order[torch.randint(0, max(1, case["pairs"] // 3), (case["pairs"],), generator=gen, device="cuda")]
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda", dtype=DTYPES[case["dtype"]])  # noqa: E731
    return {"case": case, "k_pages": rand(n, *shape), "v_pages": rand(n, shape[0], shape[2], shape[1]), "source": source, "target": order[case["pairs"]: 2 * case["pairs"]].contiguous()}


# ---- plain forms -----------------------------------------------------------------------------------------------------------
def _rows(s, n):
    """Sequence of every row of the step, and its place there."""
    starts, t = s["starts"].long(), torch.arange(n, device="cuda")
    seq = torch.searchsorted(starts, t, right=True) - 1
    return seq, t - starts[seq]


def _plain_tree(s):
    c, q = s["case"], s["q"]
    Hk, D, G, ps, N = c["kv_heads"], c["head_dim"], c["heads"] // c["kv_heads"], c["page"], s["max_new"]
    B, width = s["page_table"].shape
    pages, starts, lens = s["page_table"].long(), s["starts"].long(), s["lens"].long()
    k = s["k_pages"][pages].permute(0, 2, 4, 1, 3).reshape(B, Hk, D, width * ps).float()
    v = s["v_pages"][pages].permute(0, 2, 1, 4, 3).reshape(B, Hk, width * ps, D).float()
    rows = (starts[:-1, None] + torch.arange(N, device="cuda")).clamp(max=q.shape[0] - 1)
    qs = q[rows].view(B, N, Hk, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * N, D).float()
    scores = torch.matmul(qs * D ** -0.5, k).view(B, Hk, G, N, width * ps)
    prefix = (lens - starts[1:] + starts[:-1] if s["prefix"] is None else s["prefix"].long())[:, None, None]
    slot = torch.arange(width * ps, device="cuda")
    bit = (slot - prefix).clamp(min=0).expand(B, N, -1)
    words = s["masks"][rows].gather(2, (bit >> 6).clamp(max=s["masks"].shape[1] - 1))
    seen = (words >> (bit & 63) & 1).bool() & (bit < 64 * s["masks"].shape[1])
    before = slot < prefix
    if c["window"]:
        before = before & (slot > s["positions"].long()[rows][:, :, None] - c["window"])
    seen = (before | (seen & (slot >= prefix))) & (slot < lens[:, None, None])
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    scores = scores.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = scores.sum(-1, keepdim=True)
    out = torch.matmul(scores.view(B, Hk, G * N, width * ps), v).view(B, Hk, G, N, D) / torch.where(total == 0, 1.0, total)
    seq, i = _rows(s, q.shape[0])
    return {"out": out[seq, :, :, i].reshape(q.shape).to(q.dtype)}


def _plain_sample(s):
    x = s["logits"].double()                                           # 64 bits: a draw may fall next to a border
    n, V = x.shape
    per_row = lambda name: torch.as_tensor(s[name], device="cuda").double().expand(n)[:, None]  # noqa: E731
    temperature, top_k, top_p, min_p = (per_row(name) for name in ("temperature", "top_k", "top_p", "min_p"))
    x = torch.where(x.isnan(), -math.inf, x)
    top = x.amax(1, keepdim=True)
    w = torch.exp((x - top) / torch.where(temperature > 0, temperature, 1.0))
    w = torch.where(x == -math.inf, 0.0, torch.where(x == top, 1.0, w))
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    place = torch.arange(V, device="cuda")
    most = torch.where(temperature > 0, torch.where(top_k > 0, top_k, V), 1)
    sorted_w = torch.where(place < most, w.gather(1, order), 0.0)
    up = sorted_w.cumsum(1)
    kept = (up - sorted_w < top_p * up[:, -1:]) | (top_p >= 1) | (place == 0)
    w = torch.zeros_like(w).scatter_(1, order, torch.where(kept & (sorted_w >= min_p), sorted_w, 0.0))
    up = w.cumsum(1)
    drawn = (up <= s["uniforms"].double()[:, None] * up[:, -1:]).sum(1)
    out = {"tokens": torch.where(up[:, -1] > 0, drawn, -1).int()}
    if s["case"]["probs"]:
        out["probs"] = (w / torch.where(up[:, -1:] > 0, up[:, -1:], 1.0)).float()
    return out


def _plain_walk(s):
    tokens, sampled, parents, N = s["tokens"], s["sampled"], s["parents"].long(), s["max_new"]
    seq, i = _rows(s, tokens.shape[0])
    first = s["starts"].long()[seq]
    parent = (first + parents).clamp(min=0)
    fits = (i > 0) & (tokens == sampled[parent])
    # of the children that fit, the first one
    lowest = torch.full((tokens.shape[0],), 1 << 40, device="cuda").scatter_reduce_(0, torch.where(fits, parent, 0), torch.where(fits, i, 1 << 40), "amin")
    fits &= lowest[parent] == i
    B = s["starts"].shape[0] - 1
    above = torch.zeros(B, N, N, device="cuda")                        # above[b][i][j]: j is i or one of those it comes from
    above[seq, i, torch.where(i > 0, parents, i)] = 1
    above[seq, i, i] = 1
    for _ in range(max(1, (N - 1).bit_length())):
        above = torch.matmul(above, above).clamp_(max=1)
    broken = torch.ones(B, N, device="cuda")
    broken[seq, i] = (~fits & (i > 0)).float()
    stands = torch.matmul(above, broken[:, :, None])[:, :, 0] == 0
    stands &= torch.arange(N, device="cuda") < (s["starts"][1:] - s["starts"][:-1])[:, None]
    counts = stands.sum(1)
    place = torch.arange(N, device="cuda")
    kept = torch.sort(torch.where(stands, place, N), 1).values
    last = kept.gather(1, (counts - 1).clamp(min=0)[:, None])[:, 0]
    following = sampled[(s["starts"][:-1].long() + last).clamp(max=tokens.shape[0] - 1)]
    return {"kept": torch.where(kept < N, kept, -1).int(), "counts": counts.int(), "next": torch.where(counts > 0, following, -1).int()}


def _plain_compact(s):
    ps, kept, counts = s["case"]["page"], s["kept"].long(), s["counts"].long()
    B, K = kept.shape
    old = (s["lens"] - s["starts"][1:] + s["starts"][:-1]).long()
    b, i = torch.where(torch.arange(K, device="cuda") < counts[:, None])
    source, target = old[b] + kept[b, i], old[b] + i
    table = s["page_table"].long()
    from_page, to_page = table[b, source // ps], table[b, target // ps]
    k, v = s["k_pages"][from_page, :, source % ps], s["v_pages"][from_page, :, :, source % ps]
    s["k_pages"][to_page, :, target % ps] = k
    s["v_pages"][to_page, :, :, target % ps] = v
    return {"lens": (old + counts).int(), "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _plain_copy(s):
    source, target = s["source"].long(), s["target"].long()
    s["k_pages"][target] = s["k_pages"][source]
    s["v_pages"][target] = s["v_pages"][source]
    return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def run(state):
    if own:
        return _run_own(state)
    return {"tree": _plain_tree, "sample": _plain_sample, "walk": _plain_walk, "compact": _plain_compact, "copy": _plain_copy}[state["case"]["op"]](state)


# ---- the package's operators -----------------------------------------------------------------------------------------------
def _run_own(s):
    import paper_2312_16733_amd as sna
    c = s["case"]
    if c["op"] == "sample":
        got = sna.sample_tokens(s["logits"], s["uniforms"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], probs=c["probs"])
        return dict(zip(("tokens", "probs"), got)) if c["probs"] else {"tokens": got}
    if c["op"] == "copy":
        sna.copy_pages(sna.PagedCache(s["k_pages"], s["v_pages"]), s["source"], s["target"])
        return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    batch = sna.PagedBatch(s["starts"], s["lens"], s["page_table"], s["max_new"], s["max_len"])
    if c["op"] == "walk":
        kept, counts, following = sna.verify_tree(batch, s["sampled"], s["tokens"], s["parents"])
        return {"kept": kept, "counts": counts, "next": following}
    cache = sna.PagedCache(s["k_pages"], s["v_pages"])
    if c["op"] == "compact":
        return {"lens": sna.kv_compact(cache, batch, s["kept"], s["counts"]), "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    return {"out": sna.tree_attention(cache, batch, s["q"], s["masks"], prefix=s["prefix"], positions=s["positions"], window=c["window"])}


# ---- what a pass cannot do without, and what it returns in 64 bits ------------------------------------------------------------
def work(case):
    if case["op"] == "sample":
        n, V = case["rows"], case["vocab"]
        return {"bytes": n * V * ((4 if case["dtype"] == "fp32" else 2) + (4 if case["probs"] else 0)) + 8 * n, "flops": 3 * n * V}
    if case["op"] == "copy":
        return {"bytes": 8 * case["pairs"] * case["kv_heads"] * case["head_dim"] * case["page"], "flops": 0}     # keys and values, read and written
    if case["op"] == "walk":
        sizes = [n for _, n in _steps({**case, "length": case["nodes"]})]
        return {"bytes": 12 * sum(sizes) + 4 * case["seqs"] * (case["nodes"] + 3), "flops": 2 * sum(sizes)}
    steps = _steps(case)
    if case["op"] == "compact":
        moved = sum(max(0, (case["kept"] if not case["ragged"] else max(1, min(case["kept"], n // 2)) / 2 + 0.5) - 1) for _, n in steps)     # the root stays where it is
        return {"bytes": int(8 * moved * case["kv_heads"] * case["head_dim"]) + 8 * len(steps), "flops": 0}
    Hq, Hk, D, e = case["heads"], case["kv_heads"], case["head_dim"], case["earlier"]
    T, W = sum(n for _, n in steps), case["window"] or case["length"]
    keys = sum(min(l - n - e, W) + n + e for l, n in steps)
    pairs = sum(n * (min(l - n - e, W) + math.log2(n + e + 1)) for l, n in steps)
    return {"bytes": 4 * keys * Hk * D + 4 * T * Hq * D + 8 * T * -(-(e + case["nodes"]) // 64), "flops": int(4 * D * Hq * pairs)}


def _exact_tree(s):
    c = s["case"]
    G, D, W = c["heads"] // c["kv_heads"], c["head_dim"], 64 * s["masks"].shape[1]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    row = 0
    for b, (length, n) in enumerate(_steps(c)):
        pages, base = s["page_table"][b, : -(-length // c["page"])].long(), length - n - c["earlier"]
        m = s["masks"][row: row + n]
        bits = (m[:, :, None] >> torch.arange(64, device="cuda") & 1).reshape(n, W)[:, : length - base].bool()
        bits = torch.cat((bits, bits.new_zeros(n, length - base - bits.shape[1])), 1)
        first = s["positions"][row: row + n, None] - (c["window"] or 1 << 30)
        seen = torch.cat((torch.arange(base, device="cuda")[None] > first, bits), 1)
        for h in range(c["kv_heads"]):
            k = s["k_pages"][pages, h].reshape(-1, D)[:length].double()
            v = s["v_pages"][pages, h].transpose(1, 2).reshape(-1, D)[:length].double()
            for g in range(G):
                x = s["q"][row: row + n, h * G + g].double() @ k.t() / math.sqrt(D)
                out[row: row + n, h * G + g] = torch.softmax(x.masked_fill(~seen, -math.inf), 1) @ v
        row += n
    return {"out": out}


def _exact_sample(s):
    n, V = s["logits"].shape
    of = lambda name, i: float(s[name][i]) if torch.is_tensor(s[name]) else float(s[name])  # noqa: E731
    probs = torch.zeros(n, V, dtype=torch.float64, device="cuda")
    for i in range(n):
        t, k, p, m = (of(name, i) for name in ("temperature", "top_k", "top_p", "min_p"))
        x = s["logits"][i].double()
        if t == 0:
            probs[i, int((x == x.max()).nonzero()[0])] = 1
            continue
        values, index = torch.sort(x / t, descending=True, stable=True)
        values, index = (y[: int(k)] if k else y for y in (values, index))
        y = torch.softmax(values, 0)
        least = int((y.cumsum(0) < p).sum()) + 1 if p < 1 else V
        y, index = y[:least], index[:least]
        some = y >= m * y[0]
        probs[i, index[some]] = y[some] / y[some].sum()
    return {"tokens": None, "probs": probs}


def _exact_moved(s, moves):
    """The pools after moves of whole slots: (page, slot) from and to."""
    k, v = s["k_pages"].double(), s["v_pages"].double()
    for (p0, i0), (p1, i1) in moves:
        k[p1, :, i1] = s["k_pages"][p0, :, i0].double()
        v[p1, :, :, i1] = s["v_pages"][p0, :, :, i0].double()
    return k, v


def exact(case, seed):
    if case["op"] == "walk" or case["op"] == "sample" and not case["probs"]:
        return None                                                    # whole numbers
    s = prepare(case, seed)
    if case["op"] == "tree":
        return _exact_tree(s)
    if case["op"] == "sample":
        return _exact_sample(s)
    if case["op"] == "copy":
        k, v = s["k_pages"].double(), s["v_pages"].double()
        for a, b in zip(s["source"].tolist(), s["target"].tolist()):
            k[b], v[b] = s["k_pages"][a].double(), s["v_pages"][a].double()
        return {"k_pages": k, "v_pages": v}
    table, ps, moves = s["page_table"].tolist(), case["page"], []
    for b, ((length, new), (kept, n)) in enumerate(zip(_steps(case), zip(s["kept"].tolist(), s["counts"].tolist()))):
        at = lambda slot: (table[b][slot // ps], slot % ps)  # noqa: E731
        moves += [(at(length - new + kept[i]), at(length - new + i)) for i in range(n)]
    k, v = _exact_moved(s, moves)
    return {"lens": None, "k_pages": k, "v_pages": v}
