"""Trees of drafted tokens for the tests, and attention of their tokens in 64 bits straight from its definition."""
import math
import random

import torch

import paged_reference as ref


def parents(n, seed, chain=False):
    r = random.Random(seed)
    return [i - 1 if chain or i == 0 else r.randint(max(0, i // 3 - 1), i - 1) for i in range(n)]


def ancestors(p):
    """seen[i][j]: token j is i or one that it comes from."""
    seen = torch.eye(len(p), dtype=torch.bool)
    for i in range(1, len(p)):
        seen[i] |= seen[p[i]]
    return seen


def words_of(bits):
    """bool [tokens][any] as int64 [tokens][words]."""
    n, m = bits.shape
    w = max(1, -(-m // 64))
    b = torch.zeros(n, w * 64, dtype=torch.bool)
    b[:, :m] = bits
    b = b.view(n, w, 64)
    value = torch.zeros(n, w, dtype=torch.int64)
    for j in range(64):
        value |= b[:, :, j].long() << j
    return value


def make(seqs, heads, kv_heads, dim, page, dtype, seed=0, earlier=0, kind="tree", words=None, **k):
    """seqs as in paged_reference: (slots after the step, new tokens), of which each tree has `earlier` tokens in the cache before.
    kind: "tree", "chain", "random" masks (rows that see nothing of the tree among them) or "empty" ones."""
    s = ref.make(seqs, heads, kv_heads, dim, page, dtype, seed=seed, **k)
    g = torch.Generator().manual_seed(seed + 1)
    most = earlier + max(n for _, n in seqs)
    masks, pos = [], []
    for b, (l, n) in enumerate(seqs):
        if kind in ("tree", "chain"):
            seen = ancestors(parents(earlier + n, seed * 1000 + b, kind == "chain"))[earlier:]
            depth = seen.sum(1) - 1
        else:
            seen = torch.rand(n, earlier + n, generator=g) < (0.4 if kind == "random" else 0)
            if kind == "random":
                seen[::3] = False
            depth = torch.arange(n)
        m = torch.zeros(n, most, dtype=torch.bool)
        m[:, : seen.shape[1]] = seen
        masks.append(m)
        pos += [max(l - n - earlier, 0) + int(d) for d in depth]
    s["bits"] = masks
    s["masks"] = words_of(torch.cat(masks))
    if words:
        s["masks"] = torch.cat((s["masks"], s["masks"].new_zeros(len(s["masks"]), words - s["masks"].shape[1])), 1)
    s["masks"] = s["masks"].to(s["q"].device)
    s["base"] = [l - n - earlier for l, n in seqs]
    s["prefix"] = torch.tensor(s["base"], dtype=torch.int32, device=s["q"].device) if earlier else None
    s["positions"] = torch.tensor(pos, dtype=torch.int32, device=s["q"].device)
    return s


def seen_of(s, b, window=0):
    """bool [new tokens][slots] of sequence b."""
    (l, n), base = s["seqs"][b], s["base"][b]
    first = sum(m for _, m in s["seqs"][:b])
    seen = torch.zeros(n, l, dtype=torch.bool)
    pos = s["positions"][first: first + n].cpu()[:, None]
    seen[:, :base] = torch.arange(base)[None] > (pos - window if window else -1)
    m = s["bits"][b][:, : l - base]
    seen[:, base: base + m.shape[1]] = m
    return seen.to(s["q"].device)


def attention(s, window=0, scale=None):
    """(result, bound on the error), as paged_reference.attention gives them."""
    T, H, D = s["q"].shape
    G = H // s["kv_heads"]
    scale = D ** -0.5 if scale is None else scale
    out = torch.zeros(T, H, D, dtype=torch.float64, device=s["q"].device)
    err = torch.zeros_like(out)
    half = torch.finfo(s["dtype"]).eps / 2
    row = 0
    for b, (l, n) in enumerate(s["seqs"]):
        if n == 0:
            continue
        k, v = ref.cached(s, b)
        seen = seen_of(s, b, window)
        none = ~seen.any(1, keepdim=True)
        for h in range(H):
            q = s["q"][row: row + n, h].double()
            x = (q @ k[h // G].t() * scale).masked_fill(~seen, -math.inf)
            off = (q.abs() @ k[h // G].abs().t() * abs(scale)).masked_fill(~seen, 0).amax(1, keepdim=True) * (D * 2.0 ** -24)   # of a score, in fp32
            p = torch.softmax(x, 1).masked_fill(none, 0)
            size = p @ v[h // G].abs()
            out[row: row + n, h] = p @ v[h // G]
            # as for the causal form: probabilities and the result rounded, scores and sums in fp32, small fp16 probabilities
            e = size * (half + 2 * off + (l + 64) * 2.0 ** -24) + out[row: row + n, h].abs() * half
            if s["dtype"] == torch.float16:
                e = e + l * 2.0 ** -25 * v[h // G].abs().amax() + 2.0 ** -25
            err[row: row + n, h] = (e * 1.01 + 1e-30).masked_fill(none, 0)
        row += n
    return out, err
