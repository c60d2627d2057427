"""Paged caches for the tests, and the serving operators in 64 bits straight from their definitions."""
import math

import torch

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


def make(seqs, heads, kv_heads, dim, page, dtype, seed=0, device="cuda", spare=3, layers=1, fill=float("nan"), junk=True, at_end=False):
    """seqs: (length after the step, new tokens).  Slots behind a sequence's tokens hold `fill`, as do pages of nobody and the
    pool's other layers; table entries behind a sequence's last page name no page where `junk`."""
    g = torch.Generator().manual_seed(seed)
    used = [-(-l // page) for l, _ in seqs]
    n = sum(used) + spare
    order = torch.randperm(n, generator=g).tolist()
    width = max(max(used), 1) + 2
    table = torch.full((len(seqs), width), 0, dtype=torch.int32)
    if junk:
        table[:] = torch.tensor([-1, 2 ** 31 - 1, -2 ** 31, n], dtype=torch.int32).repeat(len(seqs) * width // 4 + 1)[: len(seqs) * width].view(len(seqs), width)
    kp = torch.full((n, layers, kv_heads, page, dim), fill, dtype=dtype)
    vp = torch.full((n, layers, kv_heads, dim, page), fill, dtype=dtype)
    at = 0
    layer = layers - 1
    for b, (l, _) in enumerate(seqs):
        ids = order[at: at + used[b]]
        at += used[b]
        table[b, : used[b]] = torch.tensor(ids, dtype=torch.int32)
        k, v = (torch.randn(kv_heads, l, dim, generator=g).to(dtype) for _ in range(2))
        for j, p in enumerate(ids):
            m = min(page, l - j * page)
            kp[p, layer, :, :m] = k[:, j * page: j * page + m]
            vp[p, layer, :, :, :m] = v[:, j * page: j * page + m].transpose(1, 2)
    starts = torch.tensor([0] + [m for _, m in seqs]).cumsum(0).int()
    tokens = int(starts[-1])
    s = {"seqs": seqs, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype, "n_pages": n,
         "starts": starts.to(device), "lens": torch.tensor([l for l, _ in seqs], dtype=torch.int32, device=device), "table": table.to(device),
         "k_pages": kp.to(device)[:, layer], "v_pages": vp.to(device)[:, layer], "max_new": max(max(m for _, m in seqs), 1), "max_len": max(l for l, _ in seqs)}
    qkv = torch.randn(tokens, (heads + 2 * kv_heads) * dim, generator=g).to(dtype).to(device)
    s["q"], s["k"], s["v"] = (x.unflatten(1, (-1, dim)) for x in qkv.split([heads * dim, kv_heads * dim, kv_heads * dim], 1))
    return s


def cached(s, b):
    """Keys and values [kv_heads][length][dim] of sequence b as the pages hold them, in 64 bits."""
    l = s["seqs"][b][0]
    ids = s["table"][b, : -(-l // s["page"])].long()
    k = s["k_pages"][ids].permute(1, 0, 2, 3).reshape(s["kv_heads"], -1, s["dim"])[:, :l].double()
    v = s["v_pages"][ids].permute(1, 0, 3, 2).reshape(s["kv_heads"], -1, s["dim"])[:, :l].double()
    return k, v


def attention(s, window=0, scale=None):
    """(result, bound on the error of a kernel that rounds the probabilities and the result to the type and keeps the rest in fp32)."""
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
        k, v = cached(s, b)
        pos = torch.arange(l - n, l, device=k.device)[:, None]
        key = torch.arange(l, device=k.device)[None]
        seen = (key <= pos) & ((key > pos - window) if window else True)
        for h in range(H):
            q = s["q"][row: row + n, h].double()
            x = q @ k[h // G].t() * scale
            off = (q.abs() @ k[h // G].abs().t() * abs(scale)).masked_fill(~seen, 0).amax(1, keepdim=True) * (D * 2.0 ** -24)   # of a score, in fp32
            p = torch.softmax(x.masked_fill(~seen, -math.inf), 1)
            size = p @ v[h // G].abs()
            out[row: row + n, h] = p @ v[h // G]
            # probabilities: half a step, the score's error twice (numerator, sum), a few steps of exp2 and its argument, sums
            # over l keys; below 2^-14 an fp16 probability (relative to the largest) is off by up to 2^-25 instead
            e = size * (half + 2 * off + (l + 64) * 2.0 ** -24) + out[row: row + n, h].abs() * half
            if s["dtype"] == torch.float16:
                e = e + l * 2.0 ** -25 * v[h // G].abs().amax() + 2.0 ** -25
            err[row: row + n, h] = e * 1.01 + 1e-30                   # terms of second order
        row += n
    return out, err


def append(s, inv_freq=None, interleaved=False, q_norm=None, k_norm=None, eps=1e-6):
    """q, k, v [tokens][heads][dim] in 64 bits and the bounds on the errors of q and k."""
    half = torch.finfo(s["dtype"]).eps / 2
    pos = torch.cat([torch.arange(l - n, l) for l, n in s["seqs"]]).to(s["q"].device).double()
    res = []
    for x, w in ((s["q"], q_norm), (s["k"], k_norm)):
        x = x.double()
        if w is not None:
            x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()
        size = x.abs().clone()
        y = x.clone()
        if inv_freq is not None:
            m = inv_freq.numel()
            a = pos[:, None, None] * inv_freq.double()
            i = torch.arange(m, device=x.device)
            ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + m)
            y[..., ia] = x[..., ia] * a.cos() - x[..., ib] * a.sin()
            y[..., ib] = x[..., ia] * a.sin() + x[..., ib] * a.cos()
            size[..., ia] = size[..., ib] = x[..., ia].abs() + x[..., ib].abs()
        # one rounding; before it fp32: a norm (sum of up to 128 squares, root, two products), sin and cos to a few steps
        res.append((y, y.abs() * half + size * (160 * 2.0 ** -24) + (2.0 ** -25 if s["dtype"] == torch.float16 else 0)))
    return res[0], res[1], s["v"]
