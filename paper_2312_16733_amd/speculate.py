"""Speculative decoding on the serving operators: a decoder whose own leading layers draft for it.

    python -m paper_2312_16733_amd.speculate [--drafts 4] [--depth 2] [--seqs 16] [--tokens 128]

The draft is the decoder with LayerSelect applied, its first `depth` layers out of the same resident weights, so that it needs no
weights and no cache of its own: what it appends for those layers is what the full depth would.  A round drafts K tokens one
by one, runs the full depth over them and the token before in one pass, and keeps what verify_draft accepts.  Weights are random
(nothing here is trained), so the share of accepted drafts says nothing about a real model.
"""
import argparse
import time

import torch

from .serving import PagedBatch, PagedCache, kv_append, paged_attention, verify_draft

PAGE = 16


class Decoder:
    """Pre-norm decoder, rotated positions, grouped heads with normalised queries and keys, tied embedding; bf16, random weights."""

    def __init__(self, layers=6, hidden=512, heads=8, kv_heads=4, head_dim=64, mlp=1024, vocab=1000, pages=1024, device="cuda:0", seed=0):
        g = torch.Generator().manual_seed(seed)
        draw = lambda n, k: (torch.randn(n, k, generator=g) * k ** -0.5).to(device, torch.bfloat16)  # noqa: E731
        self.heads, self.kv_heads, self.head_dim, self.vocab, self.device = heads, kv_heads, head_dim, vocab, device
        self.embed = (torch.randn(vocab, hidden, generator=g)).to(device, torch.bfloat16)
        self.layers = [{"qkv": draw((heads + 2 * kv_heads) * head_dim, hidden), "out": draw(hidden, heads * head_dim), "up": draw(mlp, hidden), "down": draw(hidden, mlp),
                        "q_norm": torch.ones(head_dim, device=device), "k_norm": torch.ones(head_dim, device=device)} for _ in range(layers)]
        self.inv_freq = (10000.0 ** (-torch.arange(0, head_dim, 2, dtype=torch.float64) / head_dim)).float().to(device)
        # one pool, the layers of a page next to each other
        self.k = torch.zeros(pages, layers, kv_heads, PAGE, head_dim, dtype=torch.bfloat16, device=device)
        self.v = torch.zeros(pages, layers, kv_heads, head_dim, PAGE, dtype=torch.bfloat16, device=device)
        self.caches = [PagedCache(self.k[:, i], self.v[:, i]) for i in range(layers)]

    def forward(self, tokens, batch, depth=None):
        """Logits (fp32) of the step's tokens, through the leading `depth` layers (all)."""
        x = self.embed[tokens]
        norm = lambda t: torch.nn.functional.rms_norm(t, (t.shape[-1],), eps=1e-6)  # noqa: E731
        sizes = [n * self.head_dim for n in (self.heads, self.kv_heads, self.kv_heads)]
        for layer, cache in list(zip(self.layers, self.caches))[:depth]:
            q, k, v = (t.unflatten(1, (-1, self.head_dim)) for t in (norm(x) @ layer["qkv"].t()).split(sizes, 1))
            q = kv_append(cache, batch, q, k, v, inv_freq=self.inv_freq, q_norm=layer["q_norm"], k_norm=layer["k_norm"])
            x = x + paged_attention(cache, batch, q).flatten(1) @ layer["out"].t()
            x = x + torch.nn.functional.gelu(norm(x) @ layer["up"].t()) @ layer["down"].t()
        return (norm(x) @ self.embed.t()).float() * self.embed.shape[1] ** -0.5


def generate(model, prompts, n_new, drafts=4, depth=2, temperature=1.0, seed=0):
    """Continues every prompt (a list of token lists) by at least n_new tokens, and at most `drafts` more.  Returns (token lists, share
    of drafts accepted, rounds).  A sequence that has its tokens leaves the step, so that its pages are bounded whatever the
    others still need."""
    device, B, K = model.device, len(prompts), drafts
    g = torch.Generator(device=device).manual_seed(seed)
    most = max(len(p) for p in prompts) + n_new + K
    width = -(-most // PAGE)
    if B * width > model.k.shape[0]:
        raise ValueError(f"{B} sequences of up to {most} tokens need {B * width} pages, the pool has {model.k.shape[0]}")
    table = torch.arange(B * width, dtype=torch.int32, device=device).view(B, width)
    probs = lambda logits: torch.softmax(logits / temperature, -1)  # noqa: E731
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=device)  # noqa: E731

    # the prompts enter the cache but for their last tokens
    n = [len(p) - 1 for p in prompts]
    if any(n):
        starts = ints([0] + n).cumsum(0).int()
        model.forward(torch.tensor([t for p in prompts for t in p[:-1]], device=device), PagedBatch(starts, ints(n), table, max(n), max(n)))
    lens, last = ints(n), torch.tensor([p[-1] for p in prompts], device=device)
    done, drafted, taken, rounds = [list(p) for p in prompts], 0, 0, 0
    at_work = list(range(B)) if n_new > 0 else []                      # lens, last and table hold these sequences
    while at_work:
        B, longest = len(at_work), max(len(done[b]) for b in at_work) - 1
        one = torch.arange(B + 1, dtype=torch.int32, device=device)
        step, tokens, q = last, [last], []
        for i in range(K):
            q.append(probs(model.forward(step, PagedBatch(one, lens + (i + 1), table, 1, longest + i + 1), depth)))
            step = torch.multinomial(q[-1], 1, generator=g)[:, 0]
            tokens.append(step)
        rows = torch.stack(tokens, 1)
        p = probs(model.forward(rows.flatten(), PagedBatch(one * (K + 1), lens + (K + 1), table, K + 1, longest + K + 1))).view(B, K + 1, -1)
        out, accepted = verify_draft(p, rows[:, 1:].contiguous(), torch.rand(B, K + 1, generator=g, device=device), draft_probs=torch.stack(q, 1) if K else None)
        last = out.gather(1, accepted[:, None].long())[:, 0].long()
        lens = lens + accepted + 1
        for b, row, a in zip(at_work, out.tolist(), accepted.tolist()):
            done[b].extend(row[: a + 1])
            taken += a
        drafted, rounds = drafted + B * K, rounds + 1
        left = [i for i, b in enumerate(at_work) if len(done[b]) - len(prompts[b]) < n_new]
        if len(left) < B:
            kept = torch.tensor(left, dtype=torch.long, device=device)
            lens, last, table, at_work = lens[kept], last[kept], table[kept], [at_work[i] for i in left]
    return done, taken / max(drafted, 1), rounds


def main():
    a = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("drafts", 4), ("depth", 2), ("seqs", 16), ("tokens", 128), ("prompt", 100)):
        a.add_argument("--" + name, type=int, default=value)
    a = a.parse_args()
    model = Decoder(pages=a.seqs * -(-(a.prompt + a.tokens + a.drafts) // PAGE))
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, model.vocab, (a.prompt - i % 7,), generator=g).tolist() for i in range(a.seqs)]
    for drafts in (0, a.drafts):
        generate(model, prompts, 8, drafts, a.depth)
        torch.cuda.synchronize()
        t = time.perf_counter()
        done, share, rounds = generate(model, prompts, a.tokens, drafts, a.depth)
        torch.cuda.synchronize()
        t = time.perf_counter() - t
        n = sum(len(d) - len(p) for d, p in zip(done, prompts))
        print(f"{drafts} drafts: {n} tokens of {a.seqs} sequences in {rounds} rounds, {n / t:.0f} tokens/s, {100 * share:.0f} % of the drafts accepted")


if __name__ == "__main__":
    main()
