"""Speculative decoding on the serving operators: a decoder whose own leading layers draft for it.

    python -m paper_2312_16733_amd.speculate [--drafts 4] [--depth 2] [--seqs 16] [--tokens 128] [--tree 3,2,1] [--samples 2]

The draft is the decoder with LayerSelect applied, its first `depth` layers out of the same resident weights, so that it needs no
weights and no cache of its own: what it appends for those layers is what the full depth would.  A round drafts K tokens one
by one, runs the full depth over them and the token before in one pass, and keeps what verify_draft accepts.  generate_tree drafts
several tokens for a place: level by level the draft's likeliest ones behind each, then one pass over the whole tree, of which the
path that the sampled tokens take is kept.  Weights are random (nothing here is trained), so the share of accepted drafts says
nothing about a real model.
"""
import argparse
import time

import torch

from .serving import (PagedBatch, PagedCache, PagePool, copy_pages, kv_append, kv_compact, paged_attention, sample_tokens, tree_attention, tree_masks, verify_draft,
                      verify_tree)

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
        self.cache = PagedCache(self.k.flatten(1, 2), self.v.flatten(1, 2))              # of all layers at once

    def forward(self, tokens, batch, depth=None, masks=None, prefix=None, positions=None):
        """Logits (fp32) of the step's tokens, through the leading `depth` layers (all).  masks, prefix, positions: of trees, as
        tree_attention takes them."""
        x = self.embed[tokens]
        norm = lambda t: torch.nn.functional.rms_norm(t, (t.shape[-1],), eps=1e-6)  # noqa: E731
        sizes = [n * self.head_dim for n in (self.heads, self.kv_heads, self.kv_heads)]
        for layer, cache in list(zip(self.layers, self.caches))[:depth]:
            q, k, v = (t.unflatten(1, (-1, self.head_dim)) for t in (norm(x) @ layer["qkv"].t()).split(sizes, 1))
            q = kv_append(cache, batch, q, k, v, inv_freq=self.inv_freq, q_norm=layer["q_norm"], k_norm=layer["k_norm"], positions=positions)
            a = paged_attention(cache, batch, q) if masks is None else tree_attention(cache, batch, q, masks, prefix=prefix)
            x = x + a.flatten(1) @ layer["out"].t()
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


def tree_of(widths):
    """Parents of a tree's tokens, level by level: widths[0] children of the root, widths[1] of each of these, ..; and the first token of
    each level, and of the one behind the last."""
    parents, starts = [-1], [0, 1]
    for w in widths:
        parents += [p for p in range(starts[-2], starts[-1]) for _ in range(w)]
        starts.append(len(parents))
    return parents, starts


def generate_tree(model, prompts, n_new, widths=(3, 2, 1), depth=2, samples=1, temperature=1.0, top_k=0, top_p=1.0, seed=0):
    """Continues every prompt (a list of token lists) `samples` times, by at least n_new tokens and at most len(widths) more.  Returns
    (token lists, a prompt's samples behind one another; share of the rounds' places that drafts took; rounds).  The samples of a
    prompt share its pages but for the last."""
    device, N, B = model.device, len(tree_of(widths)[0]), len(prompts) * samples
    g = torch.Generator(device=device).manual_seed(seed)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=device)  # noqa: E731
    pool, cached = PagePool(model.k.shape[0], PAGE), [len(p) - 1 for p in prompts]
    need = [-(-(n + n_new + len(widths) + N) // PAGE) for n in cached]  # a round begins with less than n_new tokens, and brings N

    # the prompts enter the cache but for their last tokens, once each; then their samples part
    pages = [pool.alloc(-(-n // PAGE)) for n in cached]
    if any(cached):
        rows = ints([p + [0] * (max(need) - len(p)) for p in pages])
        model.forward(torch.tensor([t for p in prompts for t in p[:-1]], device=device), PagedBatch(ints([0] + cached).cumsum(0).int(), ints(cached), rows, max(cached), max(cached)))
    mine, source, target = [], [], []
    for n, p, most in zip(cached, pages, need):
        for i in range(samples):
            if i == 0:
                own = list(p)
            else:
                own, a, b = pool.fork(p, n)
                source, target = source + a, target + b
            mine.append(own + pool.alloc(most - len(own)))
    if source:
        copy_pages(model.cache, ints(source), ints(target))

    parents, levels = tree_of(widths)
    masks, depths = tree_masks(parents)
    masks, depths, own_parents = masks.to(device), ints(depths), ints(parents)
    table = ints([p + [0] * (max(need) - len(p)) for p in mine])
    lens, last = ints(cached).repeat_interleave(samples), torch.tensor([p[-1] for p in prompts], device=device).repeat_interleave(samples)
    done, taken, rounds, places = [list(p) for p in prompts for _ in range(samples)], 0, 0, 0
    asked = [len(d) + n_new for d in done]
    at_work = list(range(B)) if n_new > 0 else []                      # lens, last and table hold these sequences
    while at_work:
        B, longest = len(at_work), max(len(done[b]) for b in at_work) - 1
        step = lambda n, slots: PagedBatch(ints(range(0, B * n + 1, n)), lens + slots, table, n, longest + slots)  # noqa: E731
        positions = lens[:, None] + depths
        tokens = last[:, None]
        for i, w in enumerate(widths):                                 # the draft's view of a level, and the next one from it
            a, b = levels[i], levels[i + 1]
            logits = model.forward(tokens[:, a:b].flatten(), step(b - a, b), depth, masks=masks[a:b].repeat(B, 1), prefix=lens, positions=positions[:, a:b].flatten().contiguous())
            tokens = torch.cat((tokens, logits.topk(w, 1).indices.view(B, -1)), 1)
        batch = step(N, N)
        logits = model.forward(tokens.flatten(), batch, masks=masks.repeat(B, 1), positions=positions.flatten())
        drawn = sample_tokens(logits, torch.rand(B * N, generator=g, device=device), temperature=temperature, top_k=top_k, top_p=top_p)
        kept, counts, following = verify_tree(batch, drawn, tokens.flatten(), own_parents.repeat(B))
        lens, last = kv_compact(model.cache, batch, kept, counts), following.long()
        path = tokens.gather(1, kept.clamp(min=0).long())
        for b, row, n, t in zip(at_work, path.tolist(), counts.tolist(), following.tolist()):
            done[b].extend(row[1:n] + [t])
            taken += n - 1
        rounds, places = rounds + 1, places + B * len(widths)
        left = [i for i, b in enumerate(at_work) if len(done[b]) < asked[b]]
        if len(left) < B:
            for i, b in enumerate(at_work):
                if len(done[b]) >= asked[b]:
                    pool.free(mine[b])
            keep = torch.tensor(left, dtype=torch.long, device=device)
            lens, last, table, at_work = lens[keep], last[keep], table[keep], [at_work[i] for i in left]
    return done, taken / max(places, 1), rounds


def main():
    a = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("drafts", 4), ("depth", 2), ("seqs", 16), ("tokens", 128), ("prompt", 100)):
        a.add_argument("--" + name, type=int, default=value)
    a.add_argument("--tree", default="3,2,1", help="tokens drafted behind each of a level, level by level")
    a.add_argument("--samples", type=int, default=1, help="continuations of each prompt, with trees")
    a = a.parse_args()
    widths = [int(w) for w in a.tree.split(",")]
    tree = len(tree_of(widths)[0]) + len(widths)
    model = Decoder(pages=a.seqs * max(1, a.samples) * -(-(a.prompt + a.tokens + max(a.drafts, tree)) // PAGE))
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, model.vocab, (a.prompt - i % 7,), generator=g).tolist() for i in range(a.seqs)]
    runs = [(f"{drafts} drafts", "drafts accepted", 1, lambda n, d=drafts: generate(model, prompts, n, d, a.depth)) for drafts in (0, a.drafts)]
    runs.append((f"trees of {a.tree}", "drafted places taken", a.samples, lambda n: generate_tree(model, prompts, n, widths, a.depth, a.samples, top_p=0.95)))
    for name, what, samples, run in runs:
        run(8)
        torch.cuda.synchronize()
        t = time.perf_counter()
        done, share, rounds = run(a.tokens)
        torch.cuda.synchronize()
        t = time.perf_counter() - t
        n = sum(len(d) - len(prompts[i // samples]) for i, d in enumerate(done))
        print(f"{name}: {n} tokens of {len(done)} sequences in {rounds} rounds, {n / t:.0f} tokens/s, {100 * share:.0f} % of the {what}")


if __name__ == "__main__":
    main()
