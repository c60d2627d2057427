"""Speculative decoding through the paged cache against the same decoder run whole, without a cache."""
import pytest
import torch

from paged_reference import DT  # noqa: F401  (the tests' folder is importable)

pytestmark = pytest.mark.gpu


def whole(model, tokens):
    """Logits of every position of one sequence in 64 bits, from the decoder's definition."""
    x = model.embed[torch.tensor(tokens, device=model.device)].double()
    norm = lambda t: t / (t.square().mean(-1, keepdim=True) + 1e-6).sqrt()  # noqa: E731
    n, D = len(tokens), model.head_dim
    a = torch.arange(n, device=x.device).double()[:, None, None] * model.inv_freq.double()
    hidden = torch.ones(n, n, dtype=torch.bool, device=x.device).triu(1)

    def rotated(t):
        t = norm(t)
        u, v = t[..., : D // 2], t[..., D // 2:]
        return torch.cat((u * a.cos() - v * a.sin(), u * a.sin() + v * a.cos()), -1)

    for w in model.layers:
        q, k, v = (norm(x) @ w["qkv"].double().t()).unflatten(1, (-1, D)).split([model.heads, model.kv_heads, model.kv_heads], 1)
        q, k = rotated(q), rotated(k)
        heads = [torch.softmax((q[:, h] @ k[:, h * model.kv_heads // model.heads].t() * D ** -0.5).masked_fill(hidden, -torch.inf), 1) @ v[:, h * model.kv_heads // model.heads]
                 for h in range(model.heads)]
        x = x + torch.cat(heads, 1) @ w["out"].double().t()
        x = x + torch.nn.functional.gelu(norm(x) @ w["up"].double().t()) @ w["down"].double().t()
    return norm(x) @ model.embed.double().t() * model.embed.shape[1] ** -0.5


@pytest.mark.parametrize("drafts,depth", [(0, None), (3, 2), (5, 4)])
def test_tokens_are_the_decoders(drafts, depth):
    """At a temperature next to zero every token is the whole decoder's first choice, whatever was drafted, up to what bf16 leaves
    open between the first two: activations are rounded about ten times a layer, each by 2^-9 of their size on average, and
    ride on a residual of the size of the logits' norm; 0.15 is five times that for logits of deviation 1."""
    from paper_2312_16733_amd.speculate import Decoder, generate
    model = Decoder(layers=4, hidden=256, heads=4, kv_heads=2, mlp=512, vocab=500, pages=64, seed=3)
    g = torch.Generator().manual_seed(5)
    prompts = [torch.randint(0, model.vocab, (n,), generator=g).tolist() for n in (1, 17, 40, 33)]
    done, share, rounds = generate(model, prompts, 24, drafts, depth, temperature=1e-3)
    print(f"{drafts} drafts at depth {depth}: {100 * share:.0f} % accepted in {rounds} rounds", flush=True)
    for p, d in zip(prompts, done):
        assert d[: len(p)] == p and len(d) >= len(p) + 24
        logits = whole(model, d)
        for i in range(len(p), len(d)):
            assert logits[i - 1, d[i]] >= logits[i - 1].max() - 0.15, (i, float(logits[i - 1, d[i]]), float(logits[i - 1].max()))
    if depth == 4:                                                     # the draft is the decoder itself
        assert share > 0.8 and rounds < 24


def test_a_pool_too_small_is_refused():
    from paper_2312_16733_amd.speculate import Decoder, generate
    model = Decoder(layers=1, hidden=64, heads=1, kv_heads=1, mlp=64, vocab=50, pages=3)
    with pytest.raises(ValueError):
        generate(model, [[1, 2]] * 2, 100)
