"""Generation by trees of drafted tokens through the paged cache against the same decoder run whole, without a cache."""
import pytest
import torch

from test_gpu_speculate import whole

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("widths,depth,samples", [((3, 2, 1), 2, 1), ((2,), 1, 3), ((4, 3, 2, 1), 4, 2), ((1, 1, 1, 1), 4, 1)])
def test_tokens_are_the_decoders(widths, depth, samples):
    """At temperature 0 every token is the whole decoder's first choice, whatever was drafted and wherever it was moved to, up to what
    bf16 leaves open between the first two: activations are rounded about ten times a layer, each by 2^-9 of their size on
    average, and ride on a residual of the size of the logits' norm; 0.15 is five times that for logits of deviation 1."""
    from paper_2312_16733_amd.speculate import Decoder, generate_tree
    model = Decoder(layers=4, hidden=256, heads=4, kv_heads=2, mlp=512, vocab=500, pages=160, seed=3)
    g = torch.Generator().manual_seed(5)
    prompts = [torch.randint(0, model.vocab, (n,), generator=g).tolist() for n in (1, 17, 40, 33)]
    done, share, rounds = generate_tree(model, prompts, 24, widths, depth, samples, temperature=0.0)
    print(f"{widths} at depth {depth}: {100 * share:.0f} % taken in {rounds} rounds", flush=True)
    assert len(done) == len(prompts) * samples
    for i, d in enumerate(done):
        p = prompts[i // samples]
        assert d[: len(p)] == p and len(p) + 24 <= len(d) <= len(p) + 24 + len(widths)
        logits = whole(model, d)
        for j in range(len(p), len(d)):
            assert logits[j - 1, d[j]] >= logits[j - 1].max() - 0.15, (j, float(logits[j - 1, d[j]]), float(logits[j - 1].max()))
    if depth == 4:                                                     # the draft is the decoder itself, and its first choice among its drafts
        assert share > 0.8 and rounds < 24


def test_samples_follow_the_decoders_probabilities():
    """At temperature 1 the first sampled token of many continuations has the decoder's own distribution: the share of the tokens that
    it gives half of the probability to is within five deviations."""
    from paper_2312_16733_amd.speculate import Decoder, generate_tree
    model = Decoder(layers=2, hidden=128, heads=2, kv_heads=2, mlp=128, vocab=60, pages=1200, seed=4)
    prompt, n = [5, 9, 33, 2], 400
    done, _, _ = generate_tree(model, [prompt], 1, (3, 2), 1, n, seed=11)
    p = torch.softmax(whole(model, prompt)[-1], 0).cpu()
    order = p.argsort(descending=True)
    half = order[: int((p[order].cumsum(0) < 0.5).sum()) + 1]
    want, got = float(p[half].sum()), sum(d[len(prompt)] in half.tolist() for d in done) / n
    print(f"{got:.3f} of the samples, probability {want:.3f}", flush=True)
    assert abs(got - want) < 5 * (want * (1 - want) / n) ** 0.5 + 0.02     # bf16 moves single probabilities by a few percent of themselves


def test_a_pool_too_small_is_refused():
    from paper_2312_16733_amd.speculate import Decoder, generate_tree
    model = Decoder(layers=1, hidden=64, heads=1, kv_heads=1, mlp=64, vocab=50, pages=3)
    with pytest.raises(ValueError):
        generate_tree(model, [[1, 2]] * 2, 100)
