"""The loop of generation by trees without a GPU: a decoder and operators that only keep count."""
import pytest
import torch

from paper_2312_16733_amd import serving, speculate

VOCAB = 11


class Counting:
    """Stands for the decoder: uniform logits, and every step's batch and pages checked."""
    device = "cpu"
    cache = None

    def __init__(self, pages):
        self.k = torch.zeros(pages, 1)
        self.owner = {}

    def forward(self, tokens, batch, depth=None, masks=None, prefix=None, positions=None):
        starts, lens, table, max_new, max_len = batch
        serving._validate(starts, lens, table, max_new, max_len, speculate.PAGE, self.k.shape[0], tokens.shape[0])
        written = []
        for b, (n, new) in enumerate(zip(lens.tolist(), (starts[1:] - starts[:-1]).tolist())):
            written += [int(table[b, s // speculate.PAGE]) * speculate.PAGE + s % speculate.PAGE for s in range(n - new, n)]
        assert len(set(written)) == len(written)                       # no two sequences write to one slot
        if masks is not None:
            assert masks.shape[0] == positions.shape[0] == tokens.shape[0]
        return torch.zeros(tokens.shape[0], VOCAB)


def operators(monkeypatch, follow):
    """follow(number of a round, sequence): how many drafts stand."""
    calls = {"rounds": 0, "copied": []}
    monkeypatch.setattr(speculate, "PagedBatch", lambda *a: a)
    monkeypatch.setattr(speculate, "sample_tokens", lambda logits, u, **k: torch.zeros(logits.shape[0], dtype=torch.int32))
    monkeypatch.setattr(speculate, "copy_pages", lambda cache, s, t: calls["copied"].append((s.tolist(), t.tolist())))

    def verify(batch, drawn, tokens, parents):
        starts, lens, table, max_new, max_len = batch
        n = lens.shape[0]
        p = parents[:max_new].tolist()
        kept, counts = [], []
        for b in range(n):
            path = [0]
            for _ in range(follow(calls["rounds"], b)):
                child = [j for j in range(max_new) if p[j] == path[-1]]
                if not child:
                    break
                path.append(child[-1])
            kept.append(path + [-1] * (max_new - len(path)))
            counts.append(len(path))
        calls["rounds"] += 1
        return torch.tensor(kept, dtype=torch.int32), torch.tensor(counts, dtype=torch.int32), torch.full((n,), 7, dtype=torch.int32)
    monkeypatch.setattr(speculate, "verify_tree", verify)
    monkeypatch.setattr(speculate, "kv_compact", lambda cache, batch, kept, counts: batch[1] - batch[3] + counts)
    return calls


def test_the_shape_of_a_tree():
    assert speculate.tree_of((3, 2, 1)) == ([-1, 0, 0, 0, 1, 1, 2, 2, 3, 3, 4, 5, 6, 7, 8, 9], [0, 1, 4, 10, 16])
    assert speculate.tree_of((1, 1)) == ([-1, 0, 1], [0, 1, 2, 3]) and speculate.tree_of(()) == ([-1], [0, 1])


@pytest.mark.parametrize("lengths", [[100] * 4, [1, 17, 40, 33], [5], [16, 32, 33]])
@pytest.mark.parametrize("widths", [(3, 2, 1), (2,), (1, 1, 1, 1, 1), (4, 4)])
@pytest.mark.parametrize("samples,n_new", [(1, 50), (3, 20), (2, 1)])
def test_every_prompt_gets_its_tokens(monkeypatch, lengths, widths, samples, n_new):
    calls = operators(monkeypatch, lambda r, b: (r * 7 + b * 3) % (len(widths) + 1))
    nodes = len(speculate.tree_of(widths)[0])
    pages = sum(-(-(n - 1 + n_new + len(widths) + nodes) // speculate.PAGE) for n in lengths) * samples
    prompts = [[i % VOCAB] * n for i, n in enumerate(lengths)]
    done, share, rounds = speculate.generate_tree(Counting(pages), prompts, n_new, widths, samples=samples)
    assert len(done) == len(prompts) * samples and 0 <= share <= 1 and rounds == calls["rounds"]
    for i, d in enumerate(done):
        p = prompts[i // samples]
        assert d[: len(p)] == p and n_new <= len(d) - len(p) <= n_new + len(widths)
    partial = sum((n - 1) % speculate.PAGE > 0 for n in lengths) * (samples - 1)
    assert sum(len(s) for s, _ in calls["copied"]) == partial          # the last pages of prompts that end inside one
    for s, t in calls["copied"]:
        assert len(set(t)) == len(t) and not set(s) & set(t)


def test_a_pool_that_is_too_small_is_refused(monkeypatch):
    operators(monkeypatch, lambda r, b: 0)
    with pytest.raises(ValueError):
        speculate.generate_tree(Counting(5), [[1] * 40] * 2, 20, (2, 2))
