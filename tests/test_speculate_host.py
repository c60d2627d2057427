"""The loop of speculative decoding without a GPU: a decoder and a verification that only keep count."""
import pytest
import torch

from paper_2312_16733_amd import serving, speculate

VOCAB = 7


class Counting:
    """Stands for the decoder: uniform logits, and every step's batch checked as PagedBatch.validate does."""
    device = "cpu"

    def __init__(self, pages):
        self.k = torch.zeros(pages, 1)
        self.rows = 0

    def forward(self, tokens, batch, depth=None):
        starts, lens, table, max_new, max_len = batch
        serving._validate(starts, lens, table, max_new, max_len, speculate.PAGE, self.k.shape[0], tokens.shape[0])
        used = [table[b, : -(-int(n) // speculate.PAGE)].tolist() for b, n in enumerate(lens)]
        assert len({p for u in used for p in u}) == sum(len(u) for u in used)                       # nobody's page is another's
        self.rows += tokens.shape[0]
        return torch.zeros(tokens.shape[0], VOCAB)


def accepting(share, seed):
    """Stands for verify_draft: every draft stands with the same chance, whatever it is."""
    g = torch.Generator().manual_seed(seed)

    def verify(target, tokens, uniforms, draft_probs=None, n_draft=None):
        n, K = tokens.shape
        accepted = (torch.rand(n, K, generator=g) < share).long().cumprod(1).sum(1).int()
        place = torch.arange(K + 1)
        out = torch.where(place < accepted[:, None], torch.cat((tokens, tokens[:, :1]), 1) if K else tokens.new_zeros(n, 1), -1)
        return torch.where(place == accepted[:, None], VOCAB - 1, out).int(), accepted
    return verify


@pytest.mark.parametrize("lengths", [[100] * 16, [1, 17, 40, 33], [5]])
@pytest.mark.parametrize("share", [0.0, 0.3, 0.5, 0.8, 1.0])
@pytest.mark.parametrize("drafts,n_new", [(4, 128), (1, 16), (7, 50), (0, 10)])
def test_every_prompt_gets_its_tokens(monkeypatch, lengths, share, drafts, n_new):
    """However unequal the luck of the sequences, each gets n_new tokens and at most one round's more, within a pool that holds
    just these."""
    monkeypatch.setattr(speculate, "PagedBatch", lambda *a: a)
    monkeypatch.setattr(speculate, "verify_draft", accepting(share, 3))
    width = -(-(max(lengths) + n_new + drafts) // speculate.PAGE)
    model = Counting(len(lengths) * width)
    prompts = [[i % VOCAB] * n for i, n in enumerate(lengths)]
    done, taken, rounds = speculate.generate(model, prompts, n_new, drafts)
    for p, d in zip(prompts, done):
        assert d[: len(p)] == p
        assert n_new <= len(d) - len(p) <= n_new + drafts
    assert taken == share if share in (0.0, 1.0) and drafts else 0 <= taken <= 1
    assert rounds >= -(-n_new // (drafts + 1))


def test_sequences_that_have_their_tokens_bring_none(monkeypatch):
    """A sequence whose drafts all stand is done after a quarter of the rounds of one whose never do, and costs no more rows."""
    monkeypatch.setattr(speculate, "PagedBatch", lambda *a: a)

    def verify(target, tokens, uniforms, draft_probs=None, n_draft=None):
        accepted = torch.where(tokens[:, 0] >= 0, verify.accepted[-tokens.shape[0]:], 0).int()       # the lucky one leaves first
        out = torch.where(torch.arange(4) < accepted[:, None], torch.cat((tokens, tokens[:, :1]), 1), -1)
        return torch.where(torch.arange(4) == accepted[:, None], 1, out).int(), accepted
    verify.accepted = torch.tensor([3, 0])
    monkeypatch.setattr(speculate, "verify_draft", verify)
    model = Counting(2 * 4)
    done, share, rounds = speculate.generate(model, [[1, 2], [3, 4]], 40, 3)
    assert [len(d) for d in done] == [42, 42] and rounds == 40
    # the prompts, then 3 drafts and 4 verified rows a sequence and round: 10 rounds of two sequences, 30 of one
    assert model.rows == 2 + 7 * (2 * 10 + 30) and share == pytest.approx(30 / (3 * (2 * 10 + 30)))


def test_a_pool_that_holds_one_page_less_is_refused(monkeypatch):
    monkeypatch.setattr(speculate, "PagedBatch", lambda *a: a)
    monkeypatch.setattr(speculate, "verify_draft", accepting(0.5, 1))
    with pytest.raises(ValueError):
        speculate.generate(Counting(3), [[1] * 40], 20, 4)
    assert len(speculate.generate(Counting(4), [[1] * 40], 20, 4)[0][0]) >= 60
