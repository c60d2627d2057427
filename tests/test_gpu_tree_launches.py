"""Attention of drafted trees in each of its launches (what test_tree_plan_host.py finds the steps to be launched as), in both types."""
import pytest
import torch

import paper_2312_16733_amd as sna
import paged_reference as ref
import tree_launches as launches
import tree_reference as tree
from test_gpu_serving import parts, within

pytestmark = [pytest.mark.gpu, pytest.mark.parametrize("dtype", ["bf16", "fp16"])]
each = pytest.mark.parametrize("launch,several,dim,step", launches.STEPS)


def attend(s, step, **k):
    return sna.tree_attention(*parts(s), s["q"], s["masks"], prefix=s["prefix"], positions=s["positions"], window=step[7], **k)


@each
def test_masks_of_any_bits(launch, several, dim, step, dtype):
    """Unused slots and the workspace full of NaN; the same bits each time."""
    s = launches.make(dim, step, dtype, seed=41, kind="random")
    want, err = tree.attention(s, step[7])
    out = attend(s, step, workspace=torch.full((256 << 20,), 255, dtype=torch.uint8, device="cuda"))
    within(out, want, err, launch)
    assert torch.equal(attend(s, step), out)


@each
def test_tokens_are_off_by_their_own_rounding(launch, several, dim, step, dtype):
    """Whatever else its step brings: the error is that of rounding the 64-bit result once.  fp32 scores and sums are off by a few
    hundred steps of 2^-24 at most, less than a hundredth of half a step of either type in the norm; a tenth is allowed."""
    s = launches.make(dim, step, dtype, seed=42)
    want, _ = tree.attention(s, step[7])
    off = (attend(s, step).double() - want).norm()
    own = (want.to(ref.DT[dtype]).double() - want).norm()
    print(f"{launch}: {float(off / own):.3f} of the result's own rounding", flush=True)
    assert off <= 1.1 * own


@each
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_no_number_reaches_a_token_that_does_not_see_it(launch, several, dim, step, dtype, bad):
    s = launches.make(dim, step, dtype, seed=43, kind="random")
    want, err = tree.attention(s, step[7])
    hit = torch.zeros(s["q"].shape[0], dtype=torch.bool, device="cuda")
    row = 0
    for b, (l, n) in enumerate(s["seqs"]):
        slot = l - n + n // 2
        page = int(s["table"][b, slot // 16])
        s["v_pages"][page, :, :, slot % 16] = bad
        if b == 0:
            s["k_pages"][page, :, slot % 16] = bad
        hit[row: row + n] = tree.seen_of(s, b, step[7])[:, slot]
        row += n
    out = attend(s, step)
    assert not hit.all()
    within(out[~hit], want[~hit], err[~hit], launch)
    if hit.any():
        assert not torch.isfinite(out[hit].float()).any()


@each
def test_bits_behind_the_last_slot_name_nothing(launch, several, dim, step, dtype):
    s = launches.make(dim, step, dtype, seed=44, words=-(-max(n for _, n in launches.seqs(*step[2:7])) // 64) + (0 if step[7] else 2))
    s["masks"].fill_(-1)
    s["bits"] = [torch.ones(n, s["masks"].shape[1] * 64, dtype=torch.bool) for _, n in s["seqs"]]
    want, err = tree.attention(s, step[7])
    within(attend(s, step), want, err, launch)


@each
def test_arrays_that_do_not_fit(launch, several, dim, step, dtype):
    """Pages that are none, lengths of any value, prefixes, positions and masks likewise: whatever comes back for those sequences, the
    last one is right."""
    s = launches.make(dim, step, dtype, seed=45)
    n = s["seqs"][-1][1]
    want, err = (x[-n:] for x in tree.attention(s, step[7]))
    others = len(s["seqs"]) - 1
    s["prefix"] = torch.tensor(s["base"], dtype=torch.int32, device="cuda")
    kept = {name: s[name].clone() for name in ("prefix", "positions", "masks", "table", "lens")}
    for name, values in (("prefix", [-5, 2 ** 31 - 1, -2 ** 31, 17]), ("lens", [10 ** 9, -7, 0, 3]), ("table", [-5, 2 ** 31 - 1]), ("positions", [2 ** 31 - 1, -2 ** 31, -1]), ("masks", [-1, 0])):
        for value in values:
            for x, y in kept.items():
                s[x].copy_(y)
            s[name][: -n if name in ("positions", "masks") else others] = value
            out = attend(s, step)
            within(out[-n:], want, err, f"{launch}, {name} {value}")


@each
@pytest.mark.parametrize("levels", [(0, 6, -9, 12, 3, 9, -3, 12, 10), (0, 40, -40, 12, 80, -80, 20, 0, 60)])
def test_scores_that_differ_from_share_to_share(launch, several, dim, step, dtype, levels):
    """Runs of keys whose scores lie a few powers of two apart, or dozens, rising and falling: what the exponentials are relative to
    moves within a share, and differs between the parts that are joined."""
    s = launches.make(dim, step, dtype, seed=46)
    s["q"][..., 0] = 4
    for b, (l, _) in enumerate(s["seqs"]):
        ids = s["table"][b, : -(-l // 16)].long()
        run = max(l // len(levels), 1)
        of = torch.tensor(levels, dtype=s["dtype"], device="cuda")[(torch.arange(len(ids) * 16, device="cuda") // run).clamp(max=len(levels) - 1)]
        s["k_pages"][ids, :, :, 0] = of.view(len(ids), 1, 16).expand(-1, s["kv_heads"], -1)
    want, err = tree.attention(s, step[7])
    within(attend(s, step), want, err, launch)
