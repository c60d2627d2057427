"""Attention of drafted trees in each of its launches (what test_tree_plan_host.py finds the steps to be launched as), in both types."""
import pytest
import torch

import paper_2312_16733_amd as sna
import paged_reference as ref
import tree_launches as launches
import tree_reference as tree
from test_gpu_serving import parts

pytestmark = [pytest.mark.gpu, pytest.mark.parametrize("dtype", ["bf16", "fp16"])]
each = pytest.mark.parametrize("launch,several,dim,step", launches.STEPS)


def attend(s, step, **k):
    return sna.tree_attention(*parts(s), s["q"], s["masks"], prefix=s["prefix"], positions=s["positions"], window=step[7], **k)


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
