"""Attention over scores that differ by many powers of two: a key that takes most of the weight and has no value, and levels that
rise and fall along the keys.  What is left for the others has to keep the element type's precision, however little it is."""
import math

import pytest
import torch

import paper_2312_16733_amd as sna
import paged_reference as ref
from test_gpu_serving import parts, within

pytestmark = pytest.mark.gpu


def attention(s):
    """(result in 64 bits, bound).  A probability is off by half a step of the type; where that would be less than its smallest
    number, by 2^-25 of what stands for one, which is at least half of a tile's largest: over 64 keys less than 2^-18 of that,
    and over all tiles 2^-18 of all weight.  fp32 sums over l keys, scores and exponentials, and the result's own rounding as
    everywhere; sums and products are of the size of the others' weight, but for the sum of probabilities itself."""
    T, H, D = s["q"].shape
    out = torch.zeros(T, H, D, dtype=torch.float64, device="cuda")
    err = torch.zeros_like(out)
    half, row = torch.finfo(s["dtype"]).eps / 2, 0
    for b, (l, n) in enumerate(s["seqs"]):
        k, v = ref.cached(s, b)
        pos, key = torch.arange(l - n, l, device="cuda")[:, None], torch.arange(l, device="cuda")[None]
        for h in range(H):
            q, g = s["q"][row: row + n, h].double(), h * s["kv_heads"] // H
            x = (q @ k[g].t() * D ** -0.5).masked_fill(key > pos, -math.inf)
            off = (q.abs() @ k[g].abs().t() * D ** -0.5).amax(1, keepdim=True) * (D * 2.0 ** -24)
            p = torch.softmax(x, 1)
            out[row: row + n, h] = p @ v[g]
            err[row: row + n, h] = (p @ v[g].abs()) * (half + 2 * off + (l + 64) * 2.0 ** -24) + out[row: row + n, h].abs() * half + 2.0 ** -18 * v[g].abs().amax() * (s["dtype"] == torch.float16) * (1 - p.amax(1, keepdim=True)) + 2.0 ** -25
        row += n
    return out, err * 1.01


def level(s, levels, values=1.0):
    """Every sequence's keys get the given scores (of every query, natural logarithms; a function of position and length) beside small random ones,
    and values of one sign."""
    D = s["dim"]
    s["q"] = torch.randn(s["q"].shape, generator=torch.Generator().manual_seed(2)).to(s["q"]) * 0.1
    s["q"][..., 0] = 16.0
    for b, (l, _) in enumerate(s["seqs"]):
        pos = torch.arange(l, device="cuda")
        page, slot = s["table"][b, pos // s["page"]].long(), pos % s["page"]
        s["k_pages"][page, :, slot, 0] = (levels(pos.double(), l) * D ** 0.5 / 16.0).to(s["dtype"])[:, None]
        s["v_pages"][page, :, :, slot] = values * s["v_pages"][page, :, :, slot].abs()
    return s


def silent(s, where):
    """The value of the key at `where` of each sequence is zero."""
    for b, (l, _) in enumerate(s["seqs"]):
        s["v_pages"][s["table"][b, where(l) // s["page"]].long(), :, :, where(l) % s["page"]] = 0


# few rows whole, few rows shared out, 32 and 64 rows of few tokens, chunks whole and in shares
STEPS = [((4, 4), [(3000, 1), (600, 2)]), ((8, 2), [(32768, 1)]), ((8, 2), [(9000, 5)]), ((16, 2), [(5000, 7)]), ((40, 1), [(3000, 2)]),
         ((8, 1), [(32768, 600)]), ((8, 2), [(6000, 3000)]), ((16, 16), [(480, 93)] * 60)]


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("share", [0.9, 0.99, 0.999])
@pytest.mark.parametrize("heads,seqs", STEPS)
@pytest.mark.parametrize("at", ["first", "middle", "last but the new"])
def test_one_key_that_takes_most_of_the_weight(at, heads, seqs, share, dtype):
    s = ref.make(seqs, *heads, 64 if heads[0] % 3 else 128, 16, ref.DT[dtype], seed=31)
    most = {"first": lambda l: 0, "middle": lambda l: l // 2, "last but the new": lambda l: l - max(n for _, n in seqs) - 1}[at]
    level(s, lambda p, l: torch.where(p == max(most(l), 0), math.log(share / (1 - share) * l), 0.0))
    silent(s, lambda l: max(most(l), 0))
    cache, batch = parts(s)
    want, err = attention(s)
    within(sna.paged_attention(cache, batch, s["q"]), want, err, "out")


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("heads,seqs", STEPS)
@pytest.mark.parametrize("levels", ["down", "up", "up and down", "steps", "far down", "far up and down"])
def test_levels_along_the_keys(levels, heads, seqs, dtype):
    """Weights that fall or rise by factors of up to e^10 over the keys, in waves and in steps; or by e^200, where all but the
    highest level is nothing."""
    of = {"down": lambda p, l: -10 * p / l, "up": lambda p, l: 10 * p / l, "up and down": lambda p, l: 5 * torch.sin(p / 97), "steps": lambda p, l: -3.0 * (p // 300 % 4),
          "far down": lambda p, l: -60.0 * (p // 128 % 4), "far up and down": lambda p, l: 100 * torch.sin(p / 41)}[levels]
    s = ref.make(seqs, *heads, 128 if heads[0] % 3 else 64, 32, ref.DT[dtype], seed=32)
    level(s, of)
    cache, batch = parts(s)
    want, err = attention(s)
    within(sna.paged_attention(cache, batch, s["q"]), want, err, "out")
