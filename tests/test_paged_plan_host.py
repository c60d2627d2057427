"""Which launch a step of paged attention gets (csrc/paged_plan.h, plain host code), and that every launch is reached by a case of
the GPU tests."""
import os
import random
import subprocess

import pytest

from paged_launches import STEPS, seqs

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DRIVER = r"""
#include "paged_plan.h"
#include <cstdio>
using namespace sna;
int main() {
  int b, t, h, g, n, l, w, d;
  while (scanf("%d %d %d %d %d %d %d %d", &b, &t, &h, &g, &n, &l, &w, &d) == 8) {
    const AttnPlan p = plan_of(b, t, h, g, n, l, w, d);
    printf("%d %d %d %d %d %d %d %zu %zu\n", p.mb, p.blocks, p.waves, p.most, (int)p.chunks, p.chunk.waves, p.chunk.splits, p.parts, p.chunk_parts);
  }
}
"""


@pytest.fixture(scope="session")
def plans(tmp_path_factory):
    """A function from steps (head size, (heads, kv_heads, ..., window) of paged_launches) to the launches they get, and whether rows are more than a block's."""
    d = tmp_path_factory.mktemp("plan")
    (d / "d.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(ROOT, "paper_2312_16733_amd", "csrc"), str(d / "d.cpp"), "-o", str(d / "d")], check=True)

    def of(steps):
        lines, most = [], []
        for dim, (h, k, length, new, n, ragged, singles, window) in steps:
            q = seqs(length, new, n, ragged, singles)
            lines.append(f"{len(q)} {sum(m for _, m in q)} {k} {h // k} {max(m for _, m in q)} {max(l for l, _ in q)} {window} {dim}")
            most.append(max(m for _, m in q) * (h // k))
        out = subprocess.run([str(d / "d")], input="\n".join(lines), capture_output=True, text=True, check=True).stdout.splitlines()
        got = []
        for line, rows in zip(out, most):
            mb, blocks, waves, _, chunks, cw, cs, parts, chunk_parts = map(int, line.split())
            few = [f"{16 * mb} rows, shared" if blocks else f"{16 * mb} rows, {waves} waves"] if mb else []
            many = [f"{32 * cw}-row chunks" + (", shared" if cs > 1 else "")] if chunks else []
            assert (parts > 0) == (blocks > 0) and (chunk_parts > 0) == (chunks and cs > 1)
            got.append((tuple(many + few), rows > (32 * cw if chunks else 16 * mb)))
        return got
    return of


def test_steps_get_the_launches_that_they_are_named_for(plans):
    assert len({(launch, several, dim) for launch, several, dim, _ in STEPS}) == len(STEPS)
    for (launch, several, dim, step), got in zip(STEPS, plans([(dim, step) for _, _, dim, step in STEPS])):
        assert got == (launch, several), (dim, step)


def test_there_is_no_other_launch(plans):
    """Whatever the step (20000 at random over heads, lengths, chunks and windows), its launch is one of those."""
    rng = random.Random(7)
    log = lambda lo, hi: round(lo * (hi / lo) ** rng.random())  # noqa: E731
    steps = []
    while len(steps) < 20000:
        heads, kv = rng.choice([(12, 12), (16, 4), (8, 1), (9, 3), (32, 8), (16, 2), (16, 16), (7, 1), (8, 2), (40, 1), (20, 2), (40, 2), (64, 1), (2, 1), (1, 1)])
        length = log(1, 100000)
        new, n = log(1, min(length, 4096)), log(1, 200)
        steps.append((rng.choice([64, 128]), (heads, kv, length, new, n, rng.choice([0, 1]), rng.choice([0, 0, 1, 7, 200]), rng.choice([0, 0, log(1, length)]))))
    known = {(launch, several, dim) for launch, several, dim, _ in STEPS}
    for (dim, step), (launch, several) in zip(steps, plans(steps)):
        assert (launch, several, dim) in known, (dim, step)
