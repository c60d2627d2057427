"""Steps of attention over drafted trees that get each launch there is, at both head sizes."""
import paged_reference as ref
import tree_reference as tree
from paged_launches import seqs

# As in paged_launches: launch, whether a sequence's rows are more than a block's, head size, (heads, key / value heads, length, new tokens,
# sequences, ragged, single tokens, window).  "128 rows": blocks of the many-rows kernel; "looked for": the blocks of the join look for what
# was begun; "few": fewer shares of the keys than there are XCDs
STEPS = [
    ("16 rows, 4 waves", False, 64, (12, 12, 300, 5, 2, 1, 1, 0)),
    ("16 rows, 4 waves", False, 128, (8, 2, 200, 4, 2, 1, 1, 60)),
    ("16 rows, 8 waves", False, 64, (16, 4, 700, 4, 3, 1, 1, 0)),
    ("16 rows, 8 waves", False, 128, (16, 2, 593, 2, 8, 0, 1, 0)),
    ("16 rows, shared", False, 64, (16, 4, 2600, 4, 2, 1, 1, 0)),
    ("16 rows, shared", False, 128, (8, 1, 900, 2, 2, 1, 0, 0)),
    ("32 rows, 4 waves", False, 64, (8, 1, 90, 4, 3, 1, 1, 0)),
    ("32 rows, 4 waves", False, 128, (7, 1, 120, 4, 2, 1, 1, 30)),
    ("32 rows, 4 waves", True, 64, (16, 4, 300, 70, 2, 1, 1, 0)),
    ("32 rows, 4 waves", True, 128, (8, 2, 260, 60, 2, 1, 1, 0)),
    ("32 rows, 8 waves", False, 64, (7, 1, 769, 3, 2, 1, 1, 0)),
    ("32 rows, 8 waves", False, 128, (2, 1, 525, 12, 17, 1, 7, 0)),
    ("32 rows, 8 waves", True, 64, (12, 12, 667, 40, 1, 0, 0, 0)),
    ("32 rows, 8 waves", True, 128, (2, 1, 516, 19, 1, 1, 0, 0)),
    ("32 rows, shared", False, 64, (8, 1, 1300, 3, 2, 1, 1, 0)),
    ("32 rows, shared", False, 128, (8, 1, 900, 3, 2, 1, 1, 0)),
    ("32 rows, shared", True, 64, (2, 1, 5152, 17, 1, 1, 1, 0)),
    ("32 rows, shared", True, 128, (8, 2, 3502, 9, 2, 1, 1, 0)),
    ("128 rows", False, 64, (16, 16, 700, 100, 9, 1, 1, 0)),
    ("128 rows", False, 128, (32, 8, 500, 30, 40, 1, 2, 0)),
    ("128 rows", True, 64, (16, 4, 900, 120, 24, 1, 1, 300)),
    ("128 rows", True, 128, (8, 2, 700, 150, 14, 1, 1, 0)),
    ("128 rows", True, 128, (40, 1, 90, 17, 2, 1, 1, 0)),
    ("128 rows, shared", False, 64, (16, 4, 2329, 24, 12, 1, 7, 0)),
    ("128 rows, shared", False, 128, (16, 4, 2556, 22, 16, 1, 1, 0)),
    ("128 rows, shared", True, 64, (7, 1, 1993, 608, 1, 0, 1, 0)),
    ("128 rows, shared", True, 128, (40, 1, 1672, 37, 1, 1, 7, 0)),
    ("128 rows, shared, looked for", False, 64, (40, 1, 2119, 3, 1, 0, 1, 0)),
    ("128 rows, shared, looked for", False, 128, (64, 1, 2084, 1, 2, 1, 0, 0)),
    ("128 rows, shared, looked for", True, 64, (8, 2, 7555, 90, 2, 1, 0, 0)),
    ("128 rows, shared, looked for", True, 128, (32, 8, 6001, 77, 1, 0, 0, 0)),
    ("128 rows, shared, few", True, 64, (8, 1, 2166, 1193, 1, 0, 0, 0)),
    ("128 rows, shared, few", True, 128, (64, 1, 1400, 149, 1, 1, 0, 0)),
]


def make(dim, step, dtype, seed, **k):
    """As tree_reference.make."""
    heads, kv_heads, length, new, n, ragged, singles, _ = step
    return tree.make(seqs(length, new, n, ragged, singles), heads, kv_heads, dim, 16, ref.DT[dtype], seed=seed, **k)
