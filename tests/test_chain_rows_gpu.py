"""gdn_chain with packed tables that go backwards: a sequence that would take rows
of one before it is reported and left alone, the others are as ever (tolerances:
tests/test_chain_gpu.py)."""
import numpy as np
import pytest

from tests.chain_ref import Chain
from tests.test_chain_gpu import check


@pytest.fixture(scope="module")
def L():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_06763_amd import gdn_layer as L
    return L


# table, T, rows, sequences that are reported
TABLES = [
    ([0, 10, 5, 12], 10, 12, [1, 2]),
    ([0, 10, 5, 7, 12], 10, 12, [1, 2, 3]),
    ([0, 10, 0, 10], 10, 10, [1, 2]),                    # the same rows again
    ([10, 20, 0, 10], 12, 20, [1]),                      # backwards, but rows of its own
    ([10, 20, 0, 11], 12, 20, [1, 2]),
    ([4, 4, 4, 8, 8, 2, 5, 9], 4, 9, [4, 5, 6]),         # sequences without tokens share nothing
    ([0, 10, 4, 4, 4, 10, 12], 10, 12, [1, 4]),
    ([0, 15, 3, 8], 10, 15, [0, 1]),                     # a sequence that is too long takes no rows
    ([0, 2 ** 31 - 1, 3, 8], 10, 15, [0, 1]),
    ([0, 90, 40, 120], 100, 120, [1, 2]),
    ([50, 120, 0, 50, 20, 30, 120], 100, 120, [1, 3, 4, 5]),
    (list(range(129)) + [3, 5, 128, 131], 200, 131, [128, 129, 130]),
    (list(range(129)) + [3, 5, 128, 131], 125, 131, [128, 129, 130]),
    (list(range(0, 1000, 10)) + [0, 5, 990, 999], 10, 1000, [99, 100, 101]),
    (list(range(301)) + [7, 9, 300, 302], 20, 302, [300, 301, 302]),  # 9 .. 299 is too long to take rows
    (list(range(1501)) + [700, 703, 1500, 1503], 900, 1503, [1500, 1501, 1502]),
    (list(range(1501)) + [700, 703, 1500, 1503], 20, 1503, [1500, 1501, 1502]),
    (list(range(50, 1500)) + [0, 9, 50], 60, 1499, [1449]),           # backwards, but rows of its own
]


def reported(table, T, rows):
    """The definition: by its own entries, then by those before it."""
    own = [0 <= s <= e <= rows and e - s <= T for s, e in zip(table, table[1:])]
    bad = []
    for b, (s, e) in enumerate(zip(table, table[1:])):
        before = any(own[i] and table[i] < table[i + 1] and table[i] < e and table[i + 1] > s for i in range(b))
        if not own[b] or (before and s < e):
            bad.append(b)
    return bad


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(TABLES)))
@pytest.mark.parametrize("heads", [(1, 2, 32, 32), (2, 16, 16, 64)])
def test_rows_of_another_sequence(L, case, heads):
    import torch
    table, T, rows, _ = TABLES[case]
    bad = reported(table, T, rows)
    B = len(table) - 1
    print(f"[gpu] chain T={T} rows={rows} table {table[:12]}{'...' if B > 11 else ''} reported {bad}", flush=True)
    c = Chain(900 + case, [rows] + [0] * (B - 1), *heads, packed=True, T=T, spare=0)
    c.first = np.array(table[:-1])
    c.n = np.array([0 if b in bad else table[b + 1] - table[b] for b in range(B)])
    c.first[c.n == 0] = 0
    c.live[:] = False
    for b in range(B):
        c.live[c.first[b]:c.first[b] + c.n[b]] = True
    a = c.device()
    a["start"] = torch.tensor(table, dtype=torch.int32, device="cuda")
    L.chain(c.dims(), **a)
    torch.cuda.synchronize()
    assert a["status"].tolist() == [9 * (b in bad) for b in range(B)]
    a["status"].zero_()
    check(c, a)


def test_definition():
    """The sequences that the tables are made for."""
    for table, T, rows, want in TABLES:
        assert reported(table, T, rows) == want, table
