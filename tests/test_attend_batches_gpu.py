"""Attention of more than 64 sequences, whose lengths a wave takes in turns of
64, against the definition in 64 bits (tolerances of test_attend_gpu).  Short
sequences and empty ones, and long ones that several runs share, before and
after the 64th."""
import numpy as np
import pytest

from tests.attn_ref import Case
from tests.test_attend_gpu import A, check, run  # noqa: F401

pytestmark = pytest.mark.gpu


def lengths(B, seed, longs):
    """0, 1, up to a few tiles; the sequences of longs long."""
    rng = np.random.default_rng([77, seed])
    ctx = [int(rng.choice([0, 1, rng.integers(2, 60), rng.integers(60, 400)])) for _ in range(B)]
    for b, n in longs:
        ctx[b] = n
    return ctx


CASES = [
    # seed, B, T, Hq, Hkv, d, dtype, tree, long sequences
    (1, 65, 1, 4, 1, 64, "bf16", None, [(64, 9000)]),
    (2, 65, 1, 2, 2, 32, "f32", None, [(64, 5000)]),
    (3, 150, 1, 4, 2, 128, "bf16", None, [(3, 2000), (66, 7000), (149, 3000)]),
    (4, 150, 1, 2, 1, 64, "f32", None, [(70, 6000), (128, 4000)]),
    (5, 70, 9, 8, 2, 64, "bf16", "any", [(2, 900), (66, 5000)]),      # 36 rows a key head: shared tiles
    (6, 130, 12, 4, 1, 128, "bf16", "any", [(64, 3000), (129, 2500)]),
    (7, 129, 40, 1, 1, 64, "bf16", None, [(127, 1000), (128, 2000)]),
    (8, 66, 5, 2, 1, 64, "f32", "any", [(65, 3000)]),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"B{c[1]}-T{c[2]}-H{c[3]}.{c[4]}-d{c[5]}-{c[6]}")
def test_many_sequences(A, case):  # noqa: F811
    import torch
    seed, B, T, Hq, Hkv, d, dt, tree, longs = case
    print(f"[gpu] attend {case}", flush=True)
    c = Case(900 + seed, T, lengths(B, seed, longs), Hq, Hkv, d, 64, dt, parent=tree)
    c.append_slots()
    out = run(A, c)
    torch.cuda.synchronize()
    check(c, out)


def test_skipped_sequences_among_many(A):  # noqa: F811
    """Lengths that are out of range clear their sequence's outputs and leave the others."""
    import torch
    c = Case(950, 3, lengths(140, 9, [(67, 3000)]), 4, 2, 64, 64, "bf16", parent="any")
    c.append_slots()
    g = c.device()
    bad = [0, 63, 64, 100, 139]
    for b in bad[:3]:
        g["ctx"][b] = -1
    for b in bad[3:]:
        g["ctx"][b] = c.max_pages * c.page
    out = run(A, c, g)
    torch.cuda.synchronize()
    ref, mag = c.attend_ref()
    ref[bad] = 0
    check(c, out, (ref, mag))
    assert not out[bad].any()
