"""gdn_gate_norm and gdn_add_norm at rows that lie more than 2^31 elements (and 2^32
bytes) into their tensors.  Tolerances: tests/test_norm_gpu.py."""
import numpy as np
import pytest

from tests.test_norm_gpu import REL, data, dt, f64, half

pytestmark = pytest.mark.gpu

BF16 = 2.0 ** -8
assert half("bf16") == BF16


@pytest.fixture(scope="module")
def L():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_06763_amd import gdn_layer as L
    return L


def gated(x, g):
    return f64(x) / np.sqrt((f64(x) ** 2).mean(-1, keepdims=True) + float(np.float32(1e-6))) * f64(g) / (1 + np.exp(-f64(g)))


def test_gate_norm_of_many_rows(L):
    import torch
    N, H, d = 350001, 48, 128
    assert N * H * d > 2 ** 31
    print(f"[gpu] gate_norm of {N} rows of {H} heads of {d}, bf16", flush=True)
    x = torch.zeros(N, H, d, dtype=dt("bf16"), device="cuda")
    out = torch.full_like(x, float("nan"))
    g = torch.ones_like(x)
    rows = [slice(0, 3), slice(N - 3, N)]
    for k, r in enumerate(rows):
        x[r], g[r] = data(50 + k, 3, H, d, dtype="bf16"), data(60 + k, 3, H, d, dtype="bf16")
    L.gate_norm(x, g, out)
    torch.cuda.synchronize()
    for r in rows:
        want = gated(x[r], g[r])
        assert np.all(np.abs(f64(out[r]) - want) <= (REL + BF16) * np.abs(want))
    assert int(torch.count_nonzero(out[3:N - 3])) == 0  # every row is written (NaN counts), that of zeros with zeros


@pytest.mark.parametrize("tx,tg", [("bf16", "bf16"), ("f32", "bf16")])
def test_gate_norm_of_rows_far_apart(L, tx, tg):
    import torch
    N, H, d, ld = 35, 3, 40, (1 << 26) + 24
    assert (N - 1) * ld > 2 ** 31
    print(f"[gpu] gate_norm of {N} rows {ld} elements apart, {tx} {tg}", flush=True)
    bx, bg = (torch.empty(N * ld, dtype=dt(t), device="cuda") for t in (tx, tg))
    x = bx.view(N, ld)[:, 8:8 + H * d].unflatten(1, (H, d))
    g = bg.view(N, ld)[:, ld - H * d:].unflatten(1, (H, d))
    x.copy_(data(52, N, H, d))
    g.copy_(data(53, N, H, d))
    out = torch.empty(N, H, d, device="cuda")
    L.gate_norm(x, g, out)
    torch.cuda.synchronize()
    want = gated(x, g)
    assert np.all(np.abs(f64(out) - want) <= (REL + 2.0 ** -24) * np.abs(want))


def test_add_norm_of_many_rows(L):
    import torch
    N, D = 524301, 4099
    assert N * D > 2 ** 31
    print(f"[gpu] add_norm of {N} rows of {D}, bf16", flush=True)
    x = torch.zeros(N, D, dtype=dt("bf16"), device="cuda")
    r = torch.zeros_like(x)
    rows = [slice(0, 2), slice(N - 2, N)]
    for k, s in enumerate(rows):
        x[s], r[s] = data(54 + k, 2, D, dtype="bf16"), data(56 + k, 2, D, dtype="bf16")
    mag = [np.abs(f64(x[s])) + np.abs(f64(r[s])) for s in rows]
    want = [f64(x[s]) + f64(r[s]) for s in rows]
    L.add_norm(x, r, r, x)
    torch.cuda.synchronize()
    for s, z, m in zip(rows, want, mag):
        assert np.all(np.abs(f64(r[s]) - z) <= REL * m + BF16 * np.abs(z))
        f = 1 / np.sqrt((z * z).mean(-1, keepdims=True) + float(np.float32(1e-6)))
        row = np.sqrt((m * m).mean(-1, keepdims=True)) * f
        assert np.all(np.abs(f64(x[s]) - z * f) <= REL * m * f + (REL * (1 + row) + BF16) * np.abs(z * f))
    assert int(torch.count_nonzero(x[2:N - 2])) == 0 and int(torch.count_nonzero(r[2:N - 2])) == 0
