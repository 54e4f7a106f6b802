"""gdn_gate_norm and gdn_add_norm against 64-bit numpy.

Tolerances.  A sum of d squares in 32 bits is off by less than
(8 + log2 d) 2^-24 of itself (a thread adds up to 64, the threads in a tree: 64 2^-24
at most), the root by half of that, the reciprocal root, the mean, the
exponential (|g| below 8: 2^-20) and the products by a few 2^-23: 2^-18 of a
value together.  Each output is off by half a step of its type besides:
2^-24 or 2^-8.  add_norm's norm is off by that of its sum, of which residual and
x may cancel: 2^-18 of |residual| + |scale x| relative to the row's norm."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

REL = 2.0 ** -18


@pytest.fixture(scope="module")
def L():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_06763_amd import gdn_layer as L
    return L


def dt(n):
    import torch
    return torch.bfloat16 if n == "bf16" else torch.float32


def half(n):
    return 2.0 ** -8 if n == "bf16" else 2.0 ** -24


def f64(t):
    return t.double().cpu().numpy()


def data(seed, *shape, dtype="f32", s=1.0):
    import torch
    return torch.from_numpy(s * np.random.default_rng([3, seed]).standard_normal(shape)).to(dt(dtype)).cuda()


GATES = [
    # N, H, d, types of x, gate (None: no gate), out
    (1, 1, 1, "f32", "f32", "f32"), (1, 48, 128, "f32", "bf16", "bf16"), (3, 5, 8, "bf16", "f32", "f32"),
    (7, 3, 16, "f32", None, "bf16"), (129, 2, 24, "bf16", "bf16", "bf16"), (2, 7, 33, "f32", "bf16", "f32"),
    (5, 2, 65, "bf16", "f32", "bf16"), (33, 3, 256, "f32", "f32", "f32"), (4, 1, 257, "bf16", "bf16", "f32"),
    (3, 2, 504, "f32", "bf16", "bf16"), (2, 3, 520, "f32", "f32", "f32"), (2, 1, 2049, "bf16", "f32", "f32"),
    (2, 2, 4096, "f32", "bf16", "f32"), (1, 1, 5000, "f32", "bf16", "f32"), (2, 1, 8200, "bf16", "bf16", "bf16"),
    (1, 1, 16383, "f32", "f32", "f32"), (1, 2, 16384, "bf16", "bf16", "f32"), (3000, 16, 64, "f32", "bf16", "bf16"),
]


@pytest.mark.parametrize("case", GATES, ids=lambda c: ".".join(map(str, c)))
@pytest.mark.parametrize("act", ["silu", "sigmoid"])
def test_gate_norm(L, case, act):
    import torch
    N, H, d, tx, tg, to = case
    print(f"[gpu] gate_norm {case} {act}", flush=True)
    x = data(1, N, H, d, dtype=tx, s=0.3)
    x[0, 0] = 0  # a head of zeros: out 0, not NaN
    g = None if tg is None else data(2, N, H, d, dtype=tg, s=2.0)
    w = 1 + data(3, d, s=0.2)
    weight = None if N == 3 else w
    out = torch.full((N, H, d), float("nan"), dtype=dt(to), device="cuda")
    L.gate_norm(x, g, out, weight=weight, eps=1e-5, act=act)
    torch.cuda.synchronize()
    y = f64(x) / np.sqrt((f64(x) ** 2).mean(-1, keepdims=True) + float(np.float32(1e-5)))
    if weight is not None:
        y = y * f64(weight)
    if g is not None:
        s = 1 / (1 + np.exp(-f64(g)))
        y = y * (s if act == "sigmoid" else s * f64(g))
    err = np.abs(f64(out) - y)
    tol = (REL + half(to)) * np.abs(y)
    assert np.all(err <= tol), float((err - tol).max())


@pytest.mark.parametrize("tx,tg,off", [("f32", "bf16", 8), ("bf16", "f32", 16), ("f32", "f32", 3), ("bf16", "bf16", 1)])
def test_gate_norm_of_rows_apart(L, tx, tg, off):
    """Parts of wider rows, with and without the alignment that packs need; what lies between the rows is not a number."""
    import torch
    N, H, d = 9, 3, 40
    bx = torch.full((N, H * d + 2 * off), float("nan"), dtype=dt(tx), device="cuda")
    bg = torch.full((N, H * d + 3 * off), float("nan"), dtype=dt(tg), device="cuda")
    x, g = bx[:, off:off + H * d].unflatten(1, (H, d)), bg[:, off:off + H * d].unflatten(1, (H, d))
    x.copy_(data(4, N, H, d))
    g.copy_(data(5, N, H, d))
    out = torch.empty(N, H, d, device="cuda")
    L.gate_norm(x, g, out)
    y = f64(x) / np.sqrt((f64(x) ** 2).mean(-1, keepdims=True) + 1e-6) * f64(g) / (1 + np.exp(-f64(g)))
    assert np.all(np.abs(f64(out) - y) <= (REL + 2.0 ** -24) * np.abs(y))


def test_in_place(L):
    import torch
    x, g = data(6, 50, 4, 64), data(7, 50, 4, 64)
    want = torch.empty_like(x)
    L.gate_norm(x, g, want)
    L.gate_norm(x, g, x)
    assert torch.equal(x, want)
    for D in (64, 640, 2051):
        x, r, s = data(8, 33, D), data(9, 33, D), data(10, D)
        ro, o = torch.empty_like(r), torch.empty_like(x)
        L.add_norm(x, r, ro, o, scale=s, post=True)
        L.add_norm(x, r, r, x, scale=s, post=True)
        assert torch.equal(r, ro) and torch.equal(x, o)


ADDS = [
    # N, D, types of x, residual (None), out (None), post, scale, weight
    (1, 1, "f32", "f32", "f32", True, True, True), (1, 4096, "bf16", "bf16", "bf16", False, False, True),
    (5, 8, "bf16", "f32", "bf16", True, False, True), (300, 64, "f32", "bf16", "f32", True, True, False),
    (17, 100, "f32", "f32", "f32", False, True, True), (9, 512, "bf16", "bf16", "f32", True, True, True),
    (4, 1000, "f32", None, "bf16", False, False, True), (4, 1001, "bf16", "f32", None, True, True, False),
    (33, 2051, "f32", "f32", "f32", True, False, True), (3, 4099, "bf16", "bf16", "bf16", True, True, True),
    (2500, 2048, "bf16", "f32", "bf16", True, True, True), (2, 6144, "f32", "bf16", "f32", False, True, True),
    (2, 16384, "bf16", "bf16", "bf16", True, True, True), (2, 16381, "f32", "f32", "f32", True, True, True),
    (3, 2048, "f32", None, "f32", True, True, True),
]


@pytest.mark.parametrize("case", ADDS, ids=lambda c: ".".join(map(str, c)))
def test_add_norm(L, case):
    import torch
    N, D, tx, tr, to, post, scale, weight = case
    print(f"[gpu] add_norm {case}", flush=True)
    x, r = data(11, N, D, dtype=tx), None if tr is None else data(12, N, D, dtype=tr, s=2.0)
    if post:
        x[0] = 0
    pw, s, w = (1 + data(k, D, s=0.2) if on else None for k, on in ((13, post), (14, scale), (15, weight)))
    ro = None if tr is None else torch.full((N, D), float("nan"), dtype=dt(tr), device="cuda")
    out = None if to is None else torch.full((N, D), float("nan"), dtype=dt(to), device="cuda")
    L.add_norm(x, r, ro, out, weight=w, post_weight=pw, scale=s, post=post, eps=1e-6)
    torch.cuda.synchronize()
    eps = float(np.float32(1e-6))
    y = f64(x)
    if post:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * f64(pw)
    if scale:
        y = y * f64(s)
    z = y if r is None else f64(r) + y
    mag = np.abs(y) + (0 if r is None else np.abs(f64(r)))
    if ro is not None:
        assert np.all(np.abs(f64(ro) - z) <= REL * mag + half(tr) * np.abs(z))
    if out is not None:
        f = (1 if w is None else f64(w)) / np.sqrt((z * z).mean(-1, keepdims=True) + eps)
        # the sum's own error moves the norm by at most its share of the row
        row = np.sqrt((mag * mag).mean(-1, keepdims=True)) / np.sqrt((z * z).mean(-1, keepdims=True) + eps)
        want = z * f
        assert np.all(np.abs(f64(out) - want) <= REL * mag * np.abs(f) + (REL * (1 + row) + half(to)) * np.abs(want))


@pytest.mark.parametrize("D", [16, 72, 640, 2051])
def test_rows_are_their_own(L, D):
    """NaN, infinities and zeros in some rows (heads) reach no other."""
    import torch
    x, r, g = data(16, 41, D), data(17, 41, D), data(18, 41, D, dtype="bf16")
    run = lambda: (L.add_norm(x, r, ro, o, post=True), L.gate_norm(x.view(41, 1, D), g.view(41, 1, D), h.view(41, 1, D)))
    ro, o, h = (torch.empty_like(x) for _ in range(3))
    run()
    want = [t.clone() for t in (ro, o, h)]
    x[3], x[17, D // 2], r[20], g[33, 0] = float("nan"), float("inf"), float("nan"), float("nan")
    x[5] = 0
    run()
    keep = [i for i in range(41) if i not in (3, 5, 17, 20, 33)]
    for a, b in zip((ro, o, h), want):
        assert torch.equal(a[keep], b[keep])
    assert torch.equal(ro[5], r[5]) and (h[5] == 0).all()
    assert all(torch.isnan(t[3]).all() for t in (ro, o, h))


def test_graph_and_stream(L):
    """Norms around a block captured on a stream of their own and replayed on new inputs, eager work between."""
    import torch
    x, r, g, s = data(19, 70, 384), data(20, 70, 384), data(21, 70, 384, dtype="bf16"), data(22, 384)
    ro, o = torch.empty_like(r), torch.empty_like(x, dtype=torch.bfloat16)
    y = torch.empty(70, 6, 64, device="cuda")

    def work(ro, o, y):
        L.gate_norm(x.view(70, 6, 64), g.view(70, 6, 64), y)
        L.add_norm(y.view(70, 384), r, ro, o, scale=s, post=True)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        work(ro, o, y)
    for k in range(4):
        x.copy_(data(30 + k, 70, 384))
        g.copy_(data(40 + k, 70, 384, dtype="bf16"))
        graph.replay()
        want = [torch.empty_like(t) for t in (ro, o, y)]
        work(*want)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((ro, o, y), want)), k
