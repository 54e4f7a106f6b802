"""Host-side refusals of gdn_chain, gdn_gate_norm and gdn_add_norm (no GPU: the pointers are never followed)."""
import ctypes
import os

import pytest

from paper_2607_06763_amd import gdn_layer as L
from paper_2607_06763_amd import gdn_tree as G


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(G.LIB_PATH):
        from paper_2607_06763_amd import build
        build.build()
    return G.lib()


def far(n, step=1 << 32):
    """n pointers that are far apart."""
    return [(i + 1) * step for i in range(n)]


def call(lib, name, d, ptrs):
    return getattr(lib, name)(None if d is None else ctypes.byref(d), *[ctypes.c_void_p(p) if p else None for p in ptrs], None)


def chain(lib, d, start=0, n_new=0, **put):
    names = ["q", "k", "v", "alpha", "beta", "conv_w", "conv_state", "conv_state_out", "S", "out", "status"]
    p = dict(zip(names, far(len(names))))
    p.update(put)
    return call(lib, "gdn_chain", d, [start, n_new] + [p[n] for n in names])


def test_chain_sizes(lib):
    mk = L.make_chain_dims
    bad = [
        (mk(-1, 4, 1, 1, 16, 16), G.GDN_EINVAL), (mk(1, -4, 1, 1, 16, 16), G.GDN_EINVAL), (mk(1, 4, 0, 1, 16, 16), G.GDN_EINVAL),
        (mk(1, 4, 2, 3, 16, 16), G.GDN_EINVAL), (mk(1, 4, 2, 1, 16, 16), G.GDN_EINVAL),
        (L.ChainDims(1, 4, 1, 1, 16, 16, 2, 0, 0, 0.0), G.GDN_EINVAL), (L.ChainDims(1, 4, 1, 1, 16, 16, 0, -1, 0, 0.0), G.GDN_EINVAL),
        (mk(1, 4, 1, 1, 16, 16, scale=-1.0), G.GDN_EINVAL), (mk(1, 4, 1, 1, 16, 16, scale=float("nan")), G.GDN_EINVAL),
        (mk(1, 4, 1, 1, 16, 16, scale=float("inf")), G.GDN_EINVAL),
        (mk(1, 4, 1, 1, 24, 16), G.GDN_EUNSUPPORTED), (mk(1, 4, 1, 1, 16, 256), G.GDN_EUNSUPPORTED),
        (mk(1, L.MAX_CHAIN_T + 1, 1, 1, 16, 16), G.GDN_EUNSUPPORTED), (mk(65536, 4, 1, 1, 16, 16), G.GDN_EUNSUPPORTED),
        (mk(200, L.MAX_CHAIN_T, 1, 1, 16, 16), G.GDN_EUNSUPPORTED),
    ]
    for d, want in bad:
        assert chain(lib, d) == want, d
        assert "chain" in G.last_error()
    assert call(lib, "gdn_chain", None, [0] * 13) == G.GDN_EINVAL
    ok = mk(2, 4, 1, 2, 16, 16)
    assert chain(lib, ok, start=64, n_new=1 << 40) == G.GDN_EINVAL and "n_new" in G.last_error()
    assert chain(lib, mk(2, 4, 1, 2, 16, 16, rows=-1), start=64) == G.GDN_EINVAL
    assert chain(lib, mk(2, 4, 1, 2, 16, 16, rows=1 << 31), start=64) == G.GDN_EUNSUPPORTED
    # nothing to do
    assert chain(lib, mk(0, 4, 1, 2, 16, 16), **{n: 0 for n in ("q", "S", "out", "conv_w")}) == G.GDN_OK


def test_chain_pointers(lib):
    d = L.make_chain_dims(2, 4, 1, 2, 16, 16)
    for n in ("q", "k", "v", "alpha", "beta", "conv_w", "conv_state", "conv_state_out", "S", "out"):
        assert chain(lib, d, **{n: 0}) == G.GDN_EINVAL, n
        assert "NULL" in G.last_error()
    C = 2 * 16 + 2 * 16
    sizes = dict(q=2 * 4 * 16 * 2, k=2 * 4 * 16 * 2, v=2 * 4 * 32 * 2, alpha=2 * 4 * 2 * 2, beta=2 * 4 * 2 * 2, conv_w=C * 16,
                 conv_state=2 * 3 * C * 4, conv_state_out=2 * 3 * C * 4, S=2 * 2 * 256 * 4, out=2 * 4 * 32 * 4)
    for written in ("S", "out", "conv_state_out"):
        for other in sizes:
            if other == written:
                continue
            at = 1 << 50
            for shift in (sizes[other] - 16, 16 - sizes[written]):  # their last and first bytes
                assert chain(lib, d, **{other: at, written: at + shift}) == G.GDN_EINVAL, (written, other)
                assert "overlap" in G.last_error()
    at = 1 << 50
    sizes = dict(sizes, status=8, n_new=8, start=12)
    for written in ("S", "out", "conv_state_out", "status"):
        for other in sizes:
            if "status" not in (written, other) and other not in ("n_new", "start") or other == written:
                continue
            rows = dict(start=0) if other != "start" else {}
            dims = d if other != "start" else L.make_chain_dims(2, 4, 1, 2, 16, 16, rows=8)
            for shift in (sizes[other] - 4, 4 - sizes[written]):
                assert chain(lib, dims, **dict(rows, **{other: at, written: at + shift})) == G.GDN_EINVAL, (written, other)
                assert "overlap" in G.last_error()


def gate(lib, d, x=1 << 32, g=2 << 32, w=3 << 32, out=4 << 32):
    return call(lib, "gdn_gate_norm", d, [x, g, w, out])


def test_gate_norm(lib):
    D = lambda N=2, H=3, d=8, tx=0, tg=1, to=1, act=0, ldx=0, ldg=0, eps=1e-6: L.GateNormDims(N, H, d, tx, tg, to, act, ldx, ldg, eps)
    for d in (D(N=-1), D(H=0), D(d=0), D(tx=2), D(tg=-1), D(to=7), D(act=2), D(act=-1), D(eps=0.0), D(eps=-1.0), D(eps=float("nan")),
              D(eps=float("inf")), D(eps=1e-40), D(ldx=23), D(ldg=23), D(ldx=-1)):
        assert gate(lib, d) == G.GDN_EINVAL, d.N
        assert "gate_norm" in G.last_error()
    for d in (D(d=L.MAX_NORM_D + 1), D(H=1 << 21, d=16), D(N=1 << 30, H=3), D(ldx=1 << 41)):
        assert gate(lib, d) == G.GDN_EUNSUPPORTED
    assert call(lib, "gdn_gate_norm", None, [0] * 4) == G.GDN_EINVAL
    assert gate(lib, D(), x=0) == G.GDN_EINVAL and gate(lib, D(), out=0) == G.GDN_EINVAL
    assert gate(lib, D(), x=(1 << 32) + 2) == G.GDN_EINVAL and "aligned" in G.last_error()
    assert gate(lib, D(), w=(3 << 32) + 1) == G.GDN_EINVAL and gate(lib, D(), g=(2 << 32) + 1) == G.GDN_EINVAL
    assert gate(lib, D(N=0), x=0, out=0) == G.GDN_OK
    # overlaps: in place only where types and rows are the same
    at = 1 << 40
    assert gate(lib, D(), x=at, out=at) == G.GDN_EINVAL and "overlap" in G.last_error()
    assert gate(lib, D(to=0, ldx=32), x=at, out=at) == G.GDN_EINVAL
    assert gate(lib, D(), g=at, out=at) == G.GDN_EINVAL
    assert gate(lib, D(), w=at, out=at - 64) == G.GDN_EINVAL
    assert gate(lib, D(to=0), x=at, out=at + 4) == G.GDN_EINVAL
    assert gate(lib, D(ldx=48), x=at, out=at + (48 + 23) * 4) == G.GDN_EINVAL  # the last value of the last row


def add(lib, d, x=1 << 32, r=2 << 32, w=3 << 32, pw=0, s=5 << 32, ro=6 << 32, out=7 << 32):
    return call(lib, "gdn_add_norm", d, [x, r, w, pw, s, ro, out])


def test_add_norm(lib):
    A = lambda N=2, D=24, tx=0, tr=0, to=1, post=0, eps=1e-6: L.AddNormDims(N, D, tx, tr, to, post, eps)
    for d in (A(N=-1), A(D=0), A(tx=2), A(tr=-1), A(to=7), A(eps=0.0), A(eps=float("nan")), A(eps=float("inf")), A(eps=1e-39)):
        assert add(lib, d) == G.GDN_EINVAL
        assert "add_norm" in G.last_error()
    for d in (A(D=L.MAX_NORM_D + 1), A(N=1 << 31)):
        assert add(lib, d) == G.GDN_EUNSUPPORTED
    assert call(lib, "gdn_add_norm", None, [0] * 7) == G.GDN_EINVAL
    assert add(lib, A(), x=0) == G.GDN_EINVAL and add(lib, A(), ro=0, out=0) == G.GDN_EINVAL
    assert add(lib, A(), pw=4 << 32) == G.GDN_EINVAL and "post" in G.last_error()
    assert add(lib, A(), r=(2 << 32) + 2) == G.GDN_EINVAL and "aligned" in G.last_error()
    assert add(lib, A(N=0), x=0, ro=0, out=0) == G.GDN_OK
    at = 1 << 40
    for put in (dict(x=at, ro=at), dict(r=at, ro=at + 4), dict(ro=at, out=at + 2), dict(x=at, out=at), dict(r=at, out=at),
                dict(w=at, out=at), dict(s=at, ro=at + 92), dict(out=at, ro=at)):
        assert add(lib, A(), **put) == G.GDN_EINVAL, put
        assert "overlap" in G.last_error()
    assert add(lib, A(to=0), x=at, out=at + 4) == G.GDN_EINVAL


def test_binding_refuses(lib):
    import torch
    x = torch.zeros(2, 3, 8)
    with pytest.raises(TypeError):
        L.gate_norm(None, None, x)
    with pytest.raises(ValueError):
        L.gate_norm(x[0], None, x)
    with pytest.raises(ValueError):
        L.gate_norm(x, None, x, act="tanh")
    with pytest.raises(TypeError):
        L.add_norm(None, x, x, x)
    with pytest.raises(ValueError):
        L.add_norm(x, x, x, x)
    d = L.make_chain_dims(1, 2, 1, 1, 16, 16, in_dtype="f32")
    z = torch.zeros(1, 2, 1, 16)
    with pytest.raises(ValueError):
        L.chain(d, z, z, z, z, z, z, z, z, z, z)
