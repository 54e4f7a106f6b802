"""Host-side checks of the attention, cache and sampling calls (no GPU
needed): bad arguments are refused before any device work, empty problems
succeed without touching a pointer, and the binding takes only tensors of the
stated type, shape, place and stride."""
import ctypes

import pytest

from paper_2607_06763_amd import gdn_attn as A
from paper_2607_06763_amd import gdn_tree as G

P = 1 << 20  # never followed; a multiple of 16


@pytest.fixture(scope="module")
def L():
    return G.lib()


def ptrs(n, step=1 << 26):
    """n pointers whose arrays cannot overlap at the sizes used here"""
    return [ctypes.c_void_p(P + i * step) for i in range(n)]


def calls(L, d, meta=None, n_new=None, ptr=True):
    """status of each call that takes gdn_attn_dims"""
    D = ctypes.byref(d) if d is not None else None
    p = ptrs(10) if ptr else [None] * 10
    out = [L.gdn_kv_append(D, meta, n_new, *p[:10], None), L.gdn_tree_attend(D, meta, n_new, *p[:6], None)]
    if n_new is None:
        out.append(L.gdn_kv_commit(D, meta, *p[:7], None))
    return out


def dims(**kw):
    a = dict(B=1, T=7, Hq=8, Hkv=2, d=64, page=64, n_pages=4, max_pages=2, dtype="bf16", rot=0)
    a.update(kw)
    dt = a.pop("dtype_code", None)
    r = A.make_attn_dims(**a)
    if dt is not None:
        r.dtype = dt
    return r


BAD = [
    (dict(B=-1), "EINVAL"), (dict(T=-2), "EINVAL"), (dict(Hq=0), "EINVAL"), (dict(Hkv=0), "EINVAL"),
    (dict(Hq=7), "EINVAL"), (dict(dtype_code=2), "EINVAL"), (dict(dtype_code=-1), "EINVAL"),
    (dict(scale=-1.0), "EINVAL"), (dict(scale=float("nan")), "EINVAL"), (dict(scale=float("inf")), "EINVAL"),
    (dict(n_pages=0), "EINVAL"), (dict(max_pages=0), "EINVAL"), (dict(rot=3), "EINVAL"), (dict(rot=66), "EINVAL"),
    (dict(rot=-2), "EINVAL"), (dict(n_pos=-1), "EINVAL"),
    (dict(d=0), "EUNSUPPORTED"), (dict(d=48), "EUNSUPPORTED"), (dict(d=512), "EUNSUPPORTED"),
    (dict(page=0), "EUNSUPPORTED"), (dict(page=8), "EUNSUPPORTED"), (dict(page=48), "EUNSUPPORTED"),
    (dict(page=512), "EUNSUPPORTED"), (dict(T=513), "EUNSUPPORTED"), (dict(B=65536), "EUNSUPPORTED"),
    (dict(Hq=16384, Hkv=16384), "EUNSUPPORTED"), (dict(T=512, Hq=4096, Hkv=1), "EUNSUPPORTED"),
    (dict(page=256, max_pages=1 << 23), "EUNSUPPORTED"),
]


@pytest.mark.parametrize("kw,want", BAD, ids=lambda x: "-".join(f"{k}{v}" for k, v in x.items()) if isinstance(x, dict) else x)
def test_bad_sizes(L, kw, want):
    for rc in calls(L, dims(**kw)):
        assert rc == getattr(G, "GDN_" + want)
        assert G.last_error()


def test_null_and_meta_with_lengths(L):
    for rc in calls(L, dims(), ptr=False):
        assert rc == G.GDN_EINVAL and "NULL" in G.last_error()
    for rc in calls(L, None):
        assert rc == G.GDN_EINVAL
    m = ctypes.c_void_p(P)
    for rc in calls(L, dims(), meta=m, n_new=m):
        assert rc == G.GDN_EINVAL and "n_new" in G.last_error()
    # a rotation without its table
    p = ptrs(10)
    p[3] = None
    assert L.gdn_kv_append(ctypes.byref(dims(rot=64, n_pos=9)), None, None, *p, None) == G.GDN_EINVAL


@pytest.mark.parametrize("kw", [dict(B=0), dict(T=0)])
def test_nothing_to_do(L, kw):
    assert calls(L, dims(**kw), ptr=False) == [G.GDN_OK] * 3
    s = A.SampleDims(kw.get("B", 2), kw.get("T", 3), 50, G.GDN_F32, 0)
    assert L.gdn_tree_sample(ctypes.byref(s), *([None] * 9)) == G.GDN_OK
    a = G.Dims(kw.get("B", 2), kw.get("T", 3), 1, 1, 16, 16, 0, 0.0)
    assert L.gdn_tree_accept(ctypes.byref(a), *([None] * 7)) == G.GDN_OK


def test_overlaps(L):
    d = dims(B=2)
    D = ctypes.byref(d)
    qb, kb = 2 * 7 * 8 * 64 * 2, 2 * 7 * 2 * 64 * 2
    at = lambda i, off=0: ctypes.c_void_p(P + (i << 26) + off)

    def append(q, k, v, q_out):
        return L.gdn_kv_append(D, None, None, q, k, v, None, at(3), at(4), at(5), at(6), q_out, None, None)
    assert append(at(0), at(1), at(2), at(0, 16)) == G.GDN_EINVAL
    assert append(at(0, qb - 16), at(1), at(2), at(0)) == G.GDN_EINVAL
    assert append(at(0), at(1), at(2), at(1, kb - 16)) == G.GDN_EINVAL
    assert append(at(0), at(1), at(2, qb - 16), at(2)) == G.GDN_EINVAL
    for off in (0, 16, qb - 16):
        assert L.gdn_tree_attend(D, None, None, at(0), at(1), at(2), at(3), at(4), at(0, off), None) == G.GDN_EINVAL
    for off in (0, 4):
        assert L.gdn_kv_commit(D, None, at(0), at(1), at(2), at(3), at(4), at(2, off), None, None) == G.GDN_EINVAL
        assert L.gdn_kv_commit(D, None, at(0), at(1), at(2), at(3), at(4), at(0, off), None, None) == G.GDN_EINVAL
    for src in (0, 1):
        assert L.gdn_tree_accept(ctypes.byref(G.Dims(2, 7, 1, 1, 16, 16, 0, 0.0)), None, at(0), at(1), at(2), at(3),
                                 at(src, 52), None) == G.GDN_EINVAL


@pytest.mark.parametrize("s,want", [
    ((-1, 1, 9, 0, 0), "EINVAL"), ((1, -1, 9, 0, 0), "EINVAL"), ((1, 1, 0, 0, 0), "EINVAL"),
    ((1, 1, 9, 2, 0), "EINVAL"), ((1, 1, 9, 0, 8), "EINVAL"), ((1, 1, 9, 0, -9), "EINVAL"),
    ((1, 513, 9, 0, 0), "EUNSUPPORTED"), ((1, 1, (1 << 20) + 1, 0, 0), "EUNSUPPORTED"),
    ((1 << 23, 256, 9, 0, 0), "EUNSUPPORTED")])
def test_sample_bad_sizes(L, s, want):
    d = A.SampleDims(*s)
    p = ptrs(7)
    assert L.gdn_tree_sample(ctypes.byref(d), None, *p, None) == getattr(G, "GDN_" + want)
    assert G.last_error()


def test_sample_accept_null(L):
    d = A.SampleDims(1, 1, 9, 0, 0)
    assert L.gdn_tree_sample(None, *([None] * 9)) == G.GDN_EINVAL
    p = ptrs(7)  # logits, temperature, top_k, top_p, min_p, u, token
    for i in (0, 5, 6):
        q = list(p)
        q[i] = None
        assert L.gdn_tree_sample(ctypes.byref(d), None, *q, None) == G.GDN_EINVAL and "NULL" in G.last_error()
    a = G.Dims(1, 4, 1, 1, 16, 16, 0, 0.0)
    assert L.gdn_tree_accept(None, *([None] * 7)) == G.GDN_EINVAL
    for i in range(5):
        q = ptrs(5)
        q[i] = None
        assert L.gdn_tree_accept(ctypes.byref(a), None, *q, None) == G.GDN_EINVAL
    for T in (-1, 513):
        assert L.gdn_tree_accept(ctypes.byref(G.Dims(1, T, 1, 1, 16, 16, 0, 0.0)), None, *ptrs(5), None) < 0


def test_binding_refuses_host_tensors_and_others():
    import torch
    d = dims()
    z = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t)
    kc, vc = (z(*s) for s in A.cache_shapes(d))
    assert A.cache_shapes(d) == ((4, 2, 8, 64, 8), (4, 2, 8, 64, 8))
    i = lambda *s: z(*s, t=torch.int32)
    with pytest.raises(ValueError):
        A.kv_append(d, z(1, 7, 8, 64), z(1, 7, 2, 64), z(1, 7, 2, 64), None, i(1), i(1, 2), kc, vc, z(1, 7, 8, 64))
    with pytest.raises(ValueError):
        A.attend(d, z(1, 7, 8, 64), kc, vc, i(1, 2), i(1), z(1, 7, 8, 64))
    with pytest.raises(ValueError):
        A.kv_commit(d, i(1), i(1, 2), i(1), kc, vc, i(1))
    u = z(1, 7, t=torch.float32)
    with pytest.raises(ValueError):
        A.sample(z(1, 7, 9), u, i(1, 7))
    with pytest.raises(ValueError):
        A.sample(z(7, 9), u, i(1, 7))
    with pytest.raises(ValueError):
        A.sample(z(1, 7, 9, t=torch.float16), u, i(1, 7))
    with pytest.raises(TypeError):
        A.sample([[0.0]], u, i(1, 7))
    with pytest.raises(ValueError):
        A.accept(i(1, 7), i(1, 7), i(1), i(1), i(1, 7))
    with pytest.raises(ValueError):
        A.accept(i(7), i(1, 7), i(1), i(1), i(1, 7))
    with pytest.raises(TypeError):
        A.accept([1], i(1, 7), i(1), i(1), i(1, 7))


def test_dims_forget_their_shapes_when_changed():
    d = dims(dtype="f32")
    assert A.cache_shapes(d) == ((4, 2, 16, 64, 4), (4, 2, 16, 64, 4))
    d.n_pages, d.dtype = 5, G.GDN_BF16
    assert A.cache_shapes(d) == ((5, 2, 8, 64, 8), (5, 2, 8, 64, 8))
