"""Paged cache of the softmax-attention layers: append with the rotation and
commit of the accepted path, against plain 64-bit definitions.

Tolerance of a rotated value: two products and a sum in fp32 (3 roundings of
2^-24 of the larger product each, taken as 4).  A bf16 result must be the
rounding of a value within that.  Everything that is only moved is compared
bit for bit."""
import numpy as np
import pytest

from tests.attn_ref import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_06763_amd import gdn_attn as A
    from paper_2607_06763_amd import gdn_tree as G
    G.lib()
    return A


def bits(t):
    import torch
    return t.view(torch.int16 if t.element_size() == 2 else torch.int32)


def rotated(c, x):
    """x [B][T][H][d] rotated in 64 bits: least and largest right value."""
    import torch
    h = c.rot // 2
    y = x.double().numpy().copy()
    tol = np.zeros_like(y)
    for b in range(c.B):
        for i in range(c.T):
            if not c.real[b, i]:
                continue
            cs = c.rope[c.ctx[b] + c.depth[b, i]].astype(np.float64)
            p, n = y[b, i, :, :h].copy(), y[b, i, :, h:2 * h].copy()
            y[b, i, :, :h] = p * cs[:, 0] - n * cs[:, 1]
            y[b, i, :, h:2 * h] = n * cs[:, 0] + p * cs[:, 1]
            m = np.abs(p) + np.abs(n)
            tol[b, i, :, :h] = tol[b, i, :, h:2 * h] = 4 * 2.0 ** -24 * m
    return [torch.from_numpy(y + s * tol).to(c.tdt).double().numpy() for s in (-1, 1)] if c.dtype == "bf16" else [y - tol, y + tol]


APPEND = [
    # seed, T, ctx, Hq, Hkv, d, page, dtype, tree, rot, valid nodes
    (1, 1, [0], 2, 1, 32, 16, "bf16", None, None, None),
    (2, 1, [5, 0, 1023, 64], 32, 8, 128, 64, "bf16", None, None, None),
    (3, 7, [9, 16, 250], 4, 4, 64, 32, "f32", "any", None, [7, 0, 3]),
    (4, 64, [77, 3], 6, 2, 256, 128, "bf16", "any", 64, [64, 41]),
    (5, 33, [31], 8, 1, 128, 256, "f32", "up", 0, None),
    (6, 20, [1, 2, 6, 7], 5, 5, 32, 16, "bf16", "any", 8, [20, 19, 1, 12]),   # halves of 4 values: inside a pack
    (7, 19, [13], 4, 2, 64, 16, "f32", "any", 6, None),
    (8, 512, [100], 2, 1, 64, 64, "bf16", None, 32, None),
]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: f"T{c[1]}-d{c[5]}-p{c[6]}-{c[7]}-r{c[9]}")
@pytest.mark.parametrize("inplace", [False, True])
def test_append(A, case, inplace):
    import torch
    seed, T, ctx, Hq, Hkv, d, page, dt, tree, rot, nv = case
    print(f"[gpu] append {case} inplace={inplace}", flush=True)
    c = Case(seed, T, ctx, Hq, Hkv, d, page, dt, parent=tree, rot=rot, n_valid=nv)
    g = c.device()
    qo = g["q"] if inplace else torch.full_like(g["q"], float("nan"))
    st = torch.full((c.B,), -7, dtype=torch.int32, device="cuda")
    A.kv_append(c.dims(), g["q"], g["k"], g["v"], g["rope"] if c.rot else None, g["ctx"], g["table"], g["kc"], g["vc"], qo,
                kv_status=st, meta=g["meta"])
    torch.cuda.synchronize()
    assert st.tolist() == [0] * c.B
    lo, hi = rotated(c, c.q)
    got = qo.cpu().double().numpy()
    assert np.all((lo <= got)[c.real]) and np.all((got <= hi)[c.real])
    assert np.all(got[~c.real] == 0)
    # caches: new rows where they belong, every other value as it was
    klo, khi = rotated(c, c.k)
    before_k, before_v = c.kc.clone(), c.vc.clone()
    kg, vg = g["kc"].cpu(), g["vc"].cpu()
    new_k, new_v = torch.zeros_like(before_k, dtype=torch.bool), torch.zeros_like(before_v, dtype=torch.bool)
    for b in range(c.B):
        for i in np.nonzero(c.real[b])[0]:
            pg, off = c.place(b, int(c.ctx[b] + i))
            row = kg[pg, :, :, off].reshape(Hkv, d).double().numpy()
            assert np.all(klo[b, i] <= row) and np.all(row <= khi[b, i])
            assert torch.equal(bits(vg[pg, :, off // c.x, :, off % c.x].contiguous()), bits(c.v[b, i]))
            new_k[pg, :, :, off] = True
            new_v[pg, :, off // c.x, :, off % c.x] = True
    assert torch.equal(bits(kg)[~new_k], bits(before_k)[~new_k])
    assert torch.equal(bits(vg)[~new_v], bits(before_v)[~new_v])


def test_append_chain_lengths(A):
    """n_new: slots past it are padding."""
    import torch
    c = Case(20, 9, [4, 30, 8], 4, 2, 64, 16, "bf16", n_new=[9, 0, 5])
    g = c.device()
    qo = torch.full_like(g["q"], float("nan"))
    A.kv_append(c.dims(), g["q"], g["k"], g["v"], g["rope"], g["ctx"], g["table"], g["kc"], g["vc"], qo, n_new=g["n_new"])
    c.append_slots()
    torch.cuda.synchronize()
    assert torch.equal(bits(g["vc"].cpu()), bits(c.vc))
    assert np.all(qo.cpu().double().numpy()[~c.real] == 0) and torch.isfinite(qo).all()


def test_append_skips_bad_sequences(A):
    """A bad length, position, page or tree skips its sequence only."""
    import torch
    from paper_2607_06763_amd import gdn_tree as G
    c = Case(21, 6, [10, 10, 10, 10, 10, 10], 2, 1, 32, 16, "bf16", parent="any")
    c.parent[5, :] = -1  # several roots
    ctx = c.ctx.copy()
    ctx[1], ctx[2] = -1, c.max_pages * c.page - 5
    g = c.device()
    g["ctx"] = c.i32(ctx)
    g["table"][3, 0] = c.n_pages  # a page that holds new rows
    d = c.dims()
    kc, vc = g["kc"].clone(), g["vc"].clone()
    qo = torch.full_like(g["q"], float("nan"))
    st = torch.full((6,), -7, dtype=torch.int32, device="cuda")
    A.kv_append(d, g["q"], g["k"], g["v"], g["rope"], g["ctx"], g["table"], g["kc"], g["vc"], qo, kv_status=st, meta=g["meta"])
    torch.cuda.synchronize()
    assert st.tolist() == [0, G.KV_BAD_LEN, G.KV_BAD_LEN, G.KV_BAD_PAGE, 0, G.TREE_MULTI_ROOT]
    for b in (1, 2, 3, 5):
        assert np.all(qo[b].float().cpu().numpy() == 0)
        pages = torch.from_numpy(c.table[b][c.table[b] >= 0])
        assert torch.equal(bits(g["kc"].cpu()[pages]), bits(kc.cpu()[pages]))
        assert torch.equal(bits(g["vc"].cpu()[pages]), bits(vc.cpu()[pages]))
    # a rotation table one row short
    d.n_pos = int(10 + c.depth[0].max())
    A.kv_append(d, g["q"], g["k"], g["v"], g["rope"][:d.n_pos].contiguous(), g["ctx"], g["table"], g["kc"], g["vc"], qo,
                kv_status=st, meta=g["meta"])
    assert st[0].item() == G.KV_BAD_POS


COMMIT = [
    (1, 1, [3], 1, 32, 16, "bf16", "any", None),
    (2, 40, [0, 17, 250], 2, 64, 16, "bf16", "any", [40, 23, 1]),     # any numbering: rows trade places
    (3, 64, [5, 100], 4, 128, 64, "f32", "any", [64, 30]),
    (4, 128, [1000], 2, 256, 128, "bf16", "up", None),
    (5, 512, [7, 60], 1, 128, 32, "f32", "chain-any", None),          # paths of 512 slots in any order
    (6, 300, [33], 2, 32, 256, "bf16", "chain-any", [257]),
]


@pytest.mark.parametrize("case", COMMIT, ids=lambda c: f"T{c[1]}-d{c[4]}-p{c[5]}-{c[6]}")
@pytest.mark.parametrize("where", ["deep", "any"])
def test_commit(A, case, where):
    import torch
    from paper_2607_06763_amd import workloads as W
    seed, T, ctx, Hkv, d, page, dt, tree, nv = case
    print(f"[gpu] commit {case} {where}", flush=True)
    rng = np.random.default_rng(seed)
    if tree == "chain-any":
        par = np.full((len(ctx), T), W.PAD)
        for b in range(len(ctx)):
            s = rng.permutation(T)[:nv[b] if nv else T]
            par[b, s[0]] = -1
            par[b, s[1:]] = s[:-1]
        tree, nv = par, None
    c = Case(seed, T, ctx, Hkv, Hkv, d, page, dt, parent=tree, n_valid=nv)
    c.append_slots()
    acc = np.array([int(np.argmax(c.depth[b])) if where == "deep" else int(rng.choice(np.nonzero(c.real[b])[0]))
                    for b in range(c.B)])
    g = c.device()
    new_len = torch.full((c.B,), -7, dtype=torch.int32, device="cuda")
    st = torch.full((c.B,), -7, dtype=torch.int32, device="cuda")
    A.kv_commit(c.dims(), c.i32(acc), g["table"], g["ctx"], g["kc"], g["vc"], new_len, kv_status=st, meta=g["meta"])
    torch.cuda.synchronize()
    for b in range(c.B):
        path = sorted(np.nonzero(c.vis[b, acc[b]])[0], key=lambda j: c.depth[b, j])
        c.put(b, c.ctx[b] + np.arange(len(path)), c.k[b, path], c.v[b, path])
        assert new_len[b].item() == c.ctx[b] + len(path) and st[b].item() == 0
    assert torch.equal(bits(g["kc"].cpu()), bits(c.kc))
    assert torch.equal(bits(g["vc"].cpu()), bits(c.vc))


def test_commit_nothing_and_bad(A):
    import torch
    from paper_2607_06763_amd import gdn_tree as G
    c = Case(9, 8, [10] * 7, 2, 2, 32, 16, "bf16", parent="any", n_valid=[8, 8, 8, 5, 8, 8, 8])
    c.append_slots()
    c.parent[4, :] = 0  # slot 0 is its own parent
    pad = int(np.nonzero(~c.real[3])[0][0])
    deep = [int(np.argmax(c.depth[b])) for b in range(7)]
    acc = [-1, 8, -2, pad, 0, deep[5], deep[6]]
    g = c.device()
    g["ctx"][5] = -3
    g["table"][6, 0] = -5
    kc, vc = g["kc"].clone(), g["vc"].clone()
    new_len = torch.full((7,), -7, dtype=torch.int32, device="cuda")
    st = torch.full((7,), -7, dtype=torch.int32, device="cuda")
    A.kv_commit(c.dims(), c.i32(acc), g["table"], g["ctx"], g["kc"], g["vc"], new_len, kv_status=st, meta=g["meta"])
    torch.cuda.synchronize()
    bad = G.TREE_BAD_ACCEPTED
    assert st.tolist() == [0, bad, bad, bad, G.TREE_BAD_PARENT, G.KV_BAD_LEN, G.KV_BAD_PAGE]
    assert new_len.tolist() == [10, 10, 10, 10, 10, -3, 10]
    assert torch.equal(bits(g["kc"]), bits(kc)) and torch.equal(bits(g["vc"]), bits(vc))


def test_commit_chain(A):
    """Without metadata nothing moves."""
    import torch
    c = Case(10, 5, [10, 31], 2, 2, 32, 16, "f32")
    c.append_slots()
    g = c.device()
    kc = g["kc"].clone()
    new_len = torch.zeros(2, dtype=torch.int32, device="cuda")
    A.kv_commit(c.dims(), c.i32([2, -1]), g["table"], g["ctx"], g["kc"], g["vc"], new_len)
    assert new_len.tolist() == [13, 31] and torch.equal(bits(g["kc"]), bits(kc))


def test_caches_above_2_31_elements(A):
    """Pages past 2^31 elements (bf16, 4.3 GB a cache) are reached, and their neighbours are not."""
    import torch
    c = Case(11, 12, [40], 2, 2, 128, 16, "bf16", parent="any")
    per = 2 * 128 * 16
    n = 2 ** 31 // per + 64
    far = n - 1 - np.arange(c.max_pages)  # the last pages
    g = c.device()
    shape_k, shape_v = (n, *c.kc.shape[1:]), (n, *c.vc.shape[1:])
    kc, vc = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in (shape_k, shape_v))
    near = c.table[0].copy()
    used = near >= 0
    kc[torch.from_numpy(far[used])], vc[torch.from_numpy(far[used])] = g["kc"][torch.from_numpy(near[used])], g["vc"][torch.from_numpy(near[used])]
    table = c.i32(far[None])
    c.append_slots()
    d = c.dims()
    d.n_pages = n
    d.rot = 0
    qo, out = torch.empty_like(g["q"]), torch.empty_like(g["q"])
    A.kv_append(d, g["q"], g["k"], g["v"], None, g["ctx"], table, kc, vc, qo, meta=g["meta"])
    k, v = A.gather_rows(d, kc, vc, table, 52)
    for i in np.nonzero(c.real[0])[0]:
        assert torch.equal(bits(k[0, 40 + i].cpu()), bits(c.k[0, i])) and torch.equal(bits(v[0, 40 + i].contiguous().cpu()), bits(c.v[0, i]))
    A.attend(d, qo, kc, vc, table, g["ctx"], out, meta=g["meta"])
    ref, mag = c.attend_ref()
    assert np.all(np.abs(out.double().cpu().numpy() - ref) <= 2.0 ** -8 * (mag + np.abs(ref)))
    acc = int(np.argmax(c.depth[0]))
    new_len = torch.empty(1, dtype=torch.int32, device="cuda")
    A.kv_commit(d, c.i32([acc]), table, g["ctx"], kc, vc, new_len, meta=g["meta"])
    path = sorted(np.nonzero(c.vis[0, acc])[0], key=lambda j: c.depth[0, j])
    k, v = A.gather_rows(d, kc, vc, table, 52)
    assert torch.equal(bits(k[0, 40:40 + len(path)].contiguous().cpu()), bits(c.k[0, path]))
    assert torch.equal(bits(v[0, 40:40 + len(path)].contiguous().cpu()), bits(c.v[0, path]))
    assert int((kc[:n - c.max_pages] != 0).sum()) == 0 and int((vc[:n - c.max_pages] != 0).sum()) == 0
