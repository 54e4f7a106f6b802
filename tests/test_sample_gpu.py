"""Sampling and acceptance against their definitions.

The masses of tokens are whole numbers made from 32-bit powers of two, which
the 64-bit reference rounds differently in the last unit: a token's mass may
be off by about 2^-22 of itself.  Rows whose draw (or top_p / min_p
threshold) lies within 1e-5 of the whole mass from a boundary are therefore
left out of the comparison with the reference; the random numbers that are
drawn for a row are checked for it, and few rows may be left out."""
import numpy as np
import pytest

from tests.attn_ref import closure, random_tree, sample_ref

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


def f32(a):
    import torch
    return torch.from_numpy(np.asarray(a, np.float32)).cuda()


def i32(a):
    import torch
    return torch.from_numpy(np.asarray(a, np.int32)).cuda()


def logits(rng, B, T, V, kind):
    z = rng.standard_normal((B, T, V)) * 2
    if kind == "peaked":
        z[..., rng.integers(0, V, 5)] += 9
    elif kind == "masked":
        z[..., rng.random(V) < 0.7] = -np.inf
        z[..., rng.random(V) < 0.05] = np.nan
        z[..., V // 2] = 1.0
    elif kind == "equal":
        z[:] = 0.75
    elif kind == "steps":
        z = np.round(z * 2) / 2  # many equal logits
    return z.astype(np.float32)


SETTINGS = [
    # temperature, top_k, top_p, min_p
    (1.0, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (0.7, 40, 1.0, 0.0), (1.0, 1, 1.0, 0.0), (1.3, 0, 0.9, 0.0),
    (0.9, 0, 0.3, 0.0), (1.0, 0, 1.0, 0.05), (0.8, 50, 0.95, 0.02), (1.0, 7, 0.5, 0.5), (2.0, 10 ** 6, 0.999, 0.0),
    (1e-4, 0, 0.9, 0.0), (50.0, 3, 0.7, 1.0),
]


@pytest.mark.parametrize("V", [1, 2, 7, 64, 1000, 8191, 32768, 131072])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["plain", "peaked", "masked", "equal", "steps"])
def test_sample(A, V, dt, kind):
    import torch
    rng = np.random.default_rng([V, len(kind), dt == "f32"])
    B, T = len(SETTINGS), 3 if V < 10000 else 1
    print(f"[gpu] sample V={V} {dt} {kind}", flush=True)
    z = torch.from_numpy(logits(rng, B, T, V, kind)).to(torch.bfloat16 if dt == "bf16" else torch.float32)
    u = rng.integers(0, 2 ** 24, (B, T)).astype(np.float32) / 2 ** 24
    t, k, p, m = (np.array([s[n] for s in SETTINGS]) for n in range(4))
    tok = torch.full((B, T), -7, dtype=torch.int32, device="cuda")
    A.sample(z.cuda(), f32(u), tok, temperature=f32(t), top_k=i32(k), top_p=f32(p), min_p=f32(m))
    torch.cuda.synchronize()
    got, z = tok.cpu().numpy(), z.float().numpy()
    left = 0
    for b in range(B):
        for i in range(T):
            want, far, near = sample_ref(z[b, i], float(np.float32(t[b])), int(k[b]), float(np.float32(p[b])),
                                         float(np.float32(m[b])), float(u[b, i]))
            if far < 1e-5 or near:
                left += 1
                assert 0 <= got[b, i] < V
                continue
            assert got[b, i] == want, (b, i, SETTINGS[b], got[b, i], want)
    # wide vocabularies without a cut have boundaries everywhere
    print(f"[gpu]   {left} of {B * T} rows too near a boundary", flush=True)
    assert left <= B * T // 2 or kind in ("equal", "steps") or V >= 8191


def test_defaults_and_rows_apart(A):
    """No settings: the plain distribution; rows may be further apart than V, at any alignment."""
    import torch
    rng = np.random.default_rng(5)
    for V, ld, dt in ((1001, 1009, "f32"), (777, 780, "bf16"), (513, 513, "bf16")):
        full = torch.full((4, 3, ld), 50.0)  # what lies between the rows is not read as a logit
        full[..., :V] = torch.from_numpy(logits(rng, 4, 3, V, "peaked"))
        full = full.to(torch.bfloat16 if dt == "bf16" else torch.float32).cuda()
        z = full[..., :V]
        u = rng.integers(0, 2 ** 24, (4, 3)).astype(np.float32) / 2 ** 24
        tok = torch.empty((4, 3), dtype=torch.int32, device="cuda")
        A.sample(z, f32(u), tok)
        got = tok.cpu().numpy()
        for b in range(4):
            for i in range(3):
                want, far, _ = sample_ref(z[b, i].float().cpu().numpy(), 1.0, 0, 1.0, 0.0, float(u[b, i]))
                assert far < 1e-5 or got[b, i] == want


def test_rows_without_a_token_and_infinities(A):
    import torch
    z = np.full((1, 5, 300), -np.inf, np.float32)
    z[0, 1, 17] = -3.0e38               # one token, far below zero
    z[0, 2, [5, 9, 200]] = np.inf       # share the mass
    z[0, 3] = np.nan
    z[0, 4, 299] = np.finfo(np.float32).min
    u = np.array([[0.5, 0.99, 0.5, 0.5, 0.0]], np.float32)
    for t in (0.0, 1.0, 1e-30, 1e30, np.inf):
        for k, p in ((0, 1.0), (2, 1.0), (0, 0.5), (300, 0.9)):
            tok = torch.full((1, 5), -7, dtype=torch.int32, device="cuda")
            A.sample(torch.from_numpy(z).cuda(), f32(u), tok, temperature=f32([t]), top_k=i32([k]), top_p=f32([p]))
            got = tok.tolist()[0]
            assert got[0] == -1 and got[1] == 17 and got[3] == -1 and got[4] == 299
            # the middle one of two or three equal shares
            assert got[2] == (5 if t == 0 else 9), (t, k, p)


def test_ends_of_u(A):
    """u = 0 gives the first token that stays, u just below (or at) 1 the last."""
    import torch
    z = np.zeros((1, 3, 100), np.float32)
    z[..., [0, 1, 99]] = -np.inf
    tok = torch.empty((1, 3), dtype=torch.int32, device="cuda")
    A.sample(torch.from_numpy(z).cuda(), f32([[0.0, 1 - 2.0 ** -24, 1.0]]), tok)
    assert tok.tolist() == [[2, 98, 98]]


def test_padding_slots_are_not_read(A):
    import torch
    from paper_2607_06763_amd import gdn_tree as G
    rng = np.random.default_rng(8)
    par = np.stack([random_tree(rng, 9, 5, "any"), random_tree(rng, 9, 9, "any"), np.full(9, -1)])
    meta = torch.zeros(G.meta_bytes(3, 9), dtype=torch.uint8, device="cuda")
    G.prepare(G.make_dims(3, 9, 1, 1, 16, 16), i32(par), meta)
    z = torch.from_numpy(logits(rng, 3, 9, 400, "plain")).cuda()
    u = f32(rng.random((3, 9)))
    tok, all_ = (torch.empty((3, 9), dtype=torch.int32, device="cuda") for _ in range(2))
    A.sample(z, u, tok, meta=meta)
    A.sample(z, u, all_)
    got, want = tok.cpu().numpy(), all_.cpu().numpy()
    want[par == -2] = -1
    want[2] = -1  # several roots
    assert np.array_equal(got, want)


def test_distribution(A):
    """Counts of 40000 draws against the softmax of what stays (chi-square over 12 tokens: 99.99 % below 39)."""
    import torch
    rng = np.random.default_rng(9)
    z = rng.standard_normal(12).astype(np.float32) * 1.5
    n, T = 80, 500
    u = torch.rand((n, T), device="cuda", generator=torch.Generator("cuda").manual_seed(4))
    tok = torch.empty((n, T), dtype=torch.int32, device="cuda")
    A.sample(torch.from_numpy(np.broadcast_to(z, (n, T, 12)).copy()).cuda(), u, tok, temperature=f32(np.full(n, 0.8)))
    got = np.bincount(tok.cpu().numpy().ravel(), minlength=12)
    e = np.exp((z.astype(np.float64) - z.max()) / 0.8)
    e = e / e.sum() * n * T
    assert ((got - e) ** 2 / e).sum() < 39


def accept_ref(parent, draft, token):
    B, T = parent.shape
    acc, n, out = [], [], np.full((B, T), -1)
    for b in range(B):
        node = [i for i in range(T) if parent[b, i] == -1]
        if len(node) != 1:
            acc.append(-1), n.append(0)
            continue
        node, e = node[0], []
        while True:
            nxt = [i for i in range(T) if parent[b, i] == node and draft[b, i] == token[b, node] and draft[b, i] >= 0]
            if not nxt:
                break
            node = nxt[0]
            e.append(draft[b, node])
        e.append(token[b, node])
        out[b, :len(e)] = e
        acc.append(node), n.append(len(e))
    return acc, n, out


@pytest.mark.parametrize("T", [1, 2, 9, 64, 65, 200, 512])
@pytest.mark.parametrize("chain", [False, True])
def test_accept(A, T, chain):
    import torch
    from paper_2607_06763_amd import gdn_tree as G
    rng = np.random.default_rng([T, chain])
    B = 12
    print(f"[gpu] accept T={T} chain={chain}", flush=True)
    if chain:
        par = np.broadcast_to(np.arange(T) - 1, (B, T)).copy()
    else:
        par = np.stack([random_tree(rng, T, int(rng.integers(1, T + 1)), "any") for _ in range(B)])
        par[1, :] = -2
        if T > 1:
            par[2, :] = -1
    draft = rng.integers(0, 2 if T < 100 else 1, (B, T))  # few tokens: equal siblings and long walks
    token = rng.integers(0, 2 if T < 100 else 1, (B, T))
    token[3:6][rng.random((3, T)) < 0.1] = -1
    draft[4:7][rng.random((3, T)) < 0.1] = -1
    meta = None
    if not chain:
        meta = torch.zeros(G.meta_bytes(B, T), dtype=torch.uint8, device="cuda")
        G.prepare(G.make_dims(B, T, 1, 1, 16, 16), i32(par), meta)
    acc, n = (torch.full((B,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    em = torch.full((B, T), -7, dtype=torch.int32, device="cuda")
    A.accept(i32(draft), i32(token), acc, n, em, meta=meta)
    torch.cuda.synchronize()
    wa, wn, we = accept_ref(par, draft, token)
    assert acc.tolist() == wa and n.tolist() == wn and np.array_equal(em.cpu().numpy(), we)
