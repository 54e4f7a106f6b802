"""Sampling against its definition in whole numbers, every row: the masses are
made with the device's own 32-bit power of two, which is what defines them, and
the cuts and the draw follow in exact sums.  Tokens must be equal; there is no
tolerance and no row is left out."""
import numpy as np
import pytest

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


def masses(z, t):
    """round(2^31 2^((z - max) log2(e) / t)) of rows z [n][V] (fp32 device tensor) with temperatures t [n], as int64."""
    import torch
    z = torch.where(torch.isnan(z), -float("inf"), z)
    top = z.amax(1, keepdim=True)
    c = (torch.ones_like(t) / t)[:, None] * torch.tensor(np.float32(1.44269504088896340736), device="cuda")
    w = torch.floor(torch.exp2((z - top) * c) * 2147483648.0 + 0.5)
    return torch.where(z == top, 2147483648.0, w).long().cpu().numpy()


def token_of(z, w, k, p, least, u):
    """The token of one row: logits z, masses w (both numpy), settings and random number in 32 bits."""
    order = np.lexsort((np.arange(len(z)), -z.astype(np.float64)))
    ws = w[order]
    if k > 0:
        ws[k:] = 0
    ahead = np.cumsum(ws) - ws
    if not p >= 1:
        keep = ahead < float(p) * float(ws.sum())
        keep[0] = True
        ws = np.where(keep, ws, 0)
    ws = np.where(ws >= min(float(least), 1.0) * 2.0 ** 31, ws, 0)
    kept = np.zeros_like(w)
    kept[order] = ws
    cum = np.cumsum(kept)
    return int(np.argmax(cum > float(u) * float(cum[-1])))


def check(A, z, u, settings, rows=None):
    """z [n][V] host tensor, u [n], settings: n of (temperature, top_k, top_p, min_p); rows: those to compare (all)."""
    import torch
    n = z.shape[0]
    t, p, m = (np.array([s[j] for s in settings], np.float32) for j in (0, 2, 3))
    k = [s[1] for s in settings]
    u = np.asarray(u, np.float32)
    zd, tok = z.cuda()[:, None], torch.full((n, 1), -7, dtype=torch.int32, device="cuda")
    A.sample(zd, f32(u)[:, None], tok, temperature=f32(t), top_k=i32(k), top_p=f32(p), min_p=f32(m))
    got = tok[:, 0].tolist()
    rows = np.arange(n) if rows is None else np.sort(rows)
    zf = zd[torch.from_numpy(rows).cuda(), 0].float()
    w, zf = masses(zf, f32(t[rows])), zf.cpu().numpy()
    want = [token_of(zf[j], w[j], k[r], p[r], m[r], u[r]) for j, r in enumerate(rows)]
    bad = [(int(r), settings[r], float(u[r]), got[r], x) for r, x in zip(rows, want) if got[r] != x]
    assert not bad, bad[:5]


@pytest.mark.parametrize("octaves,least", [(31.5, 2.0 ** -31), (31.9, 1e-30), (30.3, 2.0 ** -30), (28.0, 2.0 ** -28),
                                           (29.9, 1.3 * 2.0 ** -31)])
def test_min_p_of_the_smallest_masses(A, octaves, least):
    """A token stays if its whole mass reaches min_p 2^31: with min_p that small, one whose unrounded mass is below it.
    u = 0 draws the first that stays."""
    import torch
    z = torch.full((4, 300), -octaves * float(np.log(2.0)), dtype=torch.float32)
    z[:, 250] = 0.0
    z[1, :100] = -100.0
    z[2, 7] = -1.0
    z[3, :250] = -32.5 * float(np.log(2.0))  # no mass at all
    check(A, z, [0.0, 0.0, 0.0, 0.0], [(1.0, 0, 1.0, least)] * 4)


CUTS = [
    # temperature, top_k, top_p, min_p
    (1.0, 0, 1.0, 0.0), (1.0, 1500, 1.0, 0.0), (1.3, 5000, 1.0, 0.0), (1.0, 1500, 0.9, 0.0), (0.8, 5000, 0.97, 0.0),
    (2.0, 20000, 0.999, 0.0), (1.0, 0, 0.9, 0.0), (0.7, 0, 0.5, 0.0), (3.0, 0, 0.999, 0.0), (1.0, 0, 1.0, 1e-3),
    (1.0, 0, 1.0, 0.2), (1.0, 5000, 0.95, 1e-4), (0.9, 40, 0.95, 0.0), (1.0, 1024, 1.0, 0.0), (1.0, 1025, 0.8, 0.01),
    (30.0, 3000, 0.6, 0.0), (1.0, 0, 1e-6, 0.0), (1.0, 2, 0.99, 0.0),
]


def rows_of(rng, n, V, kind):
    import torch
    z = rng.standard_normal((n, V)).astype(np.float32) * 2
    if kind == "peaked":
        z[np.arange(n)[:, None], rng.integers(0, V, (n, 30))] += 8
    elif kind == "masked":
        z[:, rng.random(V) < 0.6] = -np.inf
        z[:, rng.random(V) < 0.02] = np.finfo(np.float32).min
        z[:, V // 3] = 2.0
    elif kind == "steps":
        z = np.round(z * 4) / 4  # equal logits by the thousand
    return torch.from_numpy(z)


@pytest.mark.parametrize("V", [32768, 50001, 131072])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["plain", "peaked", "masked", "steps"])
def test_wide_rows(A, V, dt, kind):
    """Every cut of a wide vocabulary, with a top_k between the threads of a row and the vocabulary too."""
    import torch
    rng = np.random.default_rng([V, len(kind), dt == "f32", 3])
    print(f"[gpu] sample V={V} {dt} {kind}", flush=True)
    z = rows_of(rng, len(CUTS), V, kind).to(torch.bfloat16 if dt == "bf16" else torch.float32)
    check(A, z, rng.integers(0, 2 ** 24, len(CUTS)) / 2 ** 24, CUTS)


@pytest.mark.parametrize("n,V,dt", [(300, 40000, "f32"), (2100, 17000, "f32"), (600, 9000, "bf16"), (2048, 20001, "bf16")])
def test_many_rows(A, n, V, dt):
    """The thread counts that many rows take."""
    import torch
    rng = np.random.default_rng([n, V])
    print(f"[gpu] sample n={n} V={V} {dt}", flush=True)
    z = rows_of(rng, 60, V, "peaked").to(torch.bfloat16 if dt == "bf16" else torch.float32).repeat(n // 60 + 1, 1)[:n]
    u = np.resize(rng.integers(0, 2 ** 24, 60 * 18) / 2 ** 24, n)
    # the same row with other settings and numbers further down; 200 of all rows are looked at
    settings = [CUTS[(r + r // 60) % len(CUTS)] for r in range(n)]
    check(A, z, u, settings, rows=rng.choice(n, 200, replace=False))
