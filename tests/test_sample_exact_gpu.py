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


def check(A, z, u, settings):
    """z [n][V] host tensor, u [n], settings: n of (temperature, top_k, top_p, min_p)."""
    import torch
    n = z.shape[0]
    t, p, m = (np.array([s[j] for s in settings], np.float32) for j in (0, 2, 3))
    k = [s[1] for s in settings]
    u = np.asarray(u, np.float32)
    zd, tok = z.cuda()[:, None], torch.full((n, 1), -7, dtype=torch.int32, device="cuda")
    A.sample(zd, f32(u)[:, None], tok, temperature=f32(t), top_k=i32(k), top_p=f32(p), min_p=f32(m))
    got = tok[:, 0].tolist()
    zf = zd[:, 0].float()
    w, zf = masses(zf, f32(t)), zf.cpu().numpy()
    want = [token_of(zf[r], w[r], k[r], p[r], m[r], u[r]) for r in range(n)]
    bad = [(r, settings[r], float(u[r]), got[r], want[r]) for r in range(n) if got[r] != want[r]]
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
