"""Attention of a step's slots over the paged cache against its definition in
64 bits.

Tolerances, per value, with A = sum_j p_j |v_j| and o the exact output: in
bf16 the weights enter the second product rounded to 8 significant bits (at
most 2^-8 A) and the output is rounded once (2^-8 |o|): 2^-8 (A + |o|).  In fp32 a score is a sum of d <= 256
products whose magnitudes sum to about 10 here, off by at most about
16 roundings of 2^-24 of that (1e-5), which moves a weight by as much:
2e-5 A."""
import numpy as np
import pytest

from tests.attn_ref import Case, random_tree
from tests.guard import check_guards, guarded

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


def run(A, c, g=None, scale=0.0, out=None, stream=None):
    import torch
    g = g or c.device()
    out = torch.full_like(g["q"], float("nan")) if out is None else out
    A.attend(c.dims(scale), g["q"], g["kc"], g["vc"], g["table"], g["ctx"], out, meta=g["meta"], n_new=g["n_new"], stream=stream)
    return out


def check(c, out, ref=None, rows=None):
    ref, mag = ref or c.attend_ref()
    got = out.double().cpu().numpy()
    tol = 2.0 ** -8 * (mag + np.abs(ref)) if c.dtype == "bf16" else 2e-5 * mag
    err = np.abs(got - ref)
    worst = float(np.max(err / np.maximum(tol, 1e-30)))
    print(f"[gpu]   worst error / tolerance {worst:.3f}", flush=True)
    assert np.all(err <= tol)
    assert np.all(got[~c.real] == 0)


CASES = [
    # seed, T, ctx, Hq, Hkv, d, page, dtype, tree, valid nodes
    (1, 1, [0], 1, 1, 32, 16, "bf16", None, None),
    (2, 1, [0], 1, 1, 32, 16, "f32", None, None),
    (3, 1, [700], 32, 8, 128, 64, "bf16", None, None),
    (4, 1, [63, 64, 65, 1, 2000], 12, 2, 128, 64, "bf16", None, None),
    (5, 1, [5000], 8, 1, 256, 128, "bf16", None, None),
    (6, 1, [130, 31, 0, 1], 16, 2, 64, 16, "f32", None, None),
    (7, 1, [1500], 16, 1, 256, 32, "f32", None, None),
    (8, 5, [40, 0], 24, 4, 256, 16, "bf16", "any", None),
    (9, 16, [100, 515, 3], 8, 2, 128, 64, "bf16", "any", [16, 0, 7]),
    (10, 64, [300, 1200], 8, 2, 128, 64, "bf16", "any", [64, 50]),
    (11, 99, [1000, 17], 16, 4, 64, 16, "f32", "any", [99, 70]),
    (12, 128, [257], 16, 4, 128, 32, "bf16", "up", None),
    (13, 130, [77], 6, 1, 256, 256, "bf16", "any", [101]),
    (14, 512, [100], 4, 2, 64, 64, "bf16", "any", None),
    (15, 512, [0, 333], 4, 1, 128, 128, "bf16", None, None),
    (16, 200, [50], 5, 5, 32, 32, "bf16", "any", None),
    (17, 33, [64], 3, 3, 32, 256, "f32", "up", None),
    (18, 2, [9000], 4, 2, 128, 16, "bf16", "any", None),
    (19, 1, [100] * 40, 7, 1, 64, 64, "bf16", None, None),
    (20, 70, [63], 1, 1, 128, 64, "f32", None, None),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}-T{c[1]}-H{c[3]}.{c[4]}-d{c[5]}-p{c[6]}-{c[7]}")
def test_attend(A, case):
    import torch
    seed, T, ctx, Hq, Hkv, d, page, dt, tree, nv = case
    print(f"[gpu] attend {case}", flush=True)
    c = Case(seed, T, ctx, Hq, Hkv, d, page, dt, parent=tree, n_valid=nv)
    c.append_slots()
    out = run(A, c)
    torch.cuda.synchronize()
    check(c, out)


def test_prompt_chunks(A):
    """Chains with n_new: slots past it are padding."""
    import torch
    c = Case(30, 40, [0, 90, 5, 64], 8, 2, 64, 32, "bf16", n_new=[40, 1, 0, 33])
    c.append_slots()
    out = run(A, c)
    torch.cuda.synchronize()
    check(c, out)


def test_scale(A):
    c = Case(31, 3, [50], 4, 2, 64, 16, "f32", parent="any")
    c.append_slots()
    check(c, run(A, c, scale=0.31), c.attend_ref(scale=np.float32(0.31)))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,ctx", [(9, 30), (150, 64), (64, 1000)])
def test_what_is_masked_does_not_matter(A, dt, T, ctx):
    """NaN and infinities in rows that a query does not see leave its output as it was, bit for bit, and reach
    the queries that see them."""
    import torch
    c = Case(40, T, [ctx], 8, 2, 64, 16, dt, parent="any", n_valid=[T - 2])
    c.append_slots()
    clean = run(A, c)
    rng = np.random.default_rng(3)
    hit = rng.choice(np.nonzero(c.real[0])[0], 3, replace=False)
    for what in (np.nan, np.inf, -np.inf):
        for which in "kv":
            c2 = Case(40, T, [ctx], 8, 2, 64, 16, dt, parent="any", n_valid=[T - 2])
            for j in hit:
                getattr(c2, which)[0, j, :, 5] = what
            c2.append_slots()
            got = run(A, c2)
            torch.cuda.synchronize()
            sees = c.vis[0][:, hit].any(1)
            print(f"[gpu] masked {dt} T={T} {which} {what}: {int(sees.sum())} of {T} see it", flush=True)
            assert torch.equal(bits(got[0, ~sees]), bits(clean[0, ~sees]))
            if what != what:
                seen = torch.from_numpy(np.nonzero(sees)[0])
                bad = got[0, seen].float().cpu()
                assert torch.isnan(bad[..., 5]).all() if which == "v" else torch.isnan(bad).all()
                if which == "v":
                    keep = [e for e in range(64) if e != 5]
                    assert torch.equal(bits(got[0, seen][..., keep].contiguous()), bits(clean[0, seen][..., keep].contiguous()))
            elif which == "v":
                seen = torch.from_numpy(np.nonzero(sees)[0])
                assert not torch.isfinite(got[0, seen][..., 5].float()).any()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_extreme_scores(A, dt):
    """Scores of thousands (either sign), equal scores, and keys of the type's lowest and largest values."""
    import torch
    c = Case(41, 20, [200, 70], 8, 2, 128, 64, dt, parent="any")
    c.q *= 60.0
    for b in range(2):
        c.hist[b][0].mul_(20.0)
        c.hist[b][0][3] = 0.0
        c.hist[b][1][7] *= 1e30  # values near the end of the range at small weights
        c.put(b, np.arange(int(c.ctx[b])), *c.hist[b])
    c.append_slots()
    ref, mag = c.attend_ref()
    out = run(A, c)
    torch.cuda.synchronize()
    got = out.double().cpu().numpy()
    # scores of magnitude M are off by 2^-24 M times the roundings of their sum, and so are the weights' exponents
    M = 60 * 20 * 8.0
    tol = (2.0 ** -8 if dt == "bf16" else 0) * (mag + np.abs(ref)) + 64 * 2.0 ** -24 * M * mag
    assert np.all(np.abs(got - ref) <= tol)


def test_missing_pages_and_bad_sequences(A):
    """Entries outside the cache are left out; a bad length or tree clears the sequence's outputs."""
    import torch
    c = Case(42, 6, [100, 100, 100, 100, 100], 4, 2, 64, 16, "bf16", parent="any")
    c.append_slots()
    c.parent[4, :] = 1  # slot 1 is its own parent
    g = c.device()
    g["ctx"][2] = -1
    g["ctx"][3] = c.max_pages * c.page - 3
    g["table"][0, 2] = c.n_pages
    g["table"][0, 4] = -2 ** 31
    g["table"][1, :] = 2 ** 31 - 1  # nothing is left
    out = run(A, c, g)
    torch.cuda.synchronize()
    ref, mag = c.attend_ref(missing=[(0, 2), (0, 4)] + [(1, p) for p in range(c.max_pages)])
    got = out.double().cpu().numpy()
    assert np.all(np.abs(got[0] - ref[0]) <= 2.0 ** -8 * (mag[0] + np.abs(ref[0])))
    assert np.all(got[1:] == 0)


def test_guards_repeats_and_streams(A):
    """Nothing is written around out, equal calls give equal bits, also on other streams at once."""
    import torch
    for dt in ("f32", "bf16"):
        c = Case(43, 31, [600, 40], 12, 2, 128, 64, dt, parent="any")
        c.append_slots()
        g = c.device()
        want = run(A, c, g)
        if dt == "f32":
            out, full = guarded(tuple(g["q"].shape))
            run(A, c, g, out=out)
            torch.cuda.synchronize()
            check_guards(full, "out")
            assert torch.equal(bits(out), bits(want))
        streams = [torch.cuda.Stream() for _ in range(3)]
        outs = []
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                outs.append([run(A, c, g) for _ in range(3)])
        other = run(A, c, g, stream=streams[0])
        torch.cuda.synchronize()
        for o in [o for l in outs for o in l] + [other]:
            assert torch.equal(bits(o), bits(want))


def test_graph(A):
    """A captured append + attend + commit replays with new lengths and contents."""
    import torch
    c = Case(44, 12, [300, 64, 0], 8, 2, 64, 32, "bf16", parent="any")
    g = c.device()
    d = c.dims()
    qo, out = torch.empty_like(g["q"]), torch.empty_like(g["q"])
    acc = c.i32([int(np.argmax(c.depth[b])) for b in range(3)])
    new_len = torch.empty(3, dtype=torch.int32, device="cuda")

    def step():
        A.kv_append(d, g["q"], g["k"], g["v"], g["rope"], g["ctx"], g["table"], g["kc"], g["vc"], qo, meta=g["meta"])
        A.attend(d, qo, g["kc"], g["vc"], g["table"], g["ctx"], out, meta=g["meta"])
        A.kv_commit(d, acc, g["table"], g["ctx"], g["kc"], g["vc"], new_len, meta=g["meta"])

    s = torch.cuda.Stream()
    kc0, vc0 = g["kc"].clone(), g["vc"].clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        step()  # the workspace belongs to the stream: allocated before the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    for n in range(4):
        g["ctx"].copy_(c.i32(np.maximum(0, c.ctx - 7 * n)))
        g["q"].copy_(torch.randn_like(g["q"], dtype=torch.float32).to(g["q"].dtype))
        g["kc"].copy_(kc0), g["vc"].copy_(vc0)
        step()
        torch.cuda.synchronize()
        eager = [t.clone() for t in (out, g["kc"], g["vc"], new_len)]
        g["kc"].copy_(kc0), g["vc"].copy_(vc0)
        out.fill_(float("nan"))
        new_len.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, (out, g["kc"], g["vc"], new_len)):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_one_token_at_a_time_is_the_chain(A):
    """Appending and attending token by token gives what one chain call gives."""
    import torch
    c = Case(45, 9, [70], 4, 2, 128, 16, "f32")
    g = c.device()
    d = c.dims()
    qo, out = torch.empty_like(g["q"]), torch.empty_like(g["q"])
    A.kv_append(d, g["q"], g["k"], g["v"], g["rope"], g["ctx"], g["table"], g["kc"], g["vc"], qo)
    A.attend(d, qo, g["kc"], g["vc"], g["table"], g["ctx"], out)
    one = Case(45, 9, [70], 4, 2, 128, 16, "f32")
    h = one.device()
    e = one.dims()
    e.T = 1
    for t in range(9):
        ctx = one.i32([70 + t])
        q1, k1, v1 = (h[n][:, t:t + 1].contiguous() for n in "qkv")
        o1 = torch.empty_like(q1)
        A.kv_append(e, q1, k1, v1, h["rope"], ctx, h["table"], h["kc"], h["vc"], q1)
        A.attend(e, q1, h["kc"], h["vc"], h["table"], ctx, o1)
        err = (o1[:, 0] - out[:, t]).abs().max().item()
        assert err <= 4e-5 * 4, (t, err)  # both within 2e-5 A of the exact output, A below 4
    torch.cuda.synchronize()
