"""gdn_chain against the recurrence in 64 bits (tests/chain_ref.py).

Tolerances.  Activations and norms are off by a few 2^-23 (an exponential of
argument y by |y| 2^-23, |y| below 8 where it matters: 2^-20), a product of the
chunked form by 2^-21 of its operands' norms, and a value passes four products
(the inverse, W, V', the state or output): below 2^-18 = 4e-6 together, held to
1e-5 of the largest output of a head, and to 1e-5 of the state's norm for every
(sequence, head).  A bf16 output is off by at most 2^-8 of itself besides."""
import numpy as np
import pytest

from tests.chain_ref import Chain

pytestmark = pytest.mark.gpu

TOL = 1e-5


@pytest.fixture(scope="module")
def L():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_06763_amd import gdn_layer as L
    return L


def check(c, a, tol=TOL, scale=None):
    import torch
    torch.cuda.synchronize()
    out, S, conv = c.ref(scale)
    got = a["out"].reshape(c.rows, c.Hv, c.dv).double().cpu().numpy()
    assert np.all(got[~c.live] == 7.0)  # rows of no sequence are left as they were
    half = 2.0 ** -8 if c.out_dtype == "bf16" else 0.0
    worst = worst_s = 0.0
    for b in range(c.B):
        r = slice(c.first[b], c.first[b] + c.n[b])
        top = np.abs(out[r]).max(axis=(0, 2), initial=0.0)[None, :, None]
        err = np.abs(got[r] - out[r]) - half * np.abs(out[r])
        worst = max(worst, float((err / np.maximum(top, 1e-30)).max(initial=0.0)))
        assert np.isfinite(got[r]).all() and np.all(err <= tol * top), (b, worst)
        d = a["S"][b].double().cpu().numpy() - S[b]
        rel = np.sqrt((d ** 2).sum((1, 2))) / np.maximum(np.sqrt((S[b] ** 2).sum((1, 2))), 1e-30)
        worst_s = max(worst_s, float(rel.max()))
        assert rel.max() <= tol, (b, rel.max())
        if c.n[b] == 0:
            assert np.array_equal(a["S"][b].cpu().numpy(), c.S[b])
    assert np.array_equal(a["conv_state_out"].cpu().numpy(), conv.astype(np.float32))
    assert a["status"].tolist() == [0] * c.B
    print(f"[gpu]   out {worst:.2e} state {worst_s:.2e} of {tol}", flush=True)


def run(L, c, scale=0.0, tol=TOL):
    print(f"[gpu] chain n={c.n.tolist()} T={c.T} {c.Hk}/{c.Hv} heads {c.dk}x{c.dv} {c.dtype} packed={c.packed}", flush=True)
    a = c.device()
    L.chain(c.dims(scale), **a)
    check(c, a, tol, scale or None)
    return a


CASES = [
    # lengths, Hk, Hv, dk, dv, dtype, out, packed, T
    ([1], 1, 1, 128, 128, "f32", "f32", False, None),
    ([1, 1, 1], 2, 6, 128, 128, "bf16", "bf16", False, None),
    ([4, 0, 3, 1], 2, 4, 64, 64, "f32", "f32", False, None),
    ([16, 2, 9], 1, 3, 32, 16, "bf16", "f32", True, None),
    ([5, 13], 2, 2, 16, 128, "f32", "f32", False, 15),
    ([17], 1, 2, 128, 128, "f32", "f32", False, None),
    ([63, 64, 65], 1, 2, 128, 64, "f32", "f32", False, None),
    ([64, 0, 1, 2, 3], 1, 1, 128, 128, "bf16", "f32", True, None),
    ([200, 0, 67, 1], 2, 6, 64, 32, "f32", "f32", True, None),
    ([129], 1, 4, 32, 128, "f32", "bf16", False, None),
    ([130, 40], 2, 4, 16, 16, "bf16", "f32", False, 150),
    ([100], 1, 7, 128, 16, "f32", "f32", False, None),   # more value heads than are inverted at once, three times
    ([300, 511], 4, 4, 128, 128, "bf16", "bf16", True, None),
    ([1025], 2, 2, 64, 128, "bf16", "f32", False, None),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{'.'.join(map(str, c[0]))}-{c[1]}.{c[2]}-{c[3]}x{c[4]}-{c[5]}-{c[6]}")
def test_against_recurrence(L, case):
    n, Hk, Hv, dk, dv, dt, out, packed, T = case
    run(L, Chain(len(n) * 100 + dk + dv, n, Hk, Hv, dk, dv, dt, out, packed, T))


@pytest.mark.parametrize("n", [9, 150])
@pytest.mark.parametrize("alpha", [1.0, 0.0, 1e-30, 0.01, "mixed"])
def test_decays(L, n, alpha):
    """No decay, a state that is forgotten at every token, and both in turn: differences of far sums of logarithms."""
    if alpha == "mixed":
        rng = np.random.default_rng(n)
        alpha = np.where(rng.random((n, 2)) < 0.2, 10.0 ** -rng.integers(1, 37, (n, 2)), 0.999)
    run(L, Chain(31, [n], 1, 2, 64, 32, alpha=alpha))


@pytest.mark.parametrize("n", [12, 192])
@pytest.mark.parametrize("beta", [0.0, 1.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_keys(L, n, beta, dtype):
    """Keys of a chunk that are all the same (the conv's first tokens aside), written at full strength and without decay:
    the triangular system is as far from the identity as it gets."""
    run(L, Chain(32, [n], 1, 2, 128, 64, dtype, alpha=1.0, beta=beta, same_keys=True))


@pytest.mark.parametrize("state,gain", [(0.0, 1.0), (1e-20, 1e-3), (1e6, 1.0), (1e-3, 30.0), (1e15, 5.0)])
def test_magnitudes(L, state, gain):
    for n in (7, 140):
        run(L, Chain(33, [n], 1, 2, 64, 64, state=state, gain=gain))


def test_scale_and_split_of_a_sequence(L):
    """A sequence in two calls is the sequence in one: the state and the conv state carry over."""
    import torch
    c = Chain(34, [150], 2, 4, 64, 64)
    whole = run(L, c, scale=0.7)
    for cut in (1, 2, 70, 149):
        a = c.device()
        outs = []
        S, conv = a["S"], a["conv_state"]
        for lo, hi in ((0, cut), (cut, 150)):
            d = L.make_chain_dims(1, hi - lo, 2, 4, 64, 64, in_dtype="f32", scale=0.7)
            o, nxt = torch.empty(1, hi - lo, 4, 64, device="cuda"), torch.empty_like(conv)
            L.chain(d, *(a[n][:, lo:hi].contiguous() for n in ("q", "k", "v", "alpha", "beta")), a["conv_w"], conv, nxt, S, o)
            outs.append(o)
            conv = nxt
        torch.cuda.synchronize()
        o = torch.cat(outs, 1)
        top = whole["out"].abs().max()
        assert (o - whole["out"]).abs().max() <= 2 * TOL * top
        assert (S - whole["S"]).norm() <= 2 * TOL * whole["S"].norm()
        assert torch.equal(conv, whole["conv_state_out"])
