"""gdn_chain where one token, or the state, is far larger than what follows it and
is forgotten at once: the outputs behind it against the recurrence in 64 bits,
each against the size of the state at its own token.

Tolerances.  N_t: the largest norm of a row of the state behind token t (of a
head); an output is scale times such a row times a unit query.
 * Relative to N_t: activations and norms 2^-20 (an exponential of argument y is
   off by |y| 2^-23, |y| below 8 where it matters), a decay over several tokens
   20 x 2^-23 (e^-20 of what came before is the most that counts here), and four
   products of the chunked form 2^-21 each: below 2^-18 + 2^-18.7 = 6.2e-6
   together, held to 1e-5.
 * Chunked form, relative to M, the largest value or row of the state in this
   chunk or the one before: operands are pairs of fp16 values scaled to
   2^14 .. 2^15, whose last step is 2^-24, so each is off by up to 2^-39 of the
   largest it is scaled by.  With decays of at most 0.8 a row of Y sums to at
   most 1 / (1 - 0.8) = 5 and so do the decays to a chunk's end; a row of
   (I + A)^-1 to less than 3 (A: 0.8 / 0.2 x 0.3 for the largest products of
   random keys, and the sum of its powers with alternating signs).  V' is then
   off by 3 (its operand) + 1 (the inverse, one large value) steps, an output by
   5 x (4 + 1) + 1 = 26 of them, the state by 5 x (4 + 1): below 2^-34 M."""
import numpy as np
import pytest

from tests.chain_ref import Chain

# exp overflows in SiLU of a large negative value, which is then 0 as it should be
pytestmark = [pytest.mark.gpu, pytest.mark.filterwarnings("ignore:overflow encountered in exp")]

TOL, FLOOR = 1e-5, 2.0 ** -34
CHUNK = 64


@pytest.fixture(scope="module")
def L():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_06763_amd import gdn_layer as L
    return L


class Uneven(Chain):
    """Sequences of n tokens: the values of token `at` are `factor` times the others (the short convolution takes a token
    alone), the decay of the token behind it is `reset`, the others 0.5 to 0.8."""

    def __init__(self, seed, B, n, Hk, Hv, dk, dv, at, factor, reset, dtype="f32", state=0.3):
        import torch
        super().__init__(seed, [n] * B, Hk, Hv, dk, dv, dtype, state=state)
        rng = np.random.default_rng([79, seed])
        self.conv_w[:, :3] = 0.0
        self.conv_w[:, 3] = 0.7 + 0.3 * rng.random(self.C)
        a = 0.5 + 0.3 * rng.random((B, n, Hv))
        if reset is not None and at + 1 < n:
            a[:, at + 1] = reset
        self.alpha = torch.from_numpy(a.reshape(-1, Hv)).to(self.alpha.dtype)
        v = self.v.reshape(B, n, Hv, dv)
        if at >= 0:
            v[:, at] *= factor
        self.v = v.reshape(-1, Hv, dv)

    def sizes(self):
        """N [B][n][Hv] and M [B][n][Hv]."""
        B, n, Hk, Hv, dk, dv = self.B, self.T, self.Hk, self.Hv, self.dk, self.dv
        silu = lambda x: x / (1 + np.exp(-x))
        w = self.conv_w[:, 3].astype(np.float64)
        f = lambda t, lo, *shape: silu(t.double().numpy().reshape(B, n, -1) * w[lo:lo + t[0].numel()]).reshape(B, n, *shape)
        k = f(self.k, Hk * dk, Hk, dk)
        k = np.repeat(k / np.sqrt((k * k).sum(-1, keepdims=True) + 1e-6), Hv // Hk, axis=2)
        v = f(self.v, 2 * Hk * dk, Hv, dv)
        al, be = (t.double().numpy().reshape(B, n, Hv, 1) for t in (self.alpha, self.beta))
        S = self.S.astype(np.float64)
        row = lambda: np.sqrt((S * S).sum(-1)).max(-1)
        N, start = np.zeros((B, n, Hv)), [row()]
        for t in range(n):
            Sk = (S * k[:, t, :, None]).sum(-1)
            S = al[:, t, :, :, None] * S + (be[:, t] * (v[:, t] - al[:, t] * Sk))[..., None] * k[:, t, :, None]
            N[:, t] = row()
            if t % CHUNK == CHUNK - 1:
                start.append(row())
        M = np.zeros((B, n, Hv))
        of = [np.maximum(np.abs(v[:, c:c + CHUNK]).max((1, 3)), start[c // CHUNK]) for c in range(0, n, CHUNK)]
        for c in range(len(of)):
            M[:, c * CHUNK:(c + 1) * CHUNK] = np.maximum(of[c], of[max(c - 1, 0)])[:, None]
        return N, M


def check(L, c):
    import torch
    from paper_2607_06763_amd import gdn_layer
    a = c.device()
    L.chain(c.dims(), **a)
    torch.cuda.synchronize()
    out, S, conv = c.ref()
    N, M = c.sizes()
    floor = 0.0 if c.T <= gdn_layer.STEP_T else FLOOR
    got = a["out"].double().cpu().numpy()
    err = np.abs(got - out.reshape(got.shape)).max(-1) * c.dk ** 0.5  # [B][n][Hv], the scale taken out
    rel = (err - floor * M) / N
    worst = np.unravel_index(np.argmax(err / N), err.shape)
    print(f"[gpu]   worst output {err[worst] / N[worst]:.2e} of the state at token {worst[1]}", flush=True)
    d = a["S"].double().cpu().numpy() - S
    rows = np.sqrt((d * d).sum(-1)).max(-1)
    print(f"[gpu]   state {(rows / N[:, -1]).max():.2e}", flush=True)
    assert np.isfinite(got).all()
    assert rel.max() <= TOL, rel.max()
    assert np.all(rows <= TOL * N[:, -1] + floor * M[:, -1])


# B, heads, dims: pairs of waves (one and two a workgroup), then 2, 4 and 8 waves
FORMS = [(1, 1, 2, 64, 64), (1, 2, 2, 128, 128), (9, 2, 8, 32, 64), (18, 2, 16, 16, 32), (9, 4, 8, 64, 128), (9, 8, 16, 128, 128)]


@pytest.mark.parametrize("reset", [None, 1e-30, 0.0])
@pytest.mark.parametrize("factor", [1e2, 1e4, 1e6])
@pytest.mark.parametrize("n,at", [(20, 0), (20, 12), (150, 0), (150, 40), (150, 62), (150, 63), (129, 64)])
def test_one_large_token(L, n, at, factor, reset):
    print(f"[gpu] chain of {n} tokens, token {at} {factor:g} times the others, then {reset}", flush=True)
    check(L, Uneven(801 + at, 1, n, 1, 2, 64, 64, at, factor, reset))


@pytest.mark.parametrize("form", FORMS, ids=lambda f: ".".join(map(str, f)))
@pytest.mark.parametrize("at", [5, 62])
def test_one_large_token_in_every_form(L, form, at):
    B, Hk, Hv, dk, dv = form
    print(f"[gpu] chain of {B} sequences of 100 tokens, heads {form}, token {at} large", flush=True)
    check(L, Uneven(821 + at, B, 100, Hk, Hv, dk, dv, at, 1e5, 1e-30, "bf16" if at == 5 else "f32"))


@pytest.mark.parametrize("form", FORMS[1:4:2], ids=lambda f: ".".join(map(str, f)))
@pytest.mark.parametrize("n", [20, 100])
def test_large_state(L, form, n):
    B, Hk, Hv, dk, dv = form
    print(f"[gpu] chain of {B} sequences of {n} tokens, heads {form}, a large state", flush=True)
    check(L, Uneven(841, B, n, Hk, Hv, dk, dv, -1, 1.0, None, state=1e5))


@pytest.mark.parametrize("n", [20, 64, 100])
def test_gates_above_one(L, n):
    """1.06 a token, which the header's (0, 1] leaves out: Y reaches 1.06^63 = 39 times what decays allow, and stays in its
    operands' range.  Held to the other tests' tolerance, relative to the largest output of a head."""
    from tests.test_chain_gpu import run
    run(L, Chain(861, [n], 1, 2, 64, 32, alpha=1.06))
