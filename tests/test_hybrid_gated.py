"""The decode loop of a model with norms and gates around its blocks, and prompts
through the chain form, against the model's definition in 64-bit numpy.

Tolerances.  A GDN output is off by at most 2e-3 of the largest of its call (the
tree form's own tests), about 3 standard deviations: 6e-3 of a head's root mean
square, and so is what the head's norm, the gate and the norm behind the
projection make of it.  Half of that is added to a hidden vector that grows to
1.4 per component: two such layers move the logits (gain 3) by
3 x 0.5 x 6e-3 x sqrt(2) / 1.4 = 0.01 and a boundary of the distribution
function by twice that, held to 0.03.  In bf16 the four layers' inputs are
rounded (2^-8, in q, k and v: 2^-7 of a block): 3 x 0.5 x 2^-7 x 2 / 1.4 = 0.017
from four of them, the attention's own rounding as much again, the boundary
twice: held to 0.1."""
import numpy as np
import pytest

from paper_2607_06763_amd import hybrid_decode as H


def gdn_layer(q, k, v, alpha, beta, cw):
    n, Hk, dk = q.shape
    Hv, dv = v.shape[1:]
    raw = np.concatenate([np.zeros((3, cw.shape[0])), np.concatenate([a.reshape(n, -1) for a in (q, k, v)], 1)])
    y = sum(raw[w:w + n] * cw[:, w] for w in range(4))
    y = y / (1 + np.exp(-y))
    q, k, v = (a.reshape(n, -1, d) for a, d in zip(np.split(y, [Hk * dk, 2 * Hk * dk], axis=1), (dk, dk, dv)))
    q, k = (np.repeat(a / np.sqrt((a * a).sum(-1, keepdims=True) + 1e-6), Hv // Hk, axis=1) for a in (q, k))
    S, out = np.zeros((Hv, dv, dk)), np.zeros((n, Hv, dv))
    for t in range(n):
        a, b = alpha[t][:, None], beta[t][:, None]
        S = a[:, :, None] * S + (b * (v[t] - a * np.einsum("hvd,hd->hv", S, k[t])))[:, :, None] * k[t][:, None]
        out[t] = np.einsum("hvd,hd->hv", S, q[t]) * dk ** -0.5
    return out


def reference_logits(m, tokens):
    n = len(tokens)
    f64 = lambda a: a.astype(np.float64)
    norm = lambda a: a / np.sqrt(np.mean(a * a, axis=-1, keepdims=True) + H.EPS)
    unit = lambda a: a / np.linalg.norm(a, axis=-1, keepdims=True)
    x = f64(m.embed[tokens])
    for kind, w in zip(m.kinds, m.layers):
        y = norm(x) * (f64(w["norm"]) if m.gated else 1.0)
        p = {c: y @ f64(w[c]).T for c in ("q", "k", "v", "alpha", "beta", "z") if c in w}
        if kind == "gdn":
            out = gdn_layer(unit(p["q"].reshape(n, m.Hk, m.dk)), unit(p["k"].reshape(n, m.Hk, m.dk)), p["v"].reshape(n, m.Hv, m.dv),
                            np.exp(-np.logaddexp(0, p["alpha"])), 1 / (1 + np.exp(-p["beta"])), f64(w["conv_w"]))
            if m.gated:
                z = p["z"].reshape(n, m.Hv, m.dv)
                out = norm(out) * f64(w["head"]) * z / (1 + np.exp(-z))
        else:
            q, k, v = (p[c].reshape(n, -1, m.d) for c in "qkv")
            cs, half = f64(m.rope[:n])[:, None], m.rot // 2
            turn = lambda a: np.concatenate([a[..., :half] * cs[..., 0] - a[..., half:m.rot] * cs[..., 1],
                                             a[..., half:m.rot] * cs[..., 0] + a[..., :half] * cs[..., 1], a[..., m.rot:]], -1)
            q, k = turn(q), turn(k)
            out = np.zeros((n, m.Hq, m.d))
            for h in range(m.Hq):
                g = h // (m.Hq // m.Hkv)
                s = np.where(np.tril(np.ones((n, n), bool)), q[:, h] @ k[:, g].T * m.d ** -0.5, -np.inf)
                e = np.exp(s - s.max(axis=1, keepdims=True))
                out[:, h] = e / e.sum(axis=1, keepdims=True) @ v[:, g]
        block = out.reshape(n, -1) @ f64(w["o"]).T
        x = x + (f64(w["scale"]) * f64(w["post"]) * norm(block) if m.gated else block)
    return norm(x) * (f64(m.final) if m.gated else 1.0) @ f64(m.unembed).T


def test_weights_do_not_depend_on_the_gates():
    a, b = H.HybridModel(seed=5), H.HybridModel(seed=5, gated=True)
    assert not a.gated and b.gated and np.array_equal(a.unembed, b.unembed)
    for x, y in zip(a.layers, b.layers):
        assert all(np.array_equal(x[n], y[n]) for n in x) and {"norm", "post", "scale"} <= set(y)


def test_unknown_prompt_form():
    with pytest.raises(ValueError):
        H.Decoder(H.HybridModel(), 1, 4, np.zeros((1, 8), np.float32), prompt_form="list")


RUNS = [
    # seed, layers, slots, dtype, temperature, gated, prompt form
    (21, ("gdn", "attn", "gdn", "attn"), 24, "f32", 1.0, True, "chain"),
    (22, ("gdn", "attn", "gdn", "attn"), 1, "f32", 0.8, True, "chain"),
    (23, ("attn", "gdn", "gdn", "attn"), 32, "bf16", 1.0, True, "chain"),
    (24, ("gdn", "attn", "gdn", "attn"), 16, "f32", None, True, "tree"),
    (25, ("gdn", "attn", "attn", "gdn"), 20, "f32", 1.0, False, "chain"),
    (26, ("gdn",), 8, "f32", 0.0, True, "chain"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("run", RUNS, ids=lambda r: f"{r[0]}-{'.'.join(r[1])}-T{r[2]}-{r[3]}-{'gated' if r[5] else 'plain'}-{r[6]}")
def test_tokens_are_samples_of_the_model(run):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    seed, layers, T, dtype, temp, gated, form = run
    rng = np.random.default_rng([9, seed])
    m = H.HybridModel(seed=seed, layers=layers, positions=700, gated=gated)
    B, want = 3, 20
    # a prompt of one token has none for the layers to read; one goes in two pieces of at most 512
    prompts = [[int(t) for t in rng.integers(0, m.V, n)] for n in ((1, 90, 17) if seed != 21 else (1, 600, 33))]
    u = rng.random((B, 700), dtype=np.float32)
    dec = H.Decoder(m, B, T, u, max_pages=44, dtype=dtype, temperature=temp, prompt_form=form)
    print(f"[gpu] hybrid decode {run}", flush=True)
    seqs, steps = H.decode(dec, prompts, want)
    torch.cuda.synchronize()
    assert all(s[:len(p)] == p for s, p in zip(seqs, prompts))
    tol, worst = (0.03 if dtype == "f32" else 0.1), 0.0
    for b, (s, p) in enumerate(zip(seqs, prompts)):
        z = reference_logits(m, s[:-1])
        for i in range(len(p), len(s)):
            zi = z[i - 1]
            if temp == 0.0:
                miss = zi.max() - zi[s[i]]
            else:
                e = np.exp((zi - zi.max()) / (1.0 if temp is None else temp))
                c = np.cumsum(e / e.sum())
                lo, hi = (c[s[i] - 1] if s[i] else 0.0), c[s[i]]
                miss = max(lo - u[b, i], u[b, i] - hi, 0.0)
            worst = max(worst, miss)
            assert miss <= tol, (b, i, s[i], miss)
    print(f"[gpu]   {steps} steps, worst miss {worst:.4f} of {tol}", flush=True)
