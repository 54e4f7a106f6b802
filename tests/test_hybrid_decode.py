"""The decode loop of a small model with GDN and attention layers
(paper_2607_06763_amd/hybrid_decode.py) against its definition in 64 bits.

The model is evaluated on every finished sequence as one chain: GDN layers by
the oracle, attention, rotation and projections in numpy.  Every token must be
a sample of that distribution with the position's random number, whichever
draft tree it came from.

Tolerances.  A GDN output is off by at most 2e-3 of the largest (its own
tests), attention by far less in fp32; through an output projection of gain
0.5 (outputs of up to 3 sigma) this moves a hidden vector of norm about 1 per
component by 3e-3 a layer, two layers of them, and logits of gain 3 by about
0.013: twice that, 0.03, for a boundary of the distribution function (a
probability moves by the difference of two logits).  In bf16 the inputs of
each of the four layers are rounded (2^-8, in q, k and v) and the attention's
outputs too: about 2^-7 of an output of gain 0.5 a layer, logits by
3 x 4 x 0.5 x 2^-7 = 0.05 and the boundary by twice that, 0.1."""
import numpy as np
import pytest

from paper_2607_06763_amd import decode_sim as D
from paper_2607_06763_amd import hybrid_decode as H
from paper_2607_06763_amd import workloads as W


def reference_logits(orc, m, tokens):
    """Logits [n][V] of the model after each of the tokens."""
    n = len(tokens)
    x = m.embed[tokens].astype(np.float64)
    f64 = lambda a: a.astype(np.float64)
    norm = lambda a: a / np.sqrt(np.mean(a * a, axis=-1, keepdims=True) + H.EPS)
    unit = lambda a: a / np.linalg.norm(a, axis=-1, keepdims=True)
    for kind, w in zip(m.kinds, m.layers):
        y = norm(x)
        p = {k: y @ f64(a).T for k, a in w.items() if k not in ("o", "conv_w")}
        if kind == "gdn":
            C = 2 * m.Hk * m.dk + m.Hv * m.dv
            g = dict(q=unit(p["q"].reshape(1, n, m.Hk, m.dk)), k=unit(p["k"].reshape(1, n, m.Hk, m.dk)),
                     v=p["v"].reshape(1, n, m.Hv, m.dv), alpha=np.exp(-np.logaddexp(0, p["alpha"]))[None],
                     beta=1 / (1 + np.exp(-p["beta"]))[None])
            work = W.Workload(name="hybrid", B=1, T=n, Hk=m.Hk, Hv=m.Hv, dk=m.dk, dv=m.dv, in_dtype="f32",
                              parent=(np.arange(n, dtype=np.int32) - 1)[None], S0=np.zeros((1, m.Hv, m.dv, m.dk), np.float32),
                              conv_w=w["conv_w"], conv_state=np.zeros((1, 3, C), np.float32), accepted=np.array([-1], np.int32),
                              **{k: a.astype(np.float32) for k, a in g.items()})
            out = orc.verify(work)[0]
        else:
            q, k, v = (p[c].reshape(n, -1, m.d) for c in "qkv")
            cs, half = f64(m.rope[:n]), m.rot // 2

            def turn(a):
                lo, hi = a[..., :half].copy(), a[..., half:m.rot].copy()
                c, s = cs[:, None, :, 0], cs[:, None, :, 1]
                return np.concatenate([lo * c - hi * s, hi * c + lo * s, a[..., m.rot:]], axis=-1)
            q, k = turn(q), turn(k)
            out = np.zeros((n, m.Hq, m.d))
            for h in range(m.Hq):
                hk = h // (m.Hq // m.Hkv)
                z = q[:, h] @ k[:, hk].T * m.d ** -0.5
                z = np.where(np.tril(np.ones((n, n), bool)), z, -np.inf)
                e = np.exp(z - z.max(axis=1, keepdims=True))
                out[:, h] = e / e.sum(axis=1, keepdims=True) @ v[:, hk]
        x = x + out.reshape(n, -1) @ f64(w["o"]).T
    return norm(x) @ f64(m.unembed).T


def test_unknown_layer_kind():
    with pytest.raises(ValueError):
        H.HybridModel(layers=("gdn", "mlp"))


def test_draft_trees_follow_the_drafter():
    m = H.HybridModel(seed=3)
    t = D.build_tree_best_first(m, [5, 9], budget=20)
    assert len(t) == 20 and t.tokens[0] == 9
    best = int(np.argmax(m.drafter([9])))
    assert best in [t.tokens[c] for c in t.children[0]]


RUNS = [
    # seed, layers, slots, budget, dtype, temperature
    (1, ("gdn", "attn", "gdn", "attn"), 32, 32, "f32", 1.0),
    (2, ("gdn", "attn", "gdn", "attn"), 32, 20, "f32", None),
    (3, ("gdn", "attn", "gdn", "attn"), 1, 1, "f32", 0.7),
    (4, ("gdn", "attn", "gdn", "attn"), 130, 130, "f32", 1.3),
    (5, ("attn", "gdn", "gdn", "attn"), 48, 48, "bf16", 1.0),
    (6, ("gdn", "attn", "attn", "gdn"), 24, 24, "f32", 0.0),
    (7, ("attn",), 16, 16, "f32", 1.0),
    (8, ("gdn",), 16, 16, "f32", 1.0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("run", RUNS, ids=lambda r: f"{r[0]}-{'.'.join(r[1])}-T{r[2]}-{r[4]}-t{r[5]}")
def test_tokens_are_samples_of_the_model(orc, run):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    seed, layers, T, budget, dtype, temp = run
    rng = np.random.default_rng([9, seed])
    m = H.HybridModel(seed=seed, layers=layers, positions=512)
    B, want = 3, 24
    prompts = [[int(t) for t in rng.integers(0, m.V, n)] for n in (1, 40, 17)]
    u = rng.random((B, 512), dtype=np.float32)
    dec = H.Decoder(m, B, T, u, max_pages=32, dtype=dtype, temperature=temp)
    print(f"[gpu] hybrid decode {run}", flush=True)
    seqs, steps = H.decode(dec, prompts, want, budget=budget)
    torch.cuda.synchronize()
    made = [len(s) - len(p) for s, p in zip(seqs, prompts)]
    print(f"[gpu]   {steps} steps, tokens {made}", flush=True)
    assert [int(n) for n in dec.ctx_len] == [len(s) - 1 for s in seqs]
    assert all(s[:len(p)] == p for s, p in zip(seqs, prompts))
    if T == 1:
        assert made == [steps] * B
    else:
        assert sum(made) > 1.1 * steps * B  # drafts are accepted
    tol = 0.03 if dtype == "f32" else 0.1
    worst = 0.0
    for b, (s, p) in enumerate(zip(seqs, prompts)):
        z = reference_logits(orc, m, s[:-1])
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
    print(f"[gpu]   worst miss {worst:.4f} of {tol}", flush=True)


@pytest.mark.gpu
def test_trees_of_any_size_give_the_same_tokens():
    """The position's random number and the context fix the token.  u is moved away from the boundaries that rounding
    could move it across: greedy, where the two largest logits of a random model are rarely close."""
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    m = H.HybridModel(seed=12, positions=512)
    prompts = [[1, 2, 3], [4], [5, 6, 7, 8, 9]]
    got = []
    for T in (1, 8, 64):
        dec = H.Decoder(m, 3, T, np.zeros((3, 512), np.float32), temperature=0.0)
        seqs, steps = H.decode(dec, prompts, 32)
        got.append([s[:len(p) + 32] for s, p in zip(seqs, prompts)])
        print(f"[gpu] {T} slots: {steps} steps", flush=True)
    assert got[0] == got[1] == got[2]
