"""Speculative decoding of a small model with GDN and attention layers, every
per-token operator of it through the library.

The weights are seeded random numbers: ``HybridModel`` is an embedding, layers
of both kinds with a residual connection each and RMS-normalised inputs, and
an output projection; the projections are plain matrix products.  A step of
``Decoder`` takes a draft tree per sequence and runs::

    prepare                                     tree metadata
    per GDN layer:        step                  commit of the last step's path, then every node's output
    per attention layer:  kv_append, attend     rotation and paged cache, then every node's output
    sample, accept                              a token per node, the walk along them
    per attention layer:  kv_commit             the accepted path's rows to the front

``Decoder.prompt`` takes the prompts in pieces: verify and commit of the GDN
layers, or with ``prompt_form="chain"`` one call of the chain form, which has no
tree to prepare; append and attend (without metadata, a length a sequence) of
the attention layers.

A ``HybridModel`` with ``gated`` has a weighted norm and a gate on every GDN
head's output, and weighted norms before and after every block: ``gate_norm``,
and ``add_norm`` from one block to the next.

The random number of a position is fixed beforehand (``u`` [B][positions]),
so the tokens do not depend on the draft trees: a node's token is the sample
of the model given its context, and the tree only decides how many of them a
step emits.

    python -m paper_2607_06763_amd.hybrid_decode [--batch 4] [--slots 32] [--tokens 64] [--gated] [--prompt-form chain]
"""
from __future__ import annotations

import argparse
from typing import List, Sequence

import numpy as np

from . import decode_sim as D
from . import workloads as W

EPS = 1e-6
PROMPT_CHUNK = 512  # slots of a chain


class HybridModel:
    """Weights (float32 numpy arrays); layers names the kind of each layer."""

    def __init__(self, vocab: int = 64, width: int = 64, layers: Sequence[str] = ("gdn", "attn", "gdn", "attn"),
                 Hk: int = 2, Hv: int = 4, dk: int = 64, dv: int = 64, Hq: int = 4, Hkv: int = 2, d: int = 64,
                 rot: int = 32, positions: int = 1024, sharpness: float = 3.0, seed: int = 0, gated: bool = False):
        rng = np.random.default_rng([seed, 15485863])
        self.V, self.width, self.positions = vocab, width, positions
        self.Hk, self.Hv, self.dk, self.dv = Hk, Hv, dk, dv
        self.Hq, self.Hkv, self.d, self.rot = Hq, Hkv, d, rot

        def mat(n_out, n_in, gain=1.0):
            return (gain / np.sqrt(n_in) * rng.standard_normal((n_out, n_in))).astype(np.float32)

        self.embed = rng.standard_normal((vocab, width)).astype(np.float32)
        self.unembed = mat(vocab, width, sharpness)
        self.kinds = list(layers)
        self.layers = []
        for kind in layers:
            if kind == "gdn":
                C = 2 * Hk * dk + Hv * dv
                self.layers.append(dict(q=mat(Hk * dk, width), k=mat(Hk * dk, width), v=mat(Hv * dv, width),
                                        alpha=mat(Hv, width), beta=mat(Hv, width), o=mat(width, Hv * dv, 0.5),
                                        conv_w=(0.5 * rng.standard_normal((C, 4))).astype(np.float32)))
            elif kind == "attn":
                self.layers.append(dict(q=mat(Hq * d, width), k=mat(Hkv * d, width), v=mat(Hkv * d, width),
                                        o=mat(width, Hq * d, 0.5)))
            else:
                raise ValueError(f"layer kind {kind!r}, expected 'gdn' or 'attn'")
        angle = np.arange(positions)[:, None] * 10000.0 ** (-np.arange(rot // 2) / max(1, rot // 2))
        self.rope = np.stack([np.cos(angle), np.sin(angle)], axis=-1).astype(np.float32)
        self.gated = gated
        if gated:  # behind all others, so that these are the same with and without
            near_one = lambda n: (1.0 + 0.2 * rng.standard_normal(n)).astype(np.float32)
            for kind, l in zip(layers, self.layers):
                l.update(norm=near_one(width), post=near_one(width), scale=(0.5 * near_one(width)).astype(np.float32))
                if kind == "gdn":
                    l.update(z=mat(Hv * dv, width), head=near_one(dv))
            self.final = near_one(width)

        # the drafter: the next token from the last one's embedding alone
        z = self.embed / np.sqrt(np.mean(self.embed ** 2, axis=1, keepdims=True) + EPS) @ self.unembed.T
        e = np.exp(z - z.max(axis=1, keepdims=True))
        self._draft = (e / e.sum(axis=1, keepdims=True)).astype(np.float64)

    def drafter(self, ctx) -> np.ndarray:
        """As ``decode_sim.SyntheticLM.drafter``: a distribution over the next token."""
        return self._draft[ctx[-1]]


class Decoder:
    """B sequences, draft trees of up to T slots.  Every sequence has
    max_pages pages of the caches to itself; u float32 [B][n] holds the random
    number of each position, for sequences of up to n tokens.  prompt_form:
    "chain" needs no tree and reads the prompt out in 32 bits instead of fp16;
    "tree" stays the default because the two round differently, and a program
    that does not choose keeps the tokens that it had."""

    def __init__(self, model: HybridModel, B: int, T: int, u: np.ndarray, max_pages: int = 32, page: int = 16,
                 dtype: str = "f32", temperature=None, top_k=None, top_p=None, min_p=None, device="cuda",
                 prompt_form: str = "tree"):
        import torch
        from . import gdn_attn as A
        from . import gdn_layer as L
        from . import gdn_tree as G
        if prompt_form not in ("tree", "chain"):
            raise ValueError(f"prompt_form: {prompt_form!r}, expected 'tree' or 'chain'")
        self.A, self.G, self.L, self.torch, self.prompt_form = A, G, L, torch, prompt_form
        self.m, self.B, self.T, self.dtype, self.device = model, B, T, dtype, device
        self.max_pages, self.page = max_pages, page
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        up = lambda a, t=None: torch.as_tensor(np.ascontiguousarray(a), dtype=t).to(device)
        self.embed, self.unembed, self.rope = up(model.embed), up(model.unembed).t().contiguous(), up(model.rope)
        self.w = [{n: up(a) if n == "conv_w" or a.ndim == 1 else up(a).t().contiguous() for n, a in l.items()} for l in model.layers]
        self.final = up(model.final) if model.gated else None
        row = lambda x, t: None if x is None else up(np.broadcast_to(x, (B,)), t)
        self.sampling = dict(temperature=row(temperature, torch.float32), top_k=row(top_k, torch.int32),
                             top_p=row(top_p, torch.float32), min_p=row(min_p, torch.float32))
        if np.ndim(u) != 2 or len(u) != B:
            raise ValueError(f"u: shape {np.shape(u)}, expected [{B}][positions]")
        self.u = up(u, torch.float32)
        # pages in an order of their own, as an allocator would hand them out
        order = np.random.default_rng(B * max_pages).permutation(B * max_pages)
        self.table = up(order.reshape(B, max_pages), torch.int32)
        self.ctx_len = torch.zeros(B, dtype=torch.int32, device=device)
        self.lengths = np.zeros(B, np.int64)  # the same on the host
        kc, vc = A.cache_shapes(self._attn(T))
        C = 2 * model.Hk * model.dk + model.Hv * model.dv
        zeros = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t, device=device)
        self.state = [dict(S=zeros(B, model.Hv, model.dv, model.dk), conv=zeros(B, 3, C)) if kind == "gdn" else
                      dict(k=zeros(*kc, t=self.dt), v=zeros(*vc, t=self.dt)) for kind in model.kinds]
        self.last = None  # the last step: metadata, accepted slots, inputs of each GDN layer

    def _attn(self, T):
        m = self.m
        return self.A.make_attn_dims(self.B, T, m.Hq, m.Hkv, m.d, self.page, self.B * self.max_pages, self.max_pages,
                                     self.dtype, rot=m.rot, n_pos=m.positions)

    def _gdn(self, T):
        m = self.m
        return self.G.make_dims(self.B, T, m.Hk, m.Hv, m.dk, m.dv, self.dtype)

    def _norm(self, x):
        return x * self.torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)

    def _next(self, i):
        """The weight of the norm before layer i (the last norm's behind the layers)."""
        return self.w[i]["norm"] if i < len(self.w) else self.final

    def _unit(self, x):
        return x / x.norm(dim=-1, keepdim=True).clamp_min(EPS)

    def _layers(self, tok, meta, n_new, gdn):
        """Normed hidden vectors after the layers; gdn(i, inputs) gives the output of GDN layer i, n_new the lengths of
        chains (None: trees).  Returns them and the inputs of the GDN layers."""
        torch, m, (B, T) = self.torch, self.m, tok.shape
        x = self.embed[tok.long()].reshape(B * T, -1)
        F = torch.nn.functional
        inputs, status = {}, []
        da = self._attn(T)
        if m.gated:
            h = torch.empty_like(x)
            self.L.add_norm(x, None, None, h, weight=self._next(0), eps=EPS)
        for i, (kind, w) in enumerate(zip(m.kinds, self.w)):
            y = (h if m.gated else self._norm(x)).view(B, T, -1)
            if kind == "gdn":
                a = dict(q=self._unit((y @ w["q"]).view(B, T, m.Hk, m.dk)), k=self._unit((y @ w["k"]).view(B, T, m.Hk, m.dk)),
                         v=(y @ w["v"]).view(B, T, m.Hv, m.dv), alpha=torch.exp(-F.softplus(y @ w["alpha"])),
                         beta=torch.sigmoid(y @ w["beta"]))
                inputs[i] = {n: t.to(self.dt).contiguous() for n, t in a.items()}
                out = gdn(i, inputs[i])
                if m.gated:
                    heads = out.view(B * T, m.Hv, m.dv)
                    self.L.gate_norm(heads, (y @ w["z"]).view(B * T, m.Hv, m.dv), heads, weight=w["head"], eps=EPS)
            else:
                s = self.state[i]
                q, k, v = ((y @ w[n]).view(B, T, -1, m.d).to(self.dt) for n in "qkv")
                st = torch.empty(B, dtype=torch.int32, device=self.device)
                tree = dict(meta=meta) if n_new is None else dict(n_new=n_new)
                self.A.kv_append(da, q, k, v, self.rope if m.rot else None, self.ctx_len, self.table, s["k"], s["v"], q,
                                 kv_status=st, **tree)
                out = torch.empty_like(q)
                self.A.attend(da, q, s["k"], s["v"], self.table, self.ctx_len, out, **tree)
                status.append(st)
            block = out.float().reshape(B * T, -1) @ w["o"]
            if m.gated:
                self.L.add_norm(block, x, x, h, weight=self._next(i + 1), post_weight=w["post"], scale=w["scale"], post=True, eps=EPS)
            else:
                x = x + block
        return (h if m.gated else self._norm(x)).view(B, T, -1), inputs, status

    def _check(self, statuses, what):
        worst = self.torch.stack(statuses).amax(0).tolist() if statuses else []
        if any(worst):
            b = next(b for b, s in enumerate(worst) if s)
            raise RuntimeError(f"{what}: sequence {b} has status {worst[b]}")

    def prompt(self, prompts: List[List[int]]) -> None:
        """The prompts without their last tokens (which are the first trees' roots), in chunks."""
        torch, G, m, B = self.torch, self.G, self.m, self.B
        if self.last is not None:
            raise RuntimeError("prompt: after a step")
        longest = max(len(p) for p in prompts) - 1
        for at in range(0, longest, PROMPT_CHUNK):
            T = min(PROMPT_CHUNK, longest - at)
            n = np.array([min(max(len(p) - 1 - at, 0), T) for p in prompts], np.int32)
            tok, parent = np.zeros((B, T), np.int32), np.full((B, T), W.PAD, np.int32)
            for b, p in enumerate(prompts):
                tok[b, :n[b]] = p[at:at + n[b]]
                parent[b, :n[b]] = np.arange(n[b]) - 1
            d = self._gdn(T)
            lengths, accepted = torch.from_numpy(n).to(self.device), torch.from_numpy(n - 1).to(self.device)
            if self.prompt_form == "tree":
                meta = torch.empty(G.meta_bytes(B, T), dtype=torch.uint8, device=self.device)
                G.prepare(d, torch.from_numpy(parent).to(self.device), meta)
            else:
                meta, dc = None, self.L.make_chain_dims(B, T, m.Hk, m.Hv, m.dk, m.dv, in_dtype=self.dtype)

            def gdn(i, a):
                s = self.state[i]
                if meta is None:
                    out = torch.zeros(B, T, m.Hv, m.dv, device=self.device)  # rows without a token are not written
                    conv, st = torch.empty_like(s["conv"]), torch.empty(B, dtype=torch.int32, device=self.device)
                    self.L.chain(dc, **a, conv_w=self.w[i]["conv_w"], conv_state=s["conv"], conv_state_out=conv, S=s["S"], out=out,
                                 n_new=lengths, status=st)
                    s["conv"] = conv
                    statuses.append(st)
                    return out
                out = torch.empty(B, T, m.Hv, m.dv, device=self.device)
                G.verify(d, meta, **a, conv_w=self.w[i]["conv_w"], conv_state=s["conv"], S0=s["S"], out=out)
                st = torch.empty(B, dtype=torch.int32, device=self.device)
                G.commit(d, meta, accepted, **a, conv_w=self.w[i]["conv_w"], conv_state=s["conv"], S=s["S"], commit_status=st)
                statuses.append(st)
                return out

            statuses = []
            _, _, st = self._layers(torch.from_numpy(tok).to(self.device), meta, lengths, gdn)
            self._check(statuses + st, "prompt")
            self.ctx_len = self.ctx_len + lengths
            self.lengths += n

    def step(self, trees: List[D.Tree]) -> List[List[int]]:
        """One step: the tokens that each sequence emits, given its draft tree (root: the last emitted token)."""
        torch, G, A, m, B, T = self.torch, self.G, self.A, self.m, self.B, self.T
        parent, tok, depth = np.full((B, T), W.PAD, np.int32), np.zeros((B, T), np.int32), np.zeros((B, T), np.int64)
        for b, t in enumerate(trees):
            n = len(t)
            parent[b, :n], tok[b, :n] = t.parent, t.tokens
            for s in range(1, n):
                depth[b, s] = depth[b, t.parent[s]] + 1
            if n and self.lengths[b] + depth[b].max() + 1 >= self.u.shape[1]:
                raise ValueError(f"step: no random number for position {self.lengths[b] + depth[b].max() + 1} of sequence {b}")
        d, i32 = self._gdn(T), torch.int32
        dev = lambda a: torch.from_numpy(a).to(self.device)
        new = lambda *s: torch.empty(*s, dtype=i32, device=self.device)
        draft, meta = dev(tok), torch.empty(G.meta_bytes(B, T), dtype=torch.uint8, device=self.device)
        tree_status, statuses = new(B), []
        G.prepare(d, dev(parent), meta, tree_status)

        def gdn(i, a):
            s, cw = self.state[i], self.w[i]["conv_w"]
            out = torch.empty(B, T, m.Hv, m.dv, device=self.device)
            if self.last is None:  # nothing to commit: the prompt did
                G.verify(d, meta, **a, conv_w=cw, conv_state=s["conv"], S0=s["S"], out=out)
            else:
                p, conv, st = self.last[2][i], torch.empty_like(s["conv"]), new(B)
                G.step(d, self.last[0], self.last[1], p["q"], p["k"], p["v"], p["alpha"], p["beta"], st, meta, **a,
                       conv_w=cw, conv_state=s["conv"], conv_state_out=conv, S=s["S"], out=out)
                s["conv"] = conv
                statuses.append(st)
            return out

        x, inputs, st = self._layers(draft, meta, None, gdn)
        logits = x @ self.unembed
        # the number of the position after a node's (that of an absent slot is not used)
        u = torch.gather(self.u, 1, (self.ctx_len.long()[:, None] + dev(depth) + 1).clamp_max(self.u.shape[1] - 1))
        token, accepted, n_emitted, emitted = new(B, T), new(B), new(B), new(B, T)
        A.sample(logits.contiguous(), u, token, meta=meta, **self.sampling)
        A.accept(draft, token, accepted, n_emitted, emitted, meta=meta)
        new_len, da = self.ctx_len, self._attn(T)
        for kind, s in zip(m.kinds, self.state):
            if kind == "attn":
                new_len, cs = new(B), new(B)
                A.kv_commit(da, accepted, self.table, self.ctx_len, s["k"], s["v"], new_len, kv_status=cs, meta=meta)
                statuses.append(cs)
        self._check([tree_status] + st + statuses, "step")
        self.ctx_len = new_len if "attn" in m.kinds else self.ctx_len + n_emitted
        self.last = (meta, accepted, inputs)
        rows, n = emitted.cpu().numpy(), n_emitted.cpu().numpy()
        self.lengths += n
        for b in range(B):
            if n[b] and rows[b, n[b] - 1] < 0:
                raise RuntimeError(f"step: no token for sequence {b}: none of its logits is above -inf")
        return [[int(t) for t in rows[b, :n[b]]] for b in range(B)]


def decode(dec: Decoder, prompts: List[List[int]], tokens: int, budget: int = 0, width: int = 4, fanout: int = 8):
    """Generates at least `tokens` tokens a sequence from best-first draft
    trees of `budget` nodes (0: the decoder's slots; 1: a token a step).
    Returns the sequences and the number of steps."""
    dec.prompt(prompts)
    seqs = [list(map(int, p)) for p in prompts]
    done = [len(p) + tokens for p in prompts]
    steps = 0
    while any(len(s) < n for s, n in zip(seqs, done)):
        trees = [D.build_tree_best_first(dec.m, s, budget=budget or dec.T, width=width, fanout=fanout) for s in seqs]
        for s, e in zip(seqs, dec.step(trees)):
            s.extend(e)
        steps += 1
    return seqs, steps


def main(argv=None) -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--slots", type=int, default=32, help="slots of a draft tree")
    ap.add_argument("--tokens", type=int, default=64, help="tokens to generate per sequence")
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="bf16")
    ap.add_argument("--temperature", type=float, default=1.0)
    ap.add_argument("--top-k", type=int, default=0)
    ap.add_argument("--top-p", type=float, default=1.0)
    ap.add_argument("--min-p", type=float, default=0.0)
    ap.add_argument("--seed", type=int, default=0)
    ap.add_argument("--gated", action="store_true", help="norms and gates around the blocks")
    ap.add_argument("--prompt-form", choices=("tree", "chain"), default="tree", help="GDN layers over the prompts")
    a = ap.parse_args(argv)
    rng = np.random.default_rng(a.seed)
    # the whole batch goes on until its last sequence is done: up to `slots` tokens a step
    longest = 16 + a.tokens * a.slots + 2 * a.slots
    model = HybridModel(seed=a.seed, positions=longest, gated=a.gated)
    prompts = [[int(t) for t in rng.integers(0, model.V, rng.integers(1, 17))] for _ in range(a.batch)]
    dec = Decoder(model, a.batch, a.slots, rng.random((a.batch, longest), dtype=np.float32), max_pages=-(-longest // 16),
                  dtype=a.dtype, temperature=a.temperature, top_k=a.top_k, top_p=a.top_p, min_p=a.min_p,
                  prompt_form=a.prompt_form)
    seqs, steps = decode(dec, prompts, a.tokens)
    made = sum(len(s) - len(p) for s, p in zip(seqs, prompts))
    print(f"{made} tokens of {a.batch} sequences in {steps} steps: {made / (steps * a.batch):.2f} a step and sequence")
    for s, p in zip(seqs, prompts):
        print(p, "->", s[len(p):len(p) + a.tokens])


if __name__ == "__main__":
    main()
