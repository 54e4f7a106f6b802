"""Inputs of the chain form of the gated delta rule and its definition in
64-bit numpy: the recurrence, token by token."""
import numpy as np


class Chain:
    """One layer's inputs on the host (values already rounded to dtype): lengths of each sequence, padded to T tokens, or
    packed (with `spare` rows behind the last sequence).  Rows that belong to no sequence hold `fill`."""

    def __init__(self, seed, lengths, Hk, Hv, dk, dv, dtype="f32", out="f32", packed=False, T=None, spare=2, fill=np.nan,
                 alpha=None, beta=None, same_keys=False, state=0.3, gain=1.0):
        import torch
        rng = np.random.default_rng([77, seed])
        self.n = np.array(lengths, np.int64)
        self.B, self.T = len(lengths), int(max(lengths)) if T is None else T
        self.Hk, self.Hv, self.dk, self.dv, self.dtype, self.out_dtype, self.packed = Hk, Hv, dk, dv, dtype, out, packed
        self.C = C = 2 * Hk * dk + Hv * dv
        B = self.B
        self.first = np.concatenate([[0], np.cumsum(self.n)])[:-1] if packed else self.T * np.arange(B)
        self.rows = int(self.n.sum()) + spare if packed else B * self.T
        tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
        live = np.zeros(self.rows, bool)
        for b in range(B):
            live[self.first[b]:self.first[b] + self.n[b]] = True
        self.live = live

        def rounded(a):
            a = torch.from_numpy(np.asarray(a, np.float64)).to(tdt)
            a[torch.from_numpy(~live)] = fill
            return a

        raw = gain * rng.standard_normal((self.rows, C))
        if same_keys:  # every token has the same raw key: the strongest coupling inside a chunk
            raw[:, Hk * dk:2 * Hk * dk] = raw[:1, Hk * dk:2 * Hk * dk]
        q, k, v = np.split(raw, [Hk * dk, 2 * Hk * dk], axis=1)
        self.q, self.k = rounded(q.reshape(-1, Hk, dk)), rounded(k.reshape(-1, Hk, dk))
        self.v = rounded(v.reshape(-1, Hv, dv))
        a = np.exp(-np.exp(-6 * rng.random(Hv)) * np.logaddexp(0, rng.standard_normal((self.rows, Hv))))
        bt = 1 / (1 + np.exp(-1.5 * rng.standard_normal((self.rows, Hv))))
        self.alpha = rounded(a if alpha is None else np.broadcast_to(alpha, a.shape).copy())
        self.beta = rounded(bt if beta is None else np.broadcast_to(beta, bt.shape).copy())
        self.conv_w = (0.5 * rng.standard_normal((C, 4))).astype(np.float32)
        self.conv_state = rng.standard_normal((B, 3, C)).astype(np.float32)
        self.S = (state * rng.standard_normal((B, Hv, dv, dk))).astype(np.float32)

    def lead(self, t):
        return t if self.packed else t.reshape(self.B, self.T, *t.shape[1:])

    def dims(self, scale=0.0):
        from paper_2607_06763_amd import gdn_layer as L
        return L.make_chain_dims(self.B, self.T, self.Hk, self.Hv, self.dk, self.dv, in_dtype=self.dtype,
                                 out_dtype=self.out_dtype, rows=self.rows if self.packed else 0, scale=scale)

    def device(self, fill=7.0):
        """Arguments of gdn_layer.chain as device tensors; outputs hold fill."""
        import torch
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        i32 = lambda a: up(np.asarray(a, np.int32))
        odt = torch.bfloat16 if self.out_dtype == "bf16" else torch.float32
        a = {n: self.lead(getattr(self, n)).contiguous().cuda() for n in ("q", "k", "v", "alpha", "beta")}
        a.update(conv_w=up(self.conv_w), conv_state=up(self.conv_state), S=up(self.S.copy()),
                 conv_state_out=torch.full((self.B, 3, self.C), fill, device="cuda"),
                 out=self.lead(torch.full((self.rows, self.Hv, self.dv), fill, dtype=odt, device="cuda")),
                 status=torch.full((self.B,), -5, dtype=torch.int32, device="cuda"),
                 start=i32(np.concatenate([self.first, [self.first[-1] + self.n[-1]]])) if self.packed else None,
                 n_new=i32(self.n) if not self.packed and (self.n != self.T).any() else None)
        return a

    def ref(self, scale=None):
        """out [rows][Hv][dv] (zeros where no token is), state and conv state, in 64 bits."""
        Hk, Hv, dk, dv = self.Hk, self.Hv, self.dk, self.dv
        scale = dk ** -0.5 if scale is None else scale
        f = lambda t: t.double().numpy()
        raw = np.concatenate([f(x).reshape(self.rows, x.shape[1] * x.shape[2]) for x in (self.q, self.k, self.v)], 1)
        al, be = f(self.alpha), f(self.beta)
        cw = self.conv_w.astype(np.float64)
        out = np.zeros((self.rows, Hv, dv))
        S, conv = self.S.astype(np.float64), self.conv_state.astype(np.float64)
        for b in range(self.B):
            for t in range(self.n[b]):
                r = self.first[b] + t
                window = np.concatenate([conv[b], raw[r][None]])
                y = (window * cw.T).sum(0)
                y = y / (1 + np.exp(-y))
                conv[b] = window[1:]
                q, k = y[:Hk * dk].reshape(Hk, dk), y[Hk * dk:2 * Hk * dk].reshape(Hk, dk)
                v = y[2 * Hk * dk:].reshape(Hv, dv)
                q, k = (x / np.sqrt((x * x).sum(1, keepdims=True) + 1e-6) for x in (q, k))
                q, k = (np.repeat(x, Hv // Hk, axis=0) for x in (q, k))
                Sk = np.einsum("hvd,hd->hv", S[b], k)
                a_, b_ = al[r][:, None], be[r][:, None]
                S[b] = a_[:, :, None] * S[b] + (b_ * (v - a_ * Sk))[:, :, None] * k[:, None, :]
                out[r] = scale * np.einsum("hvd,hd->hv", S[b], q)
        return out, S, conv
