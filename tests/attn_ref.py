"""Plain 64-bit definitions of the softmax-attention and sampling calls, and
their inputs.  Rows of a cache are written here by the documented layout, one
(position, head) at a time, in numpy."""
import numpy as np

from paper_2607_06763_amd import workloads as W


def closure(parent):
    """depth [B][T] (-1 absent) and vis [B][T][T] (slot j is an ancestor of i or i) by parent walks."""
    B, T = parent.shape
    depth = np.full((B, T), -1)
    vis = np.zeros((B, T, T), bool)
    for b in range(B):
        for i in range(T):
            if parent[b, i] == W.PAD:
                continue
            j, n = i, -1
            while j >= 0:
                vis[b, i, j] = True
                j, n = parent[b, j], n + 1
            depth[b, i] = n
    return depth, vis


class Case:
    """One layer's inputs on the host (values already rounded to dtype), with its paged caches."""

    def __init__(self, seed, T, ctx, Hq, Hkv, d, page, dtype="bf16", parent=None, rot=None, n_valid=None, n_new=None,
                 spare=3, fill=np.nan):
        import torch
        rng = np.random.default_rng([31, seed])
        self.B, self.T, self.Hq, self.Hkv, self.d, self.page = len(ctx), T, Hq, Hkv, d, page
        self.dtype = dtype
        self.tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.x = 8 if dtype == "bf16" else 4
        self.ctx = np.array(ctx, np.int64)
        self.rot = d if rot is None else rot
        self.n_new = n_new
        B = self.B
        self.chain = parent is None
        if parent is None:
            n = [T] * B if n_new is None else list(n_new)
            parent = np.full((B, T), W.PAD)
            for b in range(B):
                parent[b, :n[b]] = np.arange(n[b]) - 1
        elif isinstance(parent, str):
            parent = np.stack([random_tree(rng, T, T if n_valid is None else n_valid[b], parent) for b in range(B)])
        self.parent = np.asarray(parent)
        self.depth, self.vis = closure(self.parent)
        self.real = self.depth >= 0

        def r(*shape, s=1.0):
            t = torch.from_numpy(s * rng.standard_normal(shape)).to(self.tdt)
            return t

        self.q, self.k, self.v = r(B, T, Hq, d), r(B, T, Hkv, d), r(B, T, Hkv, d)
        need = [-(-(int(c) + T) // page) for c in self.ctx]
        self.max_pages = max(need) + 1
        self.n_pages = sum(need) + spare
        ids = rng.permutation(self.n_pages)
        self.table = np.full((B, self.max_pages), -1, np.int64)  # unused entries are never followed
        at = 0
        for b in range(B):
            self.table[b, :need[b]] = ids[at:at + need[b]]
            at += need[b]
        # rows of the context and of the slots; everything else holds fill
        self.hist = [(r(int(c), Hkv, d), r(int(c), Hkv, d)) for c in self.ctx]
        self.kc = torch.full((self.n_pages, Hkv, d // self.x, page, self.x), fill, dtype=self.tdt)
        self.vc = torch.full((self.n_pages, Hkv, page // self.x, d, self.x), fill, dtype=self.tdt)
        for b in range(B):
            self.put(b, np.arange(int(self.ctx[b])), *self.hist[b])
        self.n_pos = int(self.ctx.max()) + T + 1
        ang = np.arange(self.n_pos)[:, None] * 1e4 ** (-2.0 * np.arange(self.rot // 2) / max(1, self.rot))[None, :]
        self.rope = np.stack([np.cos(ang), np.sin(ang)], 2).astype(np.float32)

    def place(self, b, pos):
        return self.table[b, pos // self.page], pos % self.page

    def put(self, b, pos, k, v):
        """Writes rows k, v [n][Hkv][d] at positions pos of sequence b."""
        import torch
        if len(pos) == 0:
            return
        pg, off = self.place(b, np.asarray(pos))
        pg, off = torch.from_numpy(pg), torch.from_numpy(off)
        self.kc[pg, :, :, off] = k.reshape(len(pos), self.Hkv, self.d // self.x, self.x)
        self.vc[pg, :, off // self.x, :, off % self.x] = v

    def append_slots(self):
        """The state after an append whose keys are taken as they are: rows of the real slots in the caches."""
        for b in range(self.B):
            i = np.nonzero(self.real[b])[0]
            self.put(b, self.ctx[b] + i, self.k[b, i], self.v[b, i])

    def dims(self, scale=0.0):
        from paper_2607_06763_amd import gdn_attn as A
        return A.make_attn_dims(self.B, self.T, self.Hq, self.Hkv, self.d, self.page, self.n_pages, self.max_pages,
                                dtype=self.dtype, rot=self.rot, n_pos=self.n_pos, scale=scale)

    def meta(self):
        """Device metadata, or None for a chain."""
        import torch
        from paper_2607_06763_amd import gdn_tree as G
        if self.chain:
            return None
        m = torch.zeros(G.meta_bytes(self.B, self.T), dtype=torch.uint8, device="cuda")
        G.prepare(G.make_dims(self.B, self.T, 1, 1, 16, 16), torch.from_numpy(self.parent.astype(np.int32)).cuda(), m)
        return m

    def i32(self, a):
        import torch
        return torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).cuda()

    def device(self):
        """The arguments of the calls as device tensors."""
        import torch
        return dict(q=self.q.cuda(), k=self.k.cuda(), v=self.v.cuda(), rope=torch.from_numpy(self.rope).cuda(),
                    ctx=self.i32(self.ctx), table=self.i32(self.table), kc=self.kc.cuda(), vc=self.vc.cuda(),
                    meta=self.meta(), n_new=None if self.n_new is None else self.i32(self.n_new))

    def attend_ref(self, scale=None, missing=()):
        """out [B][T][Hq][d] and sum_j p_j |v_j| in 64 bits; missing: (sequence, page slot) entries left out."""
        G = self.Hq // self.Hkv
        scale = self.d ** -0.5 if scale is None else scale
        out = np.zeros((self.B, self.T, self.Hq, self.d))
        mag = np.zeros_like(out)
        for b in range(self.B):
            c = int(self.ctx[b])
            ck, cv = (a.double().numpy() for a in self.hist[b])
            gone = {p for bb, p in missing if bb == b}
            for i in range(self.T):
                if not self.real[b, i]:
                    continue
                j = np.nonzero(self.vis[b, i])[0]
                pos = np.concatenate([np.arange(c), c + j])
                keep = np.array([p // self.page not in gone for p in pos], bool)
                if not keep.any():
                    continue
                K = np.concatenate([ck, self.k[b, j].double().numpy()])[keep]
                V = np.concatenate([cv, self.v[b, j].double().numpy()])[keep]
                for h in range(self.Hq):
                    z = scale * K[:, h // G] @ self.q[b, i, h].double().numpy()
                    p = np.exp(z - z.max())
                    p /= p.sum()
                    out[b, i, h] = p @ V[:, h // G]
                    mag[b, i, h] = p @ np.abs(V[:, h // G])
        return out, mag


def random_tree(rng, T, n, kind):
    """Parents of a tree of n nodes at random slots of T, numbered in any order ("any") or parents first ("up")."""
    out = np.full(T, W.PAD)
    if n == 0:
        return out
    slots = rng.permutation(T)[:n]
    if kind == "up":
        slots = np.sort(slots)
    out[slots[0]] = -1
    for a in range(1, n):
        out[slots[a]] = slots[a - 1] if rng.random() < 0.3 else slots[rng.integers(0, a)]
    return out


def sample_ref(z, t, k, p, least, u):
    """Token of one row of logits by the definition, in 64-bit floats and whole numbers.  The masses themselves are
    taken from 32-bit powers of two, as defined; the second result is how far (relative to the whole mass) the draw
    lies from the nearest boundary, and the third whether a cut lies within a few units of its threshold."""
    z = np.where(np.isnan(z), -np.inf, z.astype(np.float64))
    V = len(z)
    top = z.max()
    if top == -np.inf:
        return -1, 1.0, False
    if not t > 0:
        return int(np.argmax(z == top)), 1.0, False
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(z == top, 2.0 ** 31, np.floor(2.0 ** 31 * 2.0 ** ((z - top) * (np.log2(np.e) / t)) + 0.5))
    w = np.where(np.isnan(w), 0, w)
    order = np.lexsort((np.arange(V), -z))
    ws = w[order]
    if 0 < k < V:
        ws[k:] = 0
    total = ws.sum()
    before = np.cumsum(ws) - ws
    near = False
    if not p >= 1:
        keep = before < p * total
        keep[0] = True
        near |= bool(np.any(np.abs(before - p * total) < 1e-5 * total))
        ws = np.where(keep, ws, 0)
    if least > 0:
        thr = min(least, 1.0) * 2.0 ** 31
        near |= bool(np.any(np.abs(ws - thr) < 1e-5 * 2.0 ** 31) and least < 1)
        ws = np.where(ws >= thr, ws, 0)
    kept = np.zeros(V)
    kept[order] = ws
    cum = np.cumsum(kept)
    want = u * cum[-1]
    tok = int(np.argmax(cum > want)) if cum[-1] > want else int(np.nonzero(kept)[0][-1])
    lo = cum[tok] - kept[tok]
    return tok, float(min(want - lo, cum[tok] - want) / cum[-1]), near
