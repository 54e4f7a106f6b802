"""Timed cases of the operators beside the Gated DeltaNet layers of a speculative decode step.

A hybrid model interleaves the recurrent layers with softmax-attention layers.
For those a decode step (a draft tree, a chunk of a prompt, or one token per
sequence) rotates and appends the new keys and values to a paged cache, lets
every new node attend to the cache and to its own ancestors, samples a token
at every node from the model's logits, walks the tree along the samples to the
accepted node, and moves that node's path to the front of the new cache rows.

``own`` False: elementary torch operations in 32 bits.  ``own`` True: the
library's kernels.  Both take the same state.  The caches are held in 16-byte
packs (x = 8 bf16 or 4 fp32): keys [pages][heads][d / x][page][x], values
[pages][heads][page / x][d][x].
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

LOG2E = 1.4426950408889634


# --------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------
def listed():
    return [
        # one user, one token, a short conversation: launch latency
        dict(name="attend-b1-t1", op="attend", B=1, T=1, Hq=32, Hkv=8, d=128, page=64, ctx=700, dtype="bf16", tree="chain",
             pad=0.0, rot=128),
        # a decode batch without drafting, conversations of very different lengths: bytes of the cache
        dict(name="attend-b32-t1-ctx8k", op="attend", B=32, T=1, Hq=32, Hkv=8, d=128, page=64, ctx=8192, dtype="bf16",
             tree="chain", pad=0.0, rot=128),
        # fp32, small heads, odd tree size, trees padded to it, the smallest pages
        dict(name="attend-b8-t99-f32", op="attend", B=8, T=99, Hq=16, Hkv=4, d=64, page=16, ctx=1000, dtype="f32",
             tree="random", pad=0.3, rot=64),
        # a 512-token chunk of two long prompts, wide heads
        dict(name="attend-b2-chain512-d256", op="attend", B=2, T=512, Hq=16, Hkv=4, d=256, page=128, ctx=12000, dtype="bf16",
             tree="chain", pad=0.0, rot=64),
        # the largest call: sixteen users with the benchmark's trees (budget 128, depth 16)
        dict(name="attend-b16-t128-ctx8k", op="attend", B=16, T=128, Hq=32, Hkv=8, d=128, page=64, ctx=8192, dtype="bf16",
             tree="large", pad=0.0, rot=128),
        # one token's keys and values: launch latency
        dict(name="append-b1-t1", op="append", B=1, T=1, Hq=32, Hkv=8, d=128, page=64, ctx=700, dtype="bf16", tree="chain",
             pad=0.0, rot=128),
        # the benchmark's batch of trees, a quarter of each head rotated
        dict(name="append-b32-t128", op="append", B=32, T=128, Hq=24, Hkv=4, d=256, page=64, ctx=900, dtype="bf16",
             tree="large", pad=0.2, rot=64),
        # the accepted paths of eight users' trees of budget 64
        dict(name="commit-b8-t64", op="commit", B=8, T=64, Hq=32, Hkv=8, d=128, page=64, ctx=700, dtype="bf16", tree="random",
             pad=0.0, rot=128),
        # the benchmark's batch, fp32 caches
        dict(name="commit-b32-t128-f32", op="commit", B=32, T=128, Hq=32, Hkv=8, d=128, page=32, ctx=500, dtype="f32",
             tree="large", pad=0.0, rot=128),
        # the next token of one user, top-k and top-p: launch latency
        dict(name="sample-b1-t1", op="sample", B=1, T=1, V=131072, dtype="f32", mode="mixed", tree="chain", pad=0.0),
        # a token at every node of eight trees of budget 64, then the accepted nodes
        dict(name="sample+accept-b8-t64", op="sample+accept", B=8, T=64, V=131072, dtype="bf16", mode="mixed", tree="random",
             pad=0.0),
        # a vocabulary of odd size (rows of no alignment), fp32 logits, padded trees
        dict(name="sample+accept-b32-t33-odd", op="sample+accept", B=32, T=33, V=50001, dtype="f32", mode="nucleus",
             tree="random", pad=0.3),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    """Another case of the same ranges: batch 1..32, 1..512 slots, contexts of
    0..32K tokens, head counts and dims, page sizes, types, tree shapes,
    vocabularies of 1000..131072 tokens and every way of cutting them."""
    op = rng.choice(["attend", "attend", "attend", "append", "commit", "sample", "sample+accept"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    tree = rng.choice(["random", "large", "chain"])
    pad = rng.choice([0.0, 0.3])
    T = rng.choice([1, _log(rng, 2, 512), _log(rng, 2, 160)])
    B = _log(rng, 1, 32)
    if op.startswith("sample"):
        T = min(T, 160)
        V = _log(rng, 1000, 131072)
        while B > 1 and B * T * V * (2 if dtype == "f32" else 1) > 8 * 64 * 131072:
            B //= 2
        T = min(T, max(1, 8 * 64 * 131072 // (B * V * 2)))
        return dict(op=op, B=B, T=T, V=V, dtype=dtype, mode=rng.choice(["mixed", "nucleus", "topk", "minp", "plain", "greedy"]),
                    tree=tree, pad=pad if T > 1 else 0.0)
    d = rng.choice([32, 64, 128, 128, 256])
    Hkv = rng.choice([1, 2, 4, 8])
    Hq = Hkv * rng.choice([1, 2, 4, 6, 8])
    ctx = rng.choice([0, _log(rng, 16, 32768), _log(rng, 500, 16384)]) if op == "attend" else _log(rng, 16, 2000)
    c = dict(op=op, B=B, T=T, Hq=Hq, Hkv=Hkv, d=d, page=rng.choice([16, 32, 64, 128, 256]), ctx=ctx, dtype=dtype, tree=tree,
             pad=pad if T > 1 else 0.0, rot=rng.choice([d, d, d // 2, d // 4]))
    most = work(listed()[4])
    while c["B"] > 1 or c["ctx"] > 64:
        w = work(c)
        # an fp32 product costs about eight times a bf16 one
        if w["bytes"] <= most["bytes"] and w["flops"] * (8 if dtype == "f32" else 1) <= most["flops"]:
            break
        if c["B"] > 1:
            c["B"] //= 2
        else:
            c["ctx"] //= 2
    return c


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _tree(rng, n, shape):
    """Parents of a tree of n nodes, root first."""
    if shape == "chain":
        return np.arange(n) - 1
    deepest, spine, most = (7, 0, n) if shape == "random" else (15, min(16, n - 1), 8)
    par, dep, kids, open_ = [-1], [0], [0], [0]
    pick = rng.random(n)
    for i in range(1, n):
        at = open_.index(i - 1) if i <= spine and i - 1 in open_ else int(pick[i] * len(open_))
        p = open_[at]
        par.append(p)
        dep.append(dep[p] + 1)
        kids.append(0)
        kids[p] += 1
        if kids[p] >= most:
            open_.pop(at)
        if dep[i] <= deepest:
            open_.append(i)
    return np.array(par)


def _trees(case, seed):
    """parent [B][T]; with pad > 0 a sequence holds (1 - pad) T .. T nodes (a
    chain at its first slots, a tree at any)."""
    rng = np.random.default_rng([5, int(seed)])
    B, T = case["B"], case["T"]
    out = np.full((B, T), -2, np.int64)
    for b in range(B):
        n = T - int(rng.integers(0, int(case["pad"] * T) + 1))
        par = _tree(rng, n, case["tree"])
        slots = np.arange(n) if case["tree"] == "chain" else np.sort(rng.permutation(T)[:n])
        out[b, slots] = np.where(par < 0, -1, slots[np.maximum(par, 0)])
    return out


def _closure(parent):
    """depth [B][T] (-1 for an absent slot) and vis [B][T][T]: slot j is an ancestor of slot i, or i itself."""
    B, T = parent.shape
    depth = np.full((B, T), -1, np.int64)
    vis = np.zeros((B, T, T), bool)
    rows = np.arange(B)
    for i in range(T):  # parents come before their children
        real, p = parent[:, i] != -2, parent[:, i]
        up = np.maximum(p, 0)
        depth[:, i] = np.where(real, np.where(p >= 0, depth[rows, up] + 1, 0), -1)
        vis[:, i] = vis[rows, up] & (p >= 0)[:, None]
        vis[:, i, i] = real
    return depth, vis


def _blob(parent, depth, vis):
    """The tree metadata of include/gdn_tree.h: ancestor words, depth, order, pos, parent, status, count, depth and parent by position."""
    B, T = parent.shape
    W = (T + 63) // 64
    order = np.argsort(np.where(depth < 0, T, depth), axis=1, kind="stable")
    pos = np.argsort(order, axis=1, kind="stable")
    bits = np.zeros((B, T, 64 * W), bool)
    bits[:, :, :T] = vis & ~np.eye(T, dtype=bool)
    pdep = np.take_along_axis(depth, order, 1)
    up = np.take_along_axis(parent, order, 1)
    ppos = np.where(up >= 0, np.take_along_axis(pos, np.maximum(up, 0), 1), -1)
    parts = [np.packbits(bits, axis=2, bitorder="little")]
    parts += [x.astype(np.int32) for x in (depth, order, pos, parent, np.zeros(B), (depth >= 0).sum(1), pdep, ppos)]
    raw = b""
    for x in parts:
        raw += b"\0" * (-len(raw) % 16) + x.tobytes()
    return np.frombuffer(raw + b"\0" * (-len(raw) % 256), np.uint8).copy()


def _lengths(case, seed):
    """Cached tokens of each sequence: a fifth of ctx .. ctx, the first one ctx, up to 15 less by the seed (None: not less)."""
    b = np.arange(case["B"])
    n = (case["ctx"] * (1 - 0.8 * np.modf(b * 0.618034)[0])).astype(np.int64)
    return n if seed is None else np.maximum(0, n - np.random.default_rng([3, int(seed)]).integers(0, 16, case["B"]))


def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + 29)
    return g


def prepare(case, seed):
    g = _generator(seed)
    parent = _trees(case, seed)
    depth, vis = _closure(parent)
    B, T = parent.shape
    s = dict(case=case, op=case["op"])

    def up(a):
        return torch.from_numpy(np.ascontiguousarray(a)).cuda()

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    s["real"], s["depth"], s["vis"], s["parent"] = up(depth >= 0), up(depth), up(vis), up(parent)
    # a chain without absent slots needs no metadata
    s["meta"] = None if case["tree"] == "chain" and not case["pad"] else up(_blob(parent, depth, vis))
    rng = np.random.default_rng([9, int(seed)])
    acc = [rng.choice(np.nonzero(depth[b] >= 0)[0]) for b in range(B)]
    if s["op"].startswith("sample"):
        V = case["V"]
        # logits of a language model: a few tokens far above a broad bulk; ends of the vocabulary and banned tokens at -inf
        x = normal(B, T, V) * 2.0
        top = torch.randint(0, V, (B, T, 24), generator=g, device="cuda")
        x.scatter_add_(2, top, 8.0 + 2.0 * normal(B, T, 24))
        x[:, :, V - V // 64:] = -math.inf
        s["logits"] = x.to(_dt(case))
        s["u"] = torch.rand((B, T), generator=g, device="cuda")
        mode = case["mode"]
        f = np.arange(B) % 4
        t = np.where(f == 3, 0.0, np.array([0.7, 1.0, 1.3, 1.0])[f]) if mode == "mixed" else np.full(B, 0.0 if mode == "greedy" else 0.9)
        k = np.array([40, 0, 200, 0])[f] if mode == "mixed" else np.full(B, 50 if mode == "topk" else 0)
        p = np.array([0.95, 0.9, 1.0, 1.0])[f] if mode == "mixed" else np.full(B, 0.95 if mode == "nucleus" else 1.0)
        m = np.array([0.0, 0.0, 0.02, 0.0])[f] if mode == "mixed" else np.full(B, 0.05 if mode == "minp" else 0.0)
        s["temperature"], s["top_p"], s["min_p"] = (up(v.astype(np.float32)) for v in (t, p, m))
        s["top_k"] = up(k.astype(np.int32))
        s["token"] = torch.empty((B, T), dtype=torch.int32, device="cuda")
        if s["op"] == "sample+accept":
            # drafts as a good drafter makes them: often one of the likely tokens
            best = x.topk(4, dim=2).indices
            pick = best.gather(2, torch.randint(0, 4, (B, T, 1), generator=g, device="cuda"))[:, :, 0]
            s["draft"] = torch.where(s["real"], pick.gather(1, s["parent"].clamp(min=0)), 0).to(torch.int32)
            s["accepted"] = torch.empty(B, dtype=torch.int32, device="cuda")
            s["n_emitted"] = torch.empty(B, dtype=torch.int32, device="cuda")
            s["emitted"] = torch.empty((B, T), dtype=torch.int32, device="cuda")
        return s
    dt, x = _dt(case), 8 if case["dtype"] == "bf16" else 4
    Hq, Hkv, d, page, rot = (case[n] for n in ("Hq", "Hkv", "d", "page", "rot"))
    ctx = _lengths(case, seed)
    need = -(-(_lengths(case, None) + T) // page)  # pages that a sequence holds
    per, pool = int(need.max()) + 1, int(need.sum()) + 3
    table = np.zeros((B, per), np.int64)
    ids = rng.permutation(pool)
    table[np.arange(per)[None, :] < need[:, None]] = ids[:int(need.sum())]
    s["table"], s["ctx"] = up(table.astype(np.int32)), up(ctx.astype(np.int32))
    s["most"] = int(need.max()) * page  # positions that any sequence may use
    s["k_cache"] = normal(pool, Hkv, d // x, page, x).to(dt)
    s["v_cache"] = normal(pool, Hkv, page // x, d, x).to(dt)
    if s["op"] == "commit":
        s["accepted"] = up(np.array(acc, np.int32))
        s["new_len"] = torch.empty(B, dtype=torch.int32, device="cuda")
        return s
    s["q"] = normal(B, T, Hq, d).to(dt)
    s["out"] = torch.empty_like(s["q"])
    if s["op"] == "append":
        s["k"], s["v"] = normal(B, T, Hkv, d).to(dt), normal(B, T, Hkv, d).to(dt)
        ang = np.arange(case["ctx"] + T + 1)[:, None] * 1e4 ** (-2.0 * np.arange(rot // 2) / rot)[None, :]
        s["rope"] = up(np.stack([np.cos(ang), np.sin(ang)], 2).astype(np.float32))
    return s


# --------------------------------------------------------------------------
# the plain forms
# --------------------------------------------------------------------------
def _where(s, pos):
    """Page and place in it of positions [B][...] of each sequence."""
    page = s["case"]["page"]
    flat = pos.reshape(pos.shape[0], -1)
    return s["table"].long().gather(1, flat // page), flat % page


def _rotate(s, x):
    """The first rot dims of every head turned by the angles of its node's position, as 32-bit floats."""
    h = s["case"]["rot"] // 2
    at = (s["ctx"].long()[:, None] + s["depth"].clamp(min=0))
    cs = s["rope"][at][:, :, None]
    x = x.float()
    a, b = x[..., :h], x[..., h:2 * h]
    c, n = cs[..., 0], cs[..., 1]
    return torch.cat([a * c - b * n, b * c + a * n, x[..., 2 * h:]], -1)


def _plain_append(s):
    T, x = s["case"]["T"], s["k_cache"].shape[-1]
    pos = s["ctx"].long()[:, None] + torch.arange(T, device="cuda")
    pid, off = (a.reshape(-1) for a in _where(s, pos))
    q, k = _rotate(s, s["q"]), _rotate(s, s["k"]).to(s["k"].dtype)
    real = s["real"].reshape(-1, 1, 1, 1)
    kc, vc = s["k_cache"], s["v_cache"]
    k = k.reshape(-1, k.shape[2], k.shape[3] // x, x)
    v = s["v"].reshape(-1, *s["v"].shape[2:])
    kc[pid, :, :, off] = torch.where(real, k, kc[pid, :, :, off])
    vc[pid, :, off // x, :, off % x] = torch.where(real[..., 0], v, vc[pid, :, off // x, :, off % x])
    return [torch.where(s["real"][:, :, None, None], q, 0.0).to(s["q"].dtype), kc, vc]


def _plain_attend(s):
    c = s["case"]
    B, T, Hq, Hkv, d, page = (c[n] for n in ("B", "T", "Hq", "Hkv", "d", "page"))
    L = s["most"]
    pid = s["table"][:, :L // page].long()
    k = s["k_cache"][pid].permute(0, 2, 3, 5, 1, 4).reshape(B, Hkv, d, L).float()  # [B][Hkv][d][L]
    v = s["v_cache"][pid].permute(0, 2, 1, 3, 5, 4).reshape(B, Hkv, L, d).float()
    q = s["q"].float().reshape(B, T, Hkv, Hq // Hkv, d).transpose(1, 2).reshape(B, Hkv, -1, d)
    z = torch.matmul(q, k) / math.sqrt(d)
    j = torch.arange(L, device="cuda") - s["ctx"][:, None]  # [B][L]: slot of a position, below 0 in the context
    slot = j.clamp(0, T - 1)[:, None].expand(B, T, L)
    seen = (j < 0)[:, None] | (s["vis"].gather(2, slot) & ((j >= 0) & (j < T))[:, None])
    seen = seen[:, None, :, None].expand(B, Hkv, T, Hq // Hkv, L).reshape(B, Hkv, -1, L)
    z = z.masked_fill(~seen, -math.inf)
    m = z.amax(-1, keepdim=True).clamp(min=-1e30)
    e = torch.exp(z - m)
    o = torch.matmul(e, v) / e.sum(-1, keepdim=True).clamp(min=1e-30)
    o = o.reshape(B, Hkv, T, Hq // Hkv, d).transpose(1, 2).reshape(B, T, Hq, d)
    return [torch.where(s["real"][:, :, None, None], o, 0.0).to(s["q"].dtype)]


def _plain_commit(s):
    c = s["case"]
    B, T, x = c["B"], c["T"], s["k_cache"].shape[-1]
    acc = s["accepted"].long()
    path = s["vis"][torch.arange(B, device="cuda"), acc]  # [B][T]: slots on the accepted path
    n = path.sum(1)
    m = torch.arange(T, device="cuda").expand(B, T)
    at = torch.where(path, s["depth"], T)  # a slot's place on the path
    src = m.contiguous()
    src = torch.cat([src, src[:, :1]], 1).scatter(1, at, torch.where(path, m, 0))[:, :T]
    src = torch.where(m < n[:, None], src, m)
    ctx = s["ctx"].long()[:, None]
    (ps, os), (pd, od) = ([a.reshape(-1) for a in _where(s, ctx + y)] for y in (src, m))
    kc, vc = s["k_cache"], s["v_cache"]
    kc[pd, :, :, od] = kc[ps, :, :, os]
    vc[pd, :, od // x, :, od % x] = vc[ps, :, os // x, :, os % x]
    return [kc, vc, (s["ctx"] + n).to(torch.int32)]


def _plain_sample(s):
    """Weights relative to the largest as whole numbers of 2^-31, so that sums do not depend on their order."""
    V, T = s["case"]["V"], s["case"]["T"]
    z = s["logits"].float().reshape(-1, V)
    z = torch.where(torch.isnan(z), -math.inf, z)
    t, k, p, least = (s[n].repeat_interleave(T)[:, None] for n in ("temperature", "top_k", "top_p", "min_p"))
    top = z.amax(1, keepdim=True)
    warm = t > 0
    c = torch.where(warm, t, 1.0).reciprocal() * LOG2E
    w = torch.floor(torch.exp2((z - top) * c) * 2147483648.0 + 0.5)
    w = torch.where(z == top, 2147483648.0, torch.where(warm, w, 0.0)).long()
    z, order = torch.sort(z, dim=1, descending=True, stable=True)
    ws = w.gather(1, order)
    rank = torch.arange(V, device="cuda")
    ws = torch.where((rank < k) | (k <= 0), ws, 0)
    before = ws.cumsum(1) - ws
    total = (before[:, -1:] + ws[:, -1:]).double()
    keep = ((before.double() < p.double() * total) | (rank == 0)) & (ws.double() >= least.clamp(max=1.0).double() * 2147483648.0)
    w = torch.zeros_like(w).scatter(1, order, torch.where(keep, ws, 0))
    cum = w.cumsum(1)
    want = s["u"].reshape(-1, 1).double() * cum[:, -1:].double()
    hit = torch.where(warm, cum.double() > want, w > 0)
    token = torch.where(hit, rank, V).amin(1)
    token = torch.where((top[:, 0] > -math.inf) & s["real"].reshape(-1), token, -1)
    return token.reshape(-1, T).to(torch.int32)


def _plain_accept(s, token):
    """The root and every node whose token was sampled at its parent (the lowest slot of equal siblings), down to the deepest."""
    B, T = token.shape
    real, slot = s["real"], torch.arange(T, device="cuda").expand(B, T)
    up = s["parent"].clamp(min=0)
    ok = real & (s["parent"] >= 0) & (s["draft"] == token.gather(1, up)) & (s["draft"] >= 0)
    first = torch.full((B, T + 1), T, device="cuda").scatter_reduce(1, torch.where(ok, up, T), slot, "amin")
    ok = (ok & (first.gather(1, up) == slot)) | (real & (s["parent"] == -1))
    on = real & ((s["vis"] & ~ok[:, None]).sum(2) == 0)  # every ancestor taken
    depth = torch.where(on, s["depth"], -1)
    last = depth.amax(1)
    accepted = torch.where(on & (depth == last[:, None]), slot, T).amin(1)
    out = torch.full((B, T + 1), -1, dtype=torch.int32, device="cuda")
    out = out.scatter(1, torch.where(on & (depth > 0), depth - 1, T), s["draft"])[:, :T].contiguous()
    bonus = token.gather(1, accepted[:, None].clamp(max=T - 1))
    out = out.scatter(1, last[:, None].clamp(min=0), bonus)
    return [accepted.to(torch.int32), (last + 1).to(torch.int32), out]


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def _run_own(s):
    from paper_2607_06763_amd import gdn_attn as A
    c, op = s["case"], s["op"]
    if op.startswith("sample"):
        A.sample(s["logits"], s["u"], s["token"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                 min_p=s["min_p"], meta=s["meta"])
        if op == "sample":
            return [s["token"]]
        A.accept(s["draft"], s["token"], s["accepted"], s["n_emitted"], s["emitted"], meta=s["meta"])
        return [s["token"], s["accepted"], s["n_emitted"], s["emitted"]]
    d = s.get("dims")
    if d is None:  # a program makes it once
        d = s["dims"] = A.make_attn_dims(c["B"], c["T"], c["Hq"], c["Hkv"], c["d"], c["page"], s["k_cache"].shape[0],
                                         s["table"].shape[1], dtype=c["dtype"], rot=c["rot"],
                                         n_pos=s["rope"].shape[0] if "rope" in s else 0)
    if op == "append":
        A.kv_append(d, s["q"], s["k"], s["v"], s["rope"], s["ctx"], s["table"], s["k_cache"], s["v_cache"], s["out"],
                    meta=s["meta"])
        return [s["out"], s["k_cache"], s["v_cache"]]
    if op == "attend":
        A.attend(d, s["q"], s["k_cache"], s["v_cache"], s["table"], s["ctx"], s["out"], meta=s["meta"])
        return [s["out"]]
    A.kv_commit(d, s["accepted"], s["table"], s["ctx"], s["k_cache"], s["v_cache"], s["new_len"], meta=s["meta"])
    return [s["k_cache"], s["v_cache"], s["new_len"]]


def run(s):
    """One layer's call of a decode step (or the step's sampling), and every output."""
    if own:
        return _run_own(s)
    if s["op"] == "append":
        return _plain_append(s)
    if s["op"] == "attend":
        return _plain_attend(s)
    if s["op"] == "commit":
        return _plain_commit(s)
    token = _plain_sample(s)
    return [token] if s["op"] == "sample" else [token, *_plain_accept(s, token)]


# --------------------------------------------------------------------------
# what a pass cannot do without, and the definition in 64 bits
# --------------------------------------------------------------------------
def work(case):
    """Bytes: the rows of the caches that a pass reads or writes, the inputs
    and the outputs.  Flops: two products per (query, visible key), ten
    operations per logit."""
    B, T = case["B"], case["T"]
    e = 2 if case["dtype"] == "bf16" else 4
    depth, vis = _closure(_trees(case, 0))
    n = int((depth >= 0).sum())
    if case["op"].startswith("sample"):
        return {"bytes": n * case["V"] * e + 8.0 * B * T + 16 * B, "flops": 10.0 * n * case["V"]}
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    meta = 8 * n * ((T + 63) // 64) + 4 * B * T
    if case["op"] == "append":
        return {"bytes": float(n * d * e * (2 * Hq + 4 * Hkv) + n * 4 * case["rot"] + meta), "flops": 3.0 * n * (Hq + Hkv) * case["rot"]}
    if case["op"] == "commit":
        return {"bytes": 4.0 * int((depth + 1).sum() / max(1, n) * B) * Hkv * d * e + meta, "flops": 0.0}
    ctx = _lengths(case, 0)
    rows = int(ctx.sum()) + n
    pairs = int((ctx * (depth >= 0).sum(1)).sum()) + int(vis.sum())
    return {"bytes": 2.0 * rows * Hkv * d * e + 2.0 * n * Hq * d * e + meta, "flops": 4.0 * pairs * Hq * d}


def _rows64(s, b, pos, which):
    """Rows [len(pos)][Hkv][d] of a sequence's cache in 64 bits, by the layout's own indices."""
    page, x = s["case"]["page"], s["k_cache"].shape[-1]
    p = s["table"][b].long()[pos // page]
    o = pos % page
    if which == "k":
        r = s["k_cache"][p, :, :, o]  # [n][Hkv][d / x][x]
        return r.reshape(r.shape[0], r.shape[1], -1).double()
    return s["v_cache"][p, :, o // x, :, o % x].double()


def _put64(s, cache, b, pos, rows, which):
    page, x = s["case"]["page"], s["k_cache"].shape[-1]
    p, o = s["table"][b].long()[pos // page], pos % page
    if which == "k":
        cache[p, :, :, o] = rows.reshape(rows.shape[0], rows.shape[1], -1, x)
    else:
        cache[p, :, o // x, :, o % x] = rows


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"].startswith("sample"):
        return None  # whole numbers
    B, T = case["B"], case["T"]
    ctx = s["ctx"].tolist()
    depth = s["depth"]
    if s["op"] == "attend":
        G = case["Hq"] // case["Hkv"]
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        for b in range(B):
            pos = torch.arange(ctx[b] + T, device="cuda")
            k, v = (_rows64(s, b, pos, w).transpose(0, 1).contiguous() for w in "kv")  # [Hkv][L][d]
            seen = torch.ones((T, ctx[b] + T), dtype=torch.bool, device="cuda")
            seen[:, ctx[b]:] = s["vis"][b]
            for h in range(case["Hq"]):
                z = (s["q"][b, :, h].double() @ k[h // G].T.contiguous()) * case["d"] ** -0.5
                z = z.masked_fill(~seen, -1e300)
                out[b, :, h] = torch.softmax(z, -1) @ v[h // G]
            out[b, depth[b] < 0] = 0.0
        return [out]
    kc, vc = s["k_cache"].double(), s["v_cache"].double()
    if s["op"] == "commit":
        for b in range(B):
            a = int(s["accepted"][b])
            path = sorted(torch.nonzero(s["vis"][b, a])[:, 0].tolist(), key=lambda j: int(depth[b, j]))
            src = torch.tensor(path, device="cuda") + ctx[b]
            dst = torch.arange(len(path), device="cuda") + ctx[b]
            for w, cache in (("k", kc), ("v", vc)):
                _put64(s, cache, b, dst, _rows64(s, b, src, w), w)
        return [kc, vc, None]
    h = case["rot"] // 2
    freq = s["rope"].double()
    at = s["ctx"].long()[:, None] + depth.clamp(min=0)
    turn = torch.view_as_complex(freq[at].contiguous())[:, :, None]  # [B][T][1][rot / 2]

    def turned(x):
        x = x.double().clone()
        y = torch.complex(x[..., :h], x[..., h:2 * h]) * turn
        x[..., :h], x[..., h:2 * h] = y.real, y.imag
        return x

    q, k = turned(s["q"]), turned(s["k"])
    q[depth < 0] = 0.0
    for b in range(B):
        i = torch.nonzero(depth[b] >= 0)[:, 0]
        _put64(s, kc, b, ctx[b] + i, k[b, i], "k")
        _put64(s, vc, b, ctx[b] + i, s["v"][b, i].double(), "v")
    return [q, kc, vc]
