"""Python binding of the softmax-attention and sampling calls of libgdntree
(include/gdn_tree.h): argument marshalling only, as ``gdn_tree``.

A decode step of a model that has both kinds of layers::

    G.prepare(dims, parent, meta)                        # once per step
    G.step(...)                                          # GDN layers
    A.kv_append(d, q, k, v, rope, ctx_len, table, kc, vc, q_rot, meta=meta)   # attention layers
    A.attend(d, q_rot, kc, vc, table, ctx_len, out, meta=meta)
    A.sample(logits, u, token, temperature=t, top_p=p, meta=meta)             # once per step
    A.accept(draft, token, accepted, n_emitted, emitted, meta=meta)
    A.kv_commit(d, accepted, table, ctx_len, kc, vc, new_len, meta=meta)      # attention layers

``attend`` works in a buffer that the library keeps per stream (the header's
"Workspaces"): before a capture the same sizes run once uncaptured on the
capture stream, and a graph must not run at the same time as other calls of
that stream, or as another graph captured there.
"""
from __future__ import annotations

import ctypes

from .gdn_tree import GDN_BF16, GDN_F32, Dims, _check, _ptrs, _stream, lib, meta_bytes

PAGES = (16, 32, 64, 128, 256)
MAX_V = 1 << 20  # GDN_MAX_V of gdn_tree.h


class AttnDims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "T", "Hq", "Hkv", "d", "page", "n_pages", "max_pages", "dtype",
                                              "rot", "n_pos")] + [("scale", ctypes.c_float)]

    def __setattr__(self, name, value):
        super().__setattr__(name, value)
        self.__dict__.pop("_shapes", None)

    def shapes(self):
        """dtype and the shapes of q, k, the caches, a page table, lengths, the rotation table and the metadata; made
        once for these sizes (reading the fields takes longer than the call)."""
        import torch
        s = self.__dict__.get("_shapes")
        if s is None:
            B, T, d, page = self.B, self.T, self.d, self.page
            bf16 = self.dtype == GDN_BF16
            x = 8 if bf16 else 4
            s = (torch.bfloat16 if bf16 else torch.float32, (B, T, self.Hq, d), (B, T, self.Hkv, d),
                 (self.n_pages, self.Hkv, d // x, page, x), (self.n_pages, self.Hkv, page // x, d, x),
                 (B, self.max_pages), (B,), (self.n_pos, self.rot // 2, 2) if self.rot else None, (meta_bytes(B, T),))
            self.__dict__["_shapes"] = s
        return s

    def __repr__(self):
        return "AttnDims(" + ", ".join(f"{n}={getattr(self, n)}" for n, _ in self._fields_) + ")"


class SampleDims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "T", "V", "dtype")] + [("ld", ctypes.c_int64)]


def make_attn_dims(B, T, Hq, Hkv, d, page, n_pages, max_pages, dtype="bf16", rot=None, n_pos=0, scale=0.0) -> AttnDims:
    dt = GDN_BF16 if dtype in ("bf16", GDN_BF16) else GDN_F32
    return AttnDims(B, T, Hq, Hkv, d, page, n_pages, max_pages, dt, d if rot is None else rot, n_pos, float(scale))


def cache_shapes(d: AttnDims):
    """Shapes of the key and the value cache."""
    return d.shapes()[3:5]


def gather_rows(d: AttnDims, k_cache, v_cache, page_table, n: int):
    """Keys and values of positions 0 .. n - 1 of every sequence as [B][n][Hkv][d] tensors (torch indexing, for
    inspection; every page-table entry of these positions must be in range)."""
    import torch
    x = k_cache.shape[-1]
    pos = torch.arange(n, device=page_table.device)
    pg, off = page_table.long()[:, pos // d.page], pos % d.page
    k = k_cache[pg, :, :, off].reshape(pg.shape[0], n, d.Hkv, d.d)
    return k, v_cache[pg, :, off // x, :, off % x]


def kv_append(d: AttnDims, q, k, v, rope, ctx_len, page_table, k_cache, v_cache, q_out, kv_status=None, meta=None,
              n_new=None, stream=None) -> None:
    """gdn_kv_append: rotates q into q_out (which may be q) and k, and appends
    k and v to the paged caches; rope fp32 [n_pos][rot / 2][2] (None for rot 0)."""
    import torch
    i32 = torch.int32
    dt, qs, ks, kc, vc, ts, ls, rs, ms = d.shapes()
    _check(lib().gdn_kv_append(ctypes.byref(d), *_ptrs((
        (meta, ms, torch.uint8, "meta", None), (n_new, ls, i32, "n_new", None), (q, qs, dt, "q"), (k, ks, dt, "k"),
        (v, ks, dt, "v"), (rope, rs, torch.float32, "rope") if rs else (None, rs, None, "rope", None),
        (ctx_len, ls, i32, "ctx_len"), (page_table, ts, i32, "page_table"), (k_cache, kc, dt, "k_cache"),
        (v_cache, vc, dt, "v_cache"), (q_out, qs, dt, "q_out"), (kv_status, ls, i32, "kv_status", None))),
        _stream(stream)))


def attend(d: AttnDims, q, k_cache, v_cache, page_table, ctx_len, out, meta=None, n_new=None, stream=None) -> None:
    """gdn_tree_attend: attention of every slot over the cached tokens, its
    ancestors and itself; q as rotated by kv_append."""
    import torch
    i32 = torch.int32
    dt, qs, _, kc, vc, ts, ls, _, ms = d.shapes()
    _check(lib().gdn_tree_attend(ctypes.byref(d), *_ptrs((
        (meta, ms, torch.uint8, "meta", None), (n_new, ls, i32, "n_new", None), (q, qs, dt, "q"),
        (k_cache, kc, dt, "k_cache"), (v_cache, vc, dt, "v_cache"), (page_table, ts, i32, "page_table"),
        (ctx_len, ls, i32, "ctx_len"), (out, qs, dt, "out"))), _stream(stream)))


def kv_commit(d: AttnDims, accepted, page_table, ctx_len, k_cache, v_cache, new_len, kv_status=None, meta=None,
              stream=None) -> None:
    """gdn_kv_commit: moves the accepted path's rows to the front of the new
    rows of both caches, in place; new_len = ctx_len + depth + 1."""
    import torch
    i32 = torch.int32
    dt, _, _, kc, vc, ts, ls, _, ms = d.shapes()
    _check(lib().gdn_kv_commit(ctypes.byref(d), *_ptrs((
        (meta, ms, torch.uint8, "meta", None), (accepted, ls, i32, "accepted"), (page_table, ts, i32, "page_table"),
        (ctx_len, ls, i32, "ctx_len"), (k_cache, kc, dt, "k_cache"), (v_cache, vc, dt, "v_cache"),
        (new_len, ls, i32, "new_len"), (kv_status, ls, i32, "kv_status", None))), _stream(stream)))


def sample(logits, u, token, temperature=None, top_k=None, top_p=None, min_p=None, meta=None, stream=None) -> None:
    """gdn_tree_sample: token int32 [B][T] from logits [B][T][V] (bf16 or
    fp32; rows may be further apart than V elements) and u fp32 [B][T]."""
    import torch
    if not isinstance(logits, torch.Tensor):
        raise TypeError("logits: expected a torch.Tensor")
    if logits.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"logits: dtype {logits.dtype}, expected bfloat16 or float32")
    if logits.dim() != 3:
        raise ValueError(f"logits: shape {tuple(logits.shape)}, expected [B][T][V]")
    if not logits.is_cuda:
        raise ValueError("logits: must be a device tensor")
    B, T, V = logits.shape
    sb, ld, sv = logits.stride()
    if T == 1:
        ld = sb if B > 1 else V
    if (V > 1 and sv != 1) or ld < V or (B > 1 and sb != T * ld):
        raise ValueError(f"logits: strides {logits.stride()}, expected (T ld, ld, 1) with ld >= V")
    p = logits.data_ptr()
    if p % 16:
        raise ValueError("logits: must be 16-byte aligned")
    f32, i32 = torch.float32, torch.int32
    d = SampleDims(B, T, V, GDN_BF16 if logits.dtype is torch.bfloat16 else GDN_F32, ld)
    m, t, k, tp, mp, pu, pt = _ptrs((
        (meta, (meta_bytes(B, T),), torch.uint8, "meta", None), (temperature, (B,), f32, "temperature", None),
        (top_k, (B,), i32, "top_k", None), (top_p, (B,), f32, "top_p", None), (min_p, (B,), f32, "min_p", None),
        (u, (B, T), f32, "u"), (token, (B, T), i32, "token")))
    _check(lib().gdn_tree_sample(ctypes.byref(d), m, p, t, k, tp, mp, pu, pt, _stream(stream)))


def accept(draft, token, accepted, n_emitted, emitted, meta=None, stream=None) -> None:
    """gdn_tree_accept: the accepted slot of every tree (for commit, step and
    kv_commit) and the emitted tokens, from the draft tokens [B][T] and the
    sampled ones."""
    import torch
    i32 = torch.int32
    if not isinstance(draft, torch.Tensor):
        raise TypeError("draft: expected a torch.Tensor")
    if draft.dim() != 2:
        raise ValueError(f"draft: shape {tuple(draft.shape)}, expected [B][T]")
    B, T = draft.shape
    d = Dims(B, T, 1, 1, 16, 16, GDN_F32, 0.0)
    _check(lib().gdn_tree_accept(ctypes.byref(d), *_ptrs((
        (meta, (meta_bytes(B, T),), torch.uint8, "meta", None), (draft, (B, T), i32, "draft"),
        (token, (B, T), i32, "token"), (accepted, (B,), i32, "accepted"), (n_emitted, (B,), i32, "n_emitted"),
        (emitted, (B, T), i32, "emitted"))), _stream(stream)))
