"""Python binding of the calls of libgdntree (include/gdn_tree.h) for layers
without draft trees: argument marshalling only, as ``gdn_tree``.

A GDN layer over prompts or single tokens, and the residual stream around it::

    L.chain(d, q, k, v, alpha, beta, conv_w, conv, conv_next, S, o, start=start)
    L.gate_norm(o, gate, y, weight=w)                    # then the output projection
    L.add_norm(p, residual, residual, x, weight=w2)      # the next block's input

``chain`` of more than 20 tokens a sequence works in a buffer that the library
keeps per stream (the header's "Workspaces"): before a capture the same sizes
run once uncaptured on the capture stream, and a graph must not run at the same
time as other such calls of that stream, or as another graph captured there.
"""
from __future__ import annotations

import ctypes
import functools

from .gdn_tree import GDN_BF16, GDN_F32, _check, _ptrs, _stream, lib

ACTS = {"silu": 0, "sigmoid": 1}
MAX_CHAIN_T = 1 << 24  # GDN_MAX_CHAIN_T of gdn_tree.h
STEP_T = 20  # GDN_CHAIN_STEP_T
MAX_NORM_D = 16384  # GDN_MAX_NORM_D


class ChainDims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "T", "Hk", "Hv", "dk", "dv", "in_dtype", "out_dtype")] + \
        [("rows", ctypes.c_int64), ("scale", ctypes.c_float)]

    def __setattr__(self, name, value):
        super().__setattr__(name, value)
        self.__dict__.pop("_shapes", None)

    def shapes(self, packed):
        """dtypes and the shapes of q and k, v, the gates, out, conv_w, the conv states, S and lengths; made once for these
        sizes (reading the fields takes longer than the call)."""
        import torch
        s = self.__dict__.get("_shapes")
        if s is None or s[0] is not packed:
            B, Hk, Hv, dk, dv = self.B, self.Hk, self.Hv, self.dk, self.dv
            C = 2 * Hk * dk + Hv * dv
            lead = (self.rows,) if packed else (B, self.T)
            t = lambda x: torch.bfloat16 if x == GDN_BF16 else torch.float32
            s = (packed, t(self.in_dtype), t(self.out_dtype), (*lead, Hk, dk), (*lead, Hv, dv), (*lead, Hv), (C, 4), (B, 3, C),
                 (B, Hv, dv, dk), (B,))
            self.__dict__["_shapes"] = s
        return s[1:]

    def __repr__(self):
        return "ChainDims(" + ", ".join(f"{n}={getattr(self, n)}" for n, _ in self._fields_) + ")"


class GateNormDims(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int64)] + [(n, ctypes.c_int32) for n in ("H", "d", "x_dtype", "gate_dtype", "out_dtype", "act")] + \
        [("ldx", ctypes.c_int64), ("ldg", ctypes.c_int64), ("eps", ctypes.c_float)]


class AddNormDims(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int64)] + [(n, ctypes.c_int32) for n in ("D", "x_dtype", "res_dtype", "out_dtype", "post")] + \
        [("eps", ctypes.c_float)]


def _dtype(name):
    return GDN_BF16 if name in ("bf16", GDN_BF16) else GDN_F32


def make_chain_dims(B, T, Hk, Hv, dk, dv, in_dtype="bf16", out_dtype="f32", rows=0, scale=0.0) -> ChainDims:
    """B sequences of up to T tokens; rows: of packed tensors (a call with start)."""
    return ChainDims(B, T, Hk, Hv, dk, dv, _dtype(in_dtype), _dtype(out_dtype), rows, float(scale))


def chain(d: ChainDims, q, k, v, alpha, beta, conv_w, conv_state, conv_state_out, S, out, start=None, n_new=None, status=None,
          stream=None) -> None:
    """gdn_chain: the gated delta rule over sequences; S in place, conv_state to
    conv_state_out.  Tensors [B][T][...] (n_new int32 [B]: tokens of each), or
    packed [rows][...] with start int32 [B + 1], which does not go backwards
    (status 9 for a sequence that would take rows of one before it)."""
    import torch
    i32, f32 = torch.int32, torch.float32
    it, ot, ks, vs, gs, ws, cs, ss, ls = d.shapes(start is not None)
    _check(lib().gdn_chain(ctypes.byref(d), *_ptrs((
        (start, (d.B + 1,), i32, "start", None), (n_new, ls, i32, "n_new", None), (q, ks, it, "q"), (k, ks, it, "k"),
        (v, vs, it, "v"), (alpha, gs, it, "alpha"), (beta, gs, it, "beta"), (conv_w, ws, f32, "conv_w"),
        (conv_state, cs, f32, "conv_state"), (conv_state_out, cs, f32, "conv_state_out"), (S, ss, f32, "S"),
        (out, vs, ot, "out"), (status, ls, i32, "status", None))), _stream(stream)))


_codes = {}  # type codes of the norms' tensors


def _code(dtype):
    if not _codes:
        import torch
        _codes.update({torch.bfloat16: GDN_BF16, torch.float32: GDN_F32})
    return _codes.get(dtype)


def _rows(t, shape, name, device, ld=False):
    """Pointer, type code and row stride of a bf16 or fp32 device tensor of this shape; ld: rows may be further apart
    (stride 0: they are not).  A tensor that is right takes the first lines; a call of few rows is bound by them."""
    try:
        code = _codes.get(t.dtype)
        if code is not None and t.shape == shape and t.is_contiguous() and t.get_device() == device:
            return t.data_ptr(), code, 0
    except AttributeError:
        raise TypeError(f"{name}: expected a torch.Tensor") from None
    code = _code(t.dtype)
    if code is None:
        raise ValueError(f"{name}: dtype {t.dtype}, expected bfloat16 or float32")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if not t.is_cuda:
        raise ValueError(f"{name}: must be a device tensor")
    if t.get_device() != device:
        raise ValueError(f"{name}: on {t.device}, expected the current device {device}")
    if t.is_contiguous():
        return t.data_ptr(), code, 0
    # every row contiguous, all of them equally far apart
    if not ld or t.shape[0] < 1 or not t[0].is_contiguous() or (t.shape[0] > 1 and t.stride(0) < t[0].numel()):
        raise ValueError(f"{name}: strides {t.stride()}, expected " + ("contiguous rows" if ld else "contiguous"))
    return t.data_ptr(), code, t.stride(0) if t.shape[0] > 1 else 0


def _param(t, n, name, device):
    if t is None:
        return None
    try:
        if _codes.get(t.dtype) == GDN_F32 and t.shape == (n,) and t.is_contiguous() and t.get_device() == device:
            return t.data_ptr()
    except AttributeError:
        raise TypeError(f"{name}: expected a torch.Tensor") from None
    if _code(t.dtype) != GDN_F32 or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)}, expected contiguous float32 ({n},)")
    if not t.is_cuda or t.get_device() != device:
        raise ValueError(f"{name}: on {t.device}, expected the current device {device}")
    return t.data_ptr()


# dims of the norms by their sizes: making one takes as long as the checks
@functools.lru_cache(maxsize=256, typed=True)
def _gate_dims(*sizes):
    d = GateNormDims(*sizes)
    return d, ctypes.byref(d)


@functools.lru_cache(maxsize=256, typed=True)
def _add_dims(*sizes):
    d = AddNormDims(*sizes)
    return d, ctypes.byref(d)


def gate_norm(x, gate, out, weight=None, eps=1e-6, act="silu", stream=None) -> None:
    """gdn_gate_norm: out = x / sqrt(mean(x^2) + eps) * weight * act(gate) over
    the last dim of [N][H][d] tensors, bf16 or fp32 each; the rows [H][d] of x and
    gate may be apart.  gate None: no gate; act "silu" or "sigmoid"; out may be x."""
    import torch
    if not isinstance(x, torch.Tensor):
        raise TypeError("x: expected a torch.Tensor")
    if x.dim() != 3:
        raise ValueError(f"x: shape {tuple(x.shape)}, expected [N][H][d]")
    if act not in ACTS:
        raise ValueError(f"act: {act!r}, expected 'silu' or 'sigmoid'")
    dev, shape = torch._C._cuda_getDevice(), x.shape
    px, tx, ldx = _rows(x, shape, "x", dev, ld=True)
    pg, tg, ldg = (None, GDN_F32, 0) if gate is None else _rows(gate, shape, "gate", dev, ld=True)
    po, to, _ = _rows(out, shape, "out", dev)
    N, H, d = shape
    dims = _gate_dims(N, H, d, tx, tg, to, ACTS[act], ldx, ldg, eps)
    _check(lib().gdn_gate_norm(dims[1], px, pg, _param(weight, d, "weight", dev), po, _stream(stream)))


def add_norm(x, residual, res_out, out, weight=None, post_weight=None, scale=None, post=False, eps=1e-6, stream=None) -> None:
    """gdn_add_norm: res_out = residual + scale * x, with post x normed first
    (times post_weight); out = res_out / sqrt(mean(res_out^2) + eps) * weight.
    Tensors [N][D], bf16 or fp32 each (residual and res_out the same); residual
    None: 0, res_out or out None: not written.  res_out may be residual, out x."""
    import torch
    if not isinstance(x, torch.Tensor):
        raise TypeError("x: expected a torch.Tensor")
    if x.dim() != 2:
        raise ValueError(f"x: shape {tuple(x.shape)}, expected [N][D]")
    dev, shape = torch._C._cuda_getDevice(), x.shape
    px, tx, _ = _rows(x, shape, "x", dev)
    pr, tr, _ = (None, None, 0) if residual is None else _rows(residual, shape, "residual", dev)
    pro, tro, _ = (None, tr, 0) if res_out is None else _rows(res_out, shape, "res_out", dev)
    if None not in (tr, tro) and tr != tro:
        raise ValueError("res_out: another dtype than residual")
    po, to, _ = (None, GDN_F32, 0) if out is None else _rows(out, shape, "out", dev)
    N, D = shape
    t = tro if tr is None else tr
    dims = _add_dims(N, D, tx, GDN_F32 if t is None else t, to, 1 if post else 0, eps)
    w, pw, sc = _param(weight, D, "weight", dev), _param(post_weight, D, "post_weight", dev), _param(scale, D, "scale", dev)
    _check(lib().gdn_add_norm(dims[1], px, pr, w, pw, sc, pro, po, _stream(stream)))
