"""The operators around a sublayer, with the names of the C ABI (include/oc.h):
norms fused with gate, modulation and residual, and their gradients; rotary
positions; products in 8-bit integers.

As in api.py this is argument marshalling only.  Tensors are on one GPU, which
need not be the current one; the work goes on that GPU's current stream.
"""
from __future__ import annotations

import contextlib
import ctypes as C
from dataclasses import dataclass
from typing import Dict, Optional, Sequence, Tuple

import torch

from . import _lib as L
from .api import Rope, Shape, _ptr


@dataclass
class Norm:
    """A norm over the channels, then weights and biases (None: 1 and 0)."""
    kind: str = "layer"      # none | rms | layer
    eps: float = 1e-6
    w: Optional[torch.Tensor] = None
    b: Optional[torch.Tensor] = None


@dataclass
class Mod:
    """Modulation vectors [n_mod, C], which may be columns of one wider
    product; rows_per_mod consecutive rows share one (None: all rows)."""
    gate: Optional[torch.Tensor] = None
    scale: Optional[torch.Tensor] = None
    shift: Optional[torch.Tensor] = None
    rows_per_mod: Optional[int] = None


_SAME = contextlib.nullcontext()


def _on(t: torch.Tensor):
    """The tensor's GPU as the current one for the call's launches."""
    return _SAME if t.device.index == torch.cuda.current_device() else torch.cuda.device(t.device)


def _stream_of(t: torch.Tensor) -> int:
    return torch.cuda.current_stream(t.device).cuda_stream


def _bad(status: int, message: str):
    return L.OmniCacheError(status, message)


def _gpu(t, name: str) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise _bad(L.OC_ERR_INVALID_ARG, f"{name} must be a GPU tensor")
    return t


def _like(t: Optional[torch.Tensor], shape, dtype, dev, name: str) -> Optional[int]:
    """The address of a contiguous tensor of this shape, type and GPU (None: NULL)."""
    if t is None:
        return None
    if _gpu(t, name).dtype != dtype:
        raise _bad(L.OC_ERR_DTYPE, f"{name} has dtype {t.dtype}, expected {dtype}")
    if t.device != dev:
        raise _bad(L.OC_ERR_INVALID_ARG, f"{name} is on {t.device}, expected {dev}")
    if t.shape != shape:
        raise _bad(L.OC_ERR_SHAPE, f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if not t.is_contiguous():
        raise _bad(L.OC_ERR_INVALID_ARG, f"{name} must be contiguous")
    return t.data_ptr()


def _norm(n: Optional[Norm], shape: Shape, dev, name: str) -> Optional[L.oc_norm]:
    if n is None:
        return None
    if n.kind not in L.NORMS:
        raise _bad(L.OC_ERR_INVALID_ARG, f"{name}: unknown norm {n.kind!r}")
    c, dt = (shape.C,), shape.torch_dtype
    return L.oc_norm(L.NORMS[n.kind], n.eps, _like(n.w, c, dt, dev, name + ".w"), _like(n.b, c, dt, dev, name + ".b"))


def _mod(m: Optional[Mod], rows: int, shape: Shape, dev) -> Optional[L.oc_mod]:
    if m is None:
        return None
    per = max(rows, 1) if m.rows_per_mod is None else m.rows_per_mod
    if per < 1:
        raise _bad(L.OC_ERR_INVALID_ARG, f"rows_per_mod={per} must be >= 1")
    n_mod, ld, at = -(-rows // per), None, []
    for name, t in (("gate", m.gate), ("scale", m.scale), ("shift", m.shift)):
        if t is None:
            at.append(None)
            continue
        if _gpu(t, name).dtype != shape.torch_dtype:
            raise _bad(L.OC_ERR_DTYPE, f"{name} has dtype {t.dtype}, expected {shape.torch_dtype}")
        if t.device != dev:
            raise _bad(L.OC_ERR_INVALID_ARG, f"{name} is on {t.device}, expected {dev}")
        if t.dim() == 1:
            t = t[None]
        if t.shape != (n_mod, shape.C):
            raise _bad(L.OC_ERR_SHAPE, f"{name} has shape {tuple(t.shape)}, expected {(n_mod, shape.C)}")
        if t.stride(1) != 1 and shape.C > 1:
            raise _bad(L.OC_ERR_INVALID_ARG, f"the channels of {name} must be contiguous")
        row = t.stride(0) if n_mod > 1 else shape.C
        if ld is not None and row != ld:
            raise _bad(L.OC_ERR_INVALID_ARG, "gate, scale and shift must have the same row stride")
        ld = row
        at.append(t.data_ptr())
    return L.oc_mod(*at, shape.C if ld is None else ld, per, 0)


def _rows_of(x: torch.Tensor, shape: Shape) -> int:
    if _gpu(x, "x").dim() < 1 or x.shape[-1] != shape.C:
        raise _bad(L.OC_ERR_SHAPE, f"x has shape {tuple(x.shape)}, expected [..., {shape.C}]")
    return x.numel() // shape.C


def _ref(s):
    return None if s is None else C.byref(s)


def norm_gate(x: torch.Tensor, shape: Shape, y: Optional[torch.Tensor] = None, post: Optional[Norm] = None,
              pre: Optional[Norm] = None, mod: Optional[Mod] = None, res_scale: float = 1.0, h=None, n=None):
    """oc_norm_gate: h = res_scale x + gate post(y) and n = pre(h)(1 + scale) +
    shift over the last dimension.  h and n: a tensor to write (x or y
    themselves are possible), None (a new one) or False (not wanted).  Without
    y, h is x.  Returns (h, n)."""
    rows = _rows_of(x, shape)
    dev, dt, full = x.device, shape.torch_dtype, x.shape
    xp, yp = _like(x, full, dt, dev, "x"), _like(y, full, dt, dev, "y")
    if y is None:
        if h is not None and h is not False:
            raise _bad(L.OC_ERR_INVALID_ARG, "h is x where y is None")
        h = False
    h = torch.empty_like(x) if h is None else h
    n = torch.empty_like(x) if n is None else n
    hp = None if h is False else _like(h, full, dt, dev, "h")
    np_ = None if n is False else _like(n, full, dt, dev, "n")
    sh, po, pr, mo = shape.c(), _norm(post, shape, dev, "post"), _norm(pre, shape, dev, "pre"), _mod(mod, rows, shape, dev)
    if rows == 0:      # (empty tensors have no address)
        hp = np_ = xp = yp = None
    with _on(x):
        L.check(L.lib().oc_norm_gate(C.byref(sh), rows, xp, yp, _ref(po), _ref(pr), _ref(mo), res_scale, hp, np_,
                                     _stream_of(x)))
    return (x if y is None else None if h is False else h), (None if n is False else n)


def norm_gate_grad_workspace_bytes(shape: Shape, rows: int, rows_per_mod: int = 0) -> int:
    sh = shape.c()
    return int(L.lib().oc_norm_gate_grad_workspace_bytes(C.byref(sh), rows, rows_per_mod))


def norm_gate_grad(x: torch.Tensor, shape: Shape, dn: Optional[torch.Tensor] = None,
                   dh: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None, post: Optional[Norm] = None,
                   pre: Optional[Norm] = None, mod: Optional[Mod] = None, res_scale: float = 1.0,
                   want: Optional[Sequence[str]] = None,
                   ws: Optional[torch.Tensor] = None) -> Dict[str, Optional[torch.Tensor]]:
    """oc_norm_gate_grad: the gradients of norm_gate's inputs from those of its
    outputs (None: zero), as a dict with dx, dy (like x) and, in fp32, gate,
    scale, shift [n_mod, C], post_w, post_b, pre_w, pre_b [C]; None for what
    the call has not, or what `want` (None: everything) leaves out."""
    rows = _rows_of(x, shape)
    dev, dt, full = x.device, shape.torch_dtype, x.shape
    xp, yp = _like(x, full, dt, dev, "x"), _like(y, full, dt, dev, "y")
    dnp, dhp = _like(dn, full, dt, dev, "dn"), _like(dh, full, dt, dev, "dh")
    sh, po, pr, mo = shape.c(), _norm(post, shape, dev, "post"), _norm(pre, shape, dev, "pre"), _mod(mod, rows, shape, dev)
    per = mo.rows_per_mod if mo is not None else 0
    n_mod = -(-rows // per) if per else 0
    has = {"dx": True, "dy": y is not None}
    has.update({k: getattr(mo, k) is not None if mo is not None else False for k in ("gate", "scale", "shift")})
    for k, s in (("post", po), ("pre", pr)):
        has.update({k + "_w": s is not None and s.w is not None, k + "_b": s is not None and s.b is not None})
    if want is not None and not set(want) <= set(has):
        raise _bad(L.OC_ERR_INVALID_ARG, f"unknown gradients {sorted(set(want) - set(has))}")
    out = {}
    for k, there in has.items():
        if not there or (want is not None and k not in want):
            out[k] = None
        elif k in ("dx", "dy"):
            out[k] = torch.empty_like(x)
        else:
            out[k] = torch.empty((n_mod, shape.C) if k in ("gate", "scale", "shift") else (shape.C,),
                                 dtype=torch.float32, device=dev)
    if ws is None:
        ws = torch.empty(max(norm_gate_grad_workspace_bytes(shape, rows, per), 256), dtype=torch.uint8, device=dev)
    elif _gpu(ws, "ws").device != dev or not ws.is_contiguous():
        raise _bad(L.OC_ERR_INVALID_ARG, f"ws must be contiguous and on {dev}")
    g = L.oc_norm_grads(*(_ptr(out[k]) for k in ("gate", "scale", "shift", "post_w", "post_b", "pre_w", "pre_b")))
    with _on(x):
        L.check(L.lib().oc_norm_gate_grad(C.byref(sh), rows, xp, yp, _ref(po), _ref(pr), _ref(mo), res_scale, dhp, dnp,
                                          _ptr(out["dx"]), _ptr(out["dy"]), C.byref(g), ws.data_ptr(),
                                          ws.numel() * ws.element_size(), _stream_of(x)))
    return out


def _heads_of(t: Optional[torch.Tensor], rows: Optional[int], heads: Optional[int], shape: Shape, dev, name: str):
    """(address, row stride, heads) of a [rows, heads, head_dim] tensor whose
    rows hold their heads contiguously."""
    if t is None:
        return None, 0, 0
    if _gpu(t, name).dtype != shape.torch_dtype:
        raise _bad(L.OC_ERR_DTYPE, f"{name} has dtype {t.dtype}, expected {shape.torch_dtype}")
    if dev is not None and t.device != dev:
        raise _bad(L.OC_ERR_INVALID_ARG, f"{name} is on {t.device}, expected {dev}")
    if t.dim() != 3 or t.shape[2] != shape.head_dim or (rows is not None and t.shape[0] != rows) or \
            (heads is not None and t.shape[1] != heads):
        raise _bad(L.OC_ERR_SHAPE, f"{name} has shape {tuple(t.shape)}, expected "
                                   f"{('rows' if rows is None else rows, 'heads' if heads is None else heads, shape.head_dim)}")
    if t.stride(2) != 1 or (t.shape[1] > 1 and t.stride(1) != shape.head_dim):
        raise _bad(L.OC_ERR_INVALID_ARG, f"the heads of a row of {name} must be contiguous")
    return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else t.shape[1] * t.shape[2], t.shape[1]


def _ids(t: Optional[torch.Tensor], shape, dev, name: str) -> Optional[int]:
    return _like(t, torch.Size(shape), torch.int32, dev, name)


def rope_qk(q: Optional[torch.Tensor], k: Optional[torch.Tensor], rope: Rope, shape: Shape,
            kept_idx: Optional[torch.Tensor] = None, pos: Optional[torch.Tensor] = None, inverse: bool = False,
            q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None
            ) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """oc_rope_qk: q [rows, heads, head_dim] and k [rows, k_heads, head_dim]
    (rows may be columns of a wider buffer) turned by their tokens' positions:
    token kept_idx[r] (None: r) of the shape's grid, or pos [rows, 3] int32.
    inverse: turned back, which is also the gradient.  q_out and k_out: new
    contiguous tensors unless given (q and k themselves: in place)."""
    first = q if q is not None else k
    if first is None:
        raise _bad(L.OC_ERR_INVALID_ARG, "neither q nor k is given")
    rows, dev = _gpu(first, "q").shape[0], first.device
    qp, ldq, _ = _heads_of(q, rows, shape.heads, shape, dev, "q")
    kp, ldk, kh = _heads_of(k, rows, None, shape, dev, "k")
    if q_out is None and q is not None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=dev)
    if k_out is None and k is not None:
        k_out = torch.empty(k.shape, dtype=k.dtype, device=dev)
    qop, ldqo, _ = _heads_of(q_out, rows, shape.heads, shape, dev, "q_out")
    kop, ldko, _ = _heads_of(k_out, rows, kh, shape, dev, "k_out")
    ip, pp = _ids(kept_idx, (rows,), dev, "kept_idx"), _ids(pos, (rows, 3), dev, "pos")
    if rows == 0:      # (empty tensors have no address)
        qp = kp = qop = kop = None
    sh, ro = shape.c(), rope.c()
    with _on(first):
        L.check(L.lib().oc_rope_qk(C.byref(sh), C.byref(ro), rows, ip, pp, qp, ldq, kp, ldk, kh, qop, ldqo, kop, ldko,
                                   1 if inverse else 0, _stream_of(first)))
    return q_out, k_out


_DTYPES = {torch.float32: L.OC_F32, torch.bfloat16: L.OC_BF16}


def _matrix(t, name: str):
    """(address, row stride) of a 2-D tensor with contiguous rows."""
    if _gpu(t, name).dtype not in _DTYPES:
        raise _bad(L.OC_ERR_DTYPE, f"{name} has dtype {t.dtype}, expected bfloat16 or float32")
    if t.dim() != 2:
        raise _bad(L.OC_ERR_SHAPE, f"{name} has shape {tuple(t.shape)}, expected two dimensions")
    if t.stride(1) != 1 and t.shape[1] > 1:
        raise _bad(L.OC_ERR_INVALID_ARG, f"the rows of {name} must be contiguous")
    return t.data_ptr() or None, t.stride(0) if t.shape[0] > 1 else t.shape[1]


def quant_rows(x: torch.Tensor, row_idx: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None,
               scale: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """oc_quant_rows: the rows row_idx (None: all) of x [n, K] in 8 bits.
    Returns (q int8 [rows, K rounded up to 16], scale fp32 [rows]); x is about
    q * scale.  Weights [out, in] are quantised by the same call, once."""
    at, ld = _matrix(x, "x")
    dev, (n, K) = x.device, x.shape
    rows = n if row_idx is None else row_idx.numel()
    ip = _ids(row_idx, (rows,), dev, "row_idx")
    Kp = (K + 15) // 16 * 16
    q = torch.empty((rows, Kp), dtype=torch.int8, device=dev) if q is None else q
    scale = torch.empty((rows,), dtype=torch.float32, device=dev) if scale is None else scale
    qp, sp = _like(q, (rows, Kp), torch.int8, dev, "q"), _like(scale, (rows,), torch.float32, dev, "scale")
    with _on(x):
        L.check(L.lib().oc_quant_rows(_DTYPES[x.dtype], at, ld, n, K, ip, rows, qp, sp, _stream_of(x)))
    return q, scale


def linear_i8(q: torch.Tensor, scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor,
              bias: Optional[torch.Tensor] = None, act: str = "none", out_idx: Optional[torch.Tensor] = None,
              y: Optional[torch.Tensor] = None, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """oc_linear_i8: act((q w^T) scale w_scale + bias) of quantised rows q
    [rows, K'] and weights w [N, K'] (both as quant_rows gives them).  y: a
    tensor to write, its rows out_idx (None: the first ones), whose other rows
    stay as they are; or None: a new [rows, N] tensor of type dtype (bfloat16
    unless given)."""
    dev = _gpu(q, "q").device
    if q.dim() != 2 or _gpu(w, "w").dim() != 2:
        raise _bad(L.OC_ERR_SHAPE, "q and w must have two dimensions")
    (rows, Kp), N = q.shape, w.shape[0]
    if act not in L.ACTS:
        raise _bad(L.OC_ERR_INVALID_ARG, f"unknown activation {act!r}")
    if Kp % 16:
        raise _bad(L.OC_ERR_SHAPE, f"q has {Kp} columns, expected a multiple of 16")
    qp, wp = _like(q, (rows, Kp), torch.int8, dev, "q"), _like(w, (N, Kp), torch.int8, dev, "w")
    sp = _like(scale, (rows,), torch.float32, dev, "scale")
    swp = _like(w_scale, (N,), torch.float32, dev, "w_scale")
    if y is None:
        if out_idx is not None:
            raise _bad(L.OC_ERR_INVALID_ARG, "out_idx needs y, the tensor whose rows it names")
        y = torch.empty((rows, N), dtype=torch.bfloat16 if dtype is None else dtype, device=dev)
    at, ld = _matrix(y, "y")
    if y.device != dev or y.shape[1] != N or (dtype is not None and y.dtype != dtype):
        raise _bad(L.OC_ERR_SHAPE, f"y is {tuple(y.shape)} {y.dtype} on {y.device}, expected [..., {N}] on {dev}")
    bp = _like(bias, (N,), y.dtype, dev, "bias")
    ip = _ids(out_idx, (rows,), dev, "out_idx")
    with _on(q):
        L.check(L.lib().oc_linear_i8(_DTYPES[y.dtype], rows, Kp, N, qp, sp, wp, swp, bp, L.ACTS[act], ip, y.shape[0],
                                     at, ld, _stream_of(q)))
    return y
