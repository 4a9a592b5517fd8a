"""The operators around a sublayer, with the names of the C ABI (include/oc.h):
norms fused with gate, modulation and residual, and their gradients; rotary
positions; products in 8-bit integers.

As in api.py this is argument marshalling only.  Tensors are on one GPU, which
need not be the current one; the work goes on that GPU's current stream.
"""
from __future__ import annotations

import ctypes as C
import functools
from dataclasses import dataclass
from typing import Dict, Optional, Sequence, Tuple

import torch

from . import _lib as L
from .api import Rope, Shape


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


def _bad(status: int, message: str):
    return L.OmniCacheError(status, message)


def _call(name: str, dev: torch.device, *args) -> None:
    """The C call with the stream last: the tensors' GPU as the current one for
    its launches, and that GPU's current stream."""
    fn, idx = getattr(L.lib(), name), dev.index
    if torch._C._cuda_getDevice() == idx:
        status = fn(*args, torch._C._cuda_getCurrentRawStream(idx))
    else:
        with torch.cuda.device(idx):
            status = fn(*args, torch._C._cuda_getCurrentRawStream(idx))
    if status:
        L.check(status)


@functools.lru_cache(maxsize=256)
def _made(v):
    return C.byref(v.c())


def _struct(v):
    """C.byref of the C struct of a Shape or Rope, made once for equal ones (the
    library only reads it)."""
    try:
        return _made(v)
    except TypeError:      # (a Rope of lists has no hash)
        return C.byref(v.c())


def _gpu(t, name: str) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise _bad(L.OC_ERR_INVALID_ARG, f"{name} must be a GPU tensor")
    return t


def _like(t: Optional[torch.Tensor], shape, dtype, dev, name: str) -> Optional[int]:
    """The address of a contiguous tensor of this shape, type and GPU (None: NULL)."""
    if t is None:
        return None
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.device == dev and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    if _gpu(t, name).dtype != dtype:
        raise _bad(L.OC_ERR_DTYPE, f"{name} has dtype {t.dtype}, expected {dtype}")
    if t.device != dev:
        raise _bad(L.OC_ERR_INVALID_ARG, f"{name} is on {t.device}, expected {dev}")
    if t.shape != shape:
        raise _bad(L.OC_ERR_SHAPE, f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    raise _bad(L.OC_ERR_INVALID_ARG, f"{name} must be contiguous")


def _norm(n: Optional[Norm], shape: Shape, dev, name: str) -> Optional[L.oc_norm]:
    if n is None:
        return None
    kind = L.NORMS.get(n.kind)
    if kind is None:
        raise _bad(L.OC_ERR_INVALID_ARG, f"{name}: unknown norm {n.kind!r}")
    if n.w is None and n.b is None:
        return L.oc_norm(kind, n.eps)
    c, dt = (shape.C,), shape.torch_dtype
    return L.oc_norm(kind, n.eps, _like(n.w, c, dt, dev, name + ".w"), _like(n.b, c, dt, dev, name + ".b"))


def _mod(m: Optional[Mod], rows: int, shape: Shape, dev) -> Optional[L.oc_mod]:
    if m is None:
        return None
    per = max(rows, 1) if m.rows_per_mod is None else m.rows_per_mod
    if per < 1:
        raise _bad(L.OC_ERR_INVALID_ARG, f"rows_per_mod={per} must be >= 1")
    n_mod, ld, at, dt, Ch = -(-rows // per), None, [], shape.torch_dtype, shape.C
    for name, t in (("gate", m.gate), ("scale", m.scale), ("shift", m.shift)):
        if t is None:
            at.append(None)
            continue
        if _gpu(t, name).dtype != dt:
            raise _bad(L.OC_ERR_DTYPE, f"{name} has dtype {t.dtype}, expected {dt}")
        if t.device != dev:
            raise _bad(L.OC_ERR_INVALID_ARG, f"{name} is on {t.device}, expected {dev}")
        size, step = t.shape, t.stride()
        # (no rows: the vector of all of them is one all the same)
        if size != (n_mod, Ch) and not ((n_mod == 1 and size == (Ch,)) or (
                rows == 0 and m.rows_per_mod is None and size in ((1, Ch), (Ch,)))):
            raise _bad(L.OC_ERR_SHAPE, f"{name} has shape {tuple(size)}, expected {(n_mod, Ch)}")
        if step[-1] != 1:
            raise _bad(L.OC_ERR_INVALID_ARG, f"the channels of {name} must be contiguous")
        row = step[0] if n_mod > 1 else Ch
        if ld is not None and row != ld:
            raise _bad(L.OC_ERR_INVALID_ARG, "gate, scale and shift must have the same row stride")
        ld = row
        at.append(t.data_ptr())
    return L.oc_mod(*at, Ch if ld is None else ld, per, 0)


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
    if h is None:
        h = torch.empty_like(x)
        hp = h.data_ptr()
    else:
        hp = None if h is False else _like(h, full, dt, dev, "h")
    if n is None:
        n = torch.empty_like(x)
        np_ = n.data_ptr()
    else:
        np_ = None if n is False else _like(n, full, dt, dev, "n")
    po, pr, mo = _norm(post, shape, dev, "post"), _norm(pre, shape, dev, "pre"), _mod(mod, rows, shape, dev)
    if rows == 0:      # (empty tensors have no address)
        hp = np_ = xp = yp = None
    _call("oc_norm_gate", dev, _struct(shape), rows, xp, yp, _ref(po), _ref(pr), _ref(mo), res_scale, hp, np_)
    return (x if y is None else None if h is False else h), (None if n is False else n)


GRADS = ("dx", "dy", "gate", "scale", "shift", "post_w", "post_b", "pre_w", "pre_b")


def norm_gate_grad_workspace_bytes(shape: Shape, rows: int, rows_per_mod: int = 0) -> int:
    return L.lib().oc_norm_gate_grad_workspace_bytes(_struct(shape), rows, rows_per_mod)


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
    po, pr, mo = _norm(post, shape, dev, "post"), _norm(pre, shape, dev, "pre"), _mod(mod, rows, shape, dev)
    per, n_mod = 0, 0
    has = [k for k, t in (("gate", mod and mod.gate), ("scale", mod and mod.scale), ("shift", mod and mod.shift),
                          ("post_w", post and post.w), ("post_b", post and post.b), ("pre_w", pre and pre.w),
                          ("pre_b", pre and pre.b)) if t is not None]
    if mo is not None:
        per = mo.rows_per_mod
        n_mod = -(-rows // per)
    out = dict.fromkeys(GRADS)
    if want is not None:
        if not set(want) <= set(GRADS):
            raise _bad(L.OC_ERR_INVALID_ARG, f"unknown gradients {sorted(set(want) - set(GRADS))}")
        has = [k for k in has if k in want]
    at = dict(out)
    # the vectors' gradients: one block for the modulation's, one for the norms'
    for names, size in (([k for k in has if k in GRADS[2:5]], (n_mod, shape.C)),
                        ([k for k in has if k in GRADS[5:]], (shape.C,))):
        if names:
            block = x.new_empty((len(names), *size), dtype=torch.float32)
            base, step = block.data_ptr(), block.stride(0) * 4
            for i, (k, t) in enumerate(zip(names, block.unbind(0))):
                out[k], at[k] = t, base + i * step
    if rows == 0:      # (nothing is written where there are no modulation rows)
        for k in has:
            if k in GRADS[2:5]:
                out[k], at[k] = x.new_zeros((getattr(mod, k).numel() // shape.C, shape.C), dtype=torch.float32), None
    for k, there in (("dx", True), ("dy", y is not None)):
        if there and (want is None or k in want):
            out[k] = torch.empty_like(x)
            at[k] = out[k].data_ptr()
    if ws is None:
        ws = x.new_empty((max(norm_gate_grad_workspace_bytes(shape, rows, per), 256),), dtype=torch.uint8)
    elif _gpu(ws, "ws").device != dev or not ws.is_contiguous():
        raise _bad(L.OC_ERR_INVALID_ARG, f"ws must be contiguous and on {dev}")
    g = L.oc_norm_grads(*(at[k] for k in GRADS[2:]))
    _call("oc_norm_gate_grad", dev, _struct(shape), rows, xp, yp, _ref(po), _ref(pr), _ref(mo), res_scale, dhp, dnp,
          at["dx"], at["dy"], C.byref(g), ws.data_ptr(), ws.nbytes)
    return out


def _heads_of(t: Optional[torch.Tensor], rows: int, heads: Optional[int], shape: Shape, dev, name: str):
    """(address, row stride, heads) of a [rows, heads, head_dim] tensor whose
    rows hold their heads contiguously."""
    if t is None:
        return None, 0, 0
    dt, dh = shape.torch_dtype, shape.head_dim
    if _gpu(t, name).dtype != dt:
        raise _bad(L.OC_ERR_DTYPE, f"{name} has dtype {t.dtype}, expected {dt}")
    if t.device != dev:
        raise _bad(L.OC_ERR_INVALID_ARG, f"{name} is on {t.device}, expected {dev}")
    size = t.shape
    if len(size) != 3 or size[2] != dh or size[0] != rows or (heads is not None and size[1] != heads):
        raise _bad(L.OC_ERR_SHAPE, f"{name} has shape {tuple(size)}, expected "
                                   f"{(rows, 'heads' if heads is None else heads, dh)}")
    step = t.stride()
    if step[2] != 1 or (size[1] > 1 and step[1] != dh):
        raise _bad(L.OC_ERR_INVALID_ARG, f"the heads of a row of {name} must be contiguous")
    return t.data_ptr(), step[0] if rows > 1 else size[1] * dh, size[1]


def _ids(t: Optional[torch.Tensor], shape, dev, name: str) -> Optional[int]:
    return _like(t, shape, torch.int32, dev, name)


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
        q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
        qop, ldqo = q_out.data_ptr(), shape.heads * shape.head_dim
    else:
        qop, ldqo, _ = _heads_of(q_out, rows, shape.heads, shape, dev, "q_out")
    if k_out is None and k is not None:
        k_out = torch.empty_like(k, memory_format=torch.contiguous_format)
        kop, ldko = k_out.data_ptr(), kh * shape.head_dim
    else:
        kop, ldko, _ = _heads_of(k_out, rows, kh, shape, dev, "k_out")
    ip, pp = _ids(kept_idx, (rows,), dev, "kept_idx"), _ids(pos, (rows, 3), dev, "pos")
    if rows == 0:      # (empty tensors have no address)
        qp = kp = qop = kop = None
    _call("oc_rope_qk", dev, _struct(shape), _struct(rope), rows, ip, pp, qp, ldq, kp, ldk, kh, qop, ldqo, kop, ldko,
          1 if inverse else 0)
    return q_out, k_out


_DTYPES = {torch.float32: L.OC_F32, torch.bfloat16: L.OC_BF16}


def _matrix(t, name: str):
    """(address, row stride) of a 2-D tensor with contiguous rows."""
    if _gpu(t, name).dtype not in _DTYPES:
        raise _bad(L.OC_ERR_DTYPE, f"{name} has dtype {t.dtype}, expected bfloat16 or float32")
    if t.dim() != 2:
        raise _bad(L.OC_ERR_SHAPE, f"{name} has shape {tuple(t.shape)}, expected two dimensions")
    size, step = t.shape, t.stride()
    if step[1] != 1 and size[1] > 1:
        raise _bad(L.OC_ERR_INVALID_ARG, f"the rows of {name} must be contiguous")
    return t.data_ptr() or None, step[0] if size[0] > 1 else size[1]


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
    if q is None:
        q = x.new_empty((rows, Kp), dtype=torch.int8)
        qp = q.data_ptr()
    else:
        qp = _like(q, (rows, Kp), torch.int8, dev, "q")
    if scale is None:
        scale = x.new_empty((rows,), dtype=torch.float32)
        sp = scale.data_ptr()
    else:
        sp = _like(scale, (rows,), torch.float32, dev, "scale")
    _call("oc_quant_rows", dev, _DTYPES[x.dtype], at, ld, n, K, ip, rows, qp, sp)
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
        y = q.new_empty((rows, N), dtype=torch.bfloat16 if dtype is None else dtype)
    at, ld = _matrix(y, "y")
    if y.device != dev or y.shape[1] != N or (dtype is not None and y.dtype != dtype):
        raise _bad(L.OC_ERR_SHAPE, f"y is {tuple(y.shape)} {y.dtype} on {y.device}, expected [..., {N}] on {dev}")
    bp = _like(bias, (N,), y.dtype, dev, "bias")
    ip = _ids(out_idx, (rows,), dev, "out_idx")
    _call("oc_linear_i8", dev, _DTYPES[y.dtype], rows, Kp, N, qp, sp, wp, swp, bp, L.ACTS[act], ip, y.shape[0], at, ld)
    return y
