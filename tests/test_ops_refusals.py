"""The operators around a sublayer refuse bad arguments on the host, before
anything is enqueued, and the 64-bit formulas of their tests are consistent.
No test here touches a GPU."""
import ctypes as C

import pytest
import torch

import paper_2607_23844_amd as oc
from paper_2607_23844_amd import _lib as L
from ops_ref import NormGate

A = 1 << 30          # addresses that are never read: every call below is refused before a launch
STEP = 1 << 24


def at(i):
    return A + i * STEP


def test_struct_sizes():
    assert C.sizeof(L.oc_norm) == 24 and C.sizeof(L.oc_mod) == 40 and C.sizeof(L.oc_norm_grads) == 56


def norm_call(shape=None, rows=4, x=at(0), y=at(1), post=None, pre=None, mod=None, rs=1.0, h=at(2), n=at(3)):
    sh = (shape or oc.Shape(1, 1, 1, 64, 1, 16, 0, "bf16")).c()
    ref = [None if v is None else C.byref(v) for v in (post, pre, mod)]
    return L.lib().oc_norm_gate(C.byref(sh), rows, x, y, *ref, rs, h, n, None)


def mod(gate=at(4), scale=at(5), shift=at(6), ld=64, per=4, reserved=0):
    return L.oc_mod(gate, scale, shift, ld, per, reserved)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), L.OC_ERR_SHAPE),
    (dict(rows=1 << 30), L.OC_ERR_SHAPE),
    (dict(shape=oc.Shape(1, 1, 1, 60, 1, 16, 0, "bf16")), L.OC_ERR_SHAPE),
    (dict(x=None), L.OC_ERR_INVALID_ARG),
    (dict(x=at(0) + 8), L.OC_ERR_INVALID_ARG),
    (dict(y=at(1) + 2), L.OC_ERR_INVALID_ARG),
    (dict(h=at(2) + 4), L.OC_ERR_INVALID_ARG),
    (dict(n=at(3) + 4), L.OC_ERR_INVALID_ARG),
    (dict(h=None, n=None), L.OC_ERR_INVALID_ARG),
    (dict(y=None), L.OC_ERR_INVALID_ARG),                                       # h without y
    (dict(y=None, h=None, rs=0.5), L.OC_ERR_INVALID_ARG),
    (dict(y=None, h=None, post=L.oc_norm(1, 1e-6, None, None)), L.OC_ERR_INVALID_ARG),
    (dict(y=None, h=None, mod=mod()), L.OC_ERR_INVALID_ARG),                     # a gate without y
    (dict(rs=float("nan")), L.OC_ERR_INVALID_ARG),
    (dict(rs=float("inf")), L.OC_ERR_INVALID_ARG),
    (dict(pre=L.oc_norm(3, 1e-6, None, None)), L.OC_ERR_INVALID_ARG),
    (dict(pre=L.oc_norm(-1, 1e-6, None, None)), L.OC_ERR_INVALID_ARG),
    (dict(pre=L.oc_norm(1, -1e-6, None, None)), L.OC_ERR_INVALID_ARG),
    (dict(pre=L.oc_norm(1, float("nan"), None, None)), L.OC_ERR_INVALID_ARG),
    (dict(post=L.oc_norm(1, float("inf"), None, None)), L.OC_ERR_INVALID_ARG),
    (dict(pre=L.oc_norm(1, 1e-6, at(7) + 8, None)), L.OC_ERR_INVALID_ARG),
    (dict(mod=mod(ld=56)), L.OC_ERR_SHAPE),
    (dict(mod=mod(ld=68)), L.OC_ERR_SHAPE),
    (dict(mod=mod(per=0)), L.OC_ERR_INVALID_ARG),
    (dict(mod=mod(per=-4)), L.OC_ERR_INVALID_ARG),
    (dict(mod=mod(reserved=1)), L.OC_ERR_INVALID_ARG),
    (dict(mod=mod(gate=at(4) + 2)), L.OC_ERR_INVALID_ARG),
    (dict(h=at(0) + 64), L.OC_ERR_INVALID_ARG),                                  # overlaps x without being it
    (dict(n=at(1) - 64), L.OC_ERR_INVALID_ARG),
    (dict(n=at(2)), L.OC_ERR_INVALID_ARG),                                       # h and n the same
    (dict(h=at(5), mod=mod()), L.OC_ERR_INVALID_ARG),
    (dict(n=at(7), pre=L.oc_norm(1, 1e-6, at(7), None)), L.OC_ERR_INVALID_ARG),
])
def test_norm_gate_refuses(kw, status):
    assert norm_call(**kw) == status
    assert L.lib().oc_last_error() != b""


def grad_call(shape=None, rows=4, x=at(0), y=at(1), post=None, pre=None, m=None, dh=at(2), dn=at(3), dx=at(4),
              dy=at(5), grads=None, ws=at(9), ws_bytes=None, rs=1.0):
    sh = (shape or oc.Shape(1, 1, 1, 64, 1, 16, 0, "bf16")).c()
    need = L.lib().oc_norm_gate_grad_workspace_bytes(C.byref(sh), rows, m.rows_per_mod if m else 0)
    ref = [None if v is None else C.byref(v) for v in (post, pre, m)]
    g = None if grads is None else C.byref(grads)
    return L.lib().oc_norm_gate_grad(C.byref(sh), rows, x, y, *ref, rs, dh, dn, dx, dy, g, ws,
                                     need if ws_bytes is None else ws_bytes, None)


def grads(**kw):
    return L.oc_norm_grads(*(kw.get(k) for k, _ in L.oc_norm_grads._fields_))


@pytest.mark.parametrize("kw,status", [
    (dict(dh=None, dn=None), L.OC_ERR_INVALID_ARG),
    (dict(y=None), L.OC_ERR_INVALID_ARG),                                        # dy without y
    (dict(grads=grads(gate=at(6))), L.OC_ERR_INVALID_ARG),                       # no gate
    (dict(grads=grads(pre_w=at(6)), pre=L.oc_norm(1, 1e-6, None, None)), L.OC_ERR_INVALID_ARG),
    (dict(grads=grads(post_b=at(6)), post=L.oc_norm(1, 1e-6, at(7), None)), L.OC_ERR_INVALID_ARG),
    (dict(grads=grads(pre_w=at(6) + 4), pre=L.oc_norm(1, 1e-6, at(7), None)), L.OC_ERR_INVALID_ARG),
    (dict(ws_bytes=1), L.OC_ERR_WORKSPACE),
    (dict(ws=None), L.OC_ERR_INVALID_ARG),
    (dict(ws=at(9) + 16), L.OC_ERR_INVALID_ARG),
    (dict(dx=at(0)), L.OC_ERR_INVALID_ARG),
    (dict(dx=at(2)), L.OC_ERR_INVALID_ARG),
    (dict(dy=at(4)), L.OC_ERR_INVALID_ARG),
    (dict(dy=at(9)), L.OC_ERR_INVALID_ARG),
    (dict(dh=at(2) + 2), L.OC_ERR_INVALID_ARG),
    (dict(grads=grads(pre_w=at(4)), pre=L.oc_norm(1, 1e-6, at(7), None)), L.OC_ERR_INVALID_ARG),
    (dict(grads=grads(pre_w=at(7)), pre=L.oc_norm(1, 1e-6, at(7), None)), L.OC_ERR_INVALID_ARG),
    (dict(rows=-2, ws_bytes=1 << 20), L.OC_ERR_SHAPE),
])
def test_norm_gate_grad_refuses(kw, status):
    assert grad_call(**kw) == status


def test_gradient_workspace_covers_its_parts():
    f = L.lib().oc_norm_gate_grad_workspace_bytes
    sh = oc.Shape(1, 1, 1, 64, 1, 16, 0, "bf16").c()
    assert f(C.byref(sh), 0, 0) == 0 and f(C.byref(sh), -1, 0) == 0 and f(C.byref(sh), 4, -1) == 0
    assert f(C.byref(sh), 1000, 1) >= f(C.byref(sh), 1000, 0) > 0


def test_python_wrappers_refuse_host_tensors():
    sh = oc.Shape(1, 1, 1, 64, 1, 16, 0, "f32")
    with pytest.raises(oc.OmniCacheError):
        oc.norm_gate(torch.zeros(2, 64), sh)
    with pytest.raises(oc.OmniCacheError):
        oc.norm_gate_grad(torch.zeros(2, 64), sh, dn=torch.zeros(2, 64))


@pytest.mark.parametrize("pre,post", [("layer", "rms"), ("rms", "layer"), ("none", "layer"), ("layer", "none")])
def test_norm_formulas_against_differences(pre, post):
    g = torch.Generator().manual_seed(3)

    def r(*s):
        return torch.randn(*s, generator=g, dtype=torch.float64)

    rows, ch, per = 5, 16, 2
    t = dict(x=r(rows, ch), y=r(rows, ch), gate=r(3, ch), scale=r(3, ch), shift=r(3, ch), post_w=r(ch), post_b=r(ch),
             pre_w=r(ch), pre_b=r(ch))
    dh, dn = r(rows, ch), r(rows, ch)

    def make(v):
        return NormGate(v["x"], v["y"], (post, 1e-3, v["post_w"], v["post_b"]), (pre, 1e-3, v["pre_w"], v["pre_b"]),
                        v["gate"], v["scale"], v["shift"], per, 0.6)

    got = make(t).grads(dh, dn)
    for k in t:
        by = r(*t[k].shape) * 1e-5
        val = []
        for s in (1, -1):
            o = make({**t, k: t[k] + s * by})
            val.append(float((o.h * dh + o.n * dn).sum()))
        along = 2 * float((got["d" + k if k in "xy" else k][0].reshape(by.shape) * by).sum())
        assert abs(val[0] - val[1] - along) <= 1e-6 * (abs(along) + 1e-5), k


def rope_call(shape=None, rope=oc.Rope((0, 32, 32)), rows=4, idx=None, pos=None, q=at(0), ld_q=128, k=at(1), ld_k=128,
              kh=2, qo=at(2), ld_qo=128, ko=at(3), ld_ko=128, inverse=0, **fields):
    sh = (shape or oc.Shape(1, 4, 4, 128, 2, 64, 0, "bf16")).c()
    ro = None if rope is None else rope.c()
    for name, v in fields.items():
        setattr(ro, name, v)
    return L.lib().oc_rope_qk(C.byref(sh), None if ro is None else C.byref(ro), rows, idx, pos, q, ld_q, k, ld_k, kh,
                              qo, ld_qo, ko, ld_ko, inverse, None)


@pytest.mark.parametrize("kw,status", [
    (dict(rope=None), L.OC_ERR_INVALID_ARG),
    (dict(rope=oc.Rope((0, 31, 32))), L.OC_ERR_SHAPE),
    (dict(rope=oc.Rope((-2, 32, 32))), L.OC_ERR_SHAPE),
    (dict(rope=oc.Rope((2, 32, 32))), L.OC_ERR_SHAPE),                           # more than the head
    (dict(rope=oc.Rope((1 << 30, 1 << 30, 1 << 30))), L.OC_ERR_SHAPE),
    (dict(rope=oc.Rope((0, 0, 0))), L.OC_ERR_SHAPE),
    (dict(rope=oc.Rope((0, 32, 32), theta=0.0)), L.OC_ERR_INVALID_ARG),
    (dict(rope=oc.Rope((0, 32, 32), theta=-1.0)), L.OC_ERR_INVALID_ARG),
    (dict(rope=oc.Rope((0, 32, 32), theta=float("inf"))), L.OC_ERR_INVALID_ARG),
    (dict(rope=oc.Rope((0, 32, 32), scale=(1.0, float("nan"), 1.0))), L.OC_ERR_INVALID_ARG),
    (dict(rope=oc.Rope((0, 32, 32), scale=(1.0, 1.0, 1e308))), L.OC_ERR_INVALID_ARG),
    (dict(layout=3), L.OC_ERR_INVALID_ARG),
    (dict(shared=2), L.OC_ERR_INVALID_ARG),
    (dict(rows=-1), L.OC_ERR_SHAPE),
    (dict(rows=17), L.OC_ERR_SHAPE),                                             # past the grid
    (dict(rows=1 << 30, idx=at(5)), L.OC_ERR_SHAPE),
    (dict(idx=at(5), pos=at(6)), L.OC_ERR_INVALID_ARG),
    (dict(inverse=2), L.OC_ERR_INVALID_ARG),
    (dict(q=None, qo=None, k=None, ko=None), L.OC_ERR_INVALID_ARG),
    (dict(qo=None), L.OC_ERR_INVALID_ARG),
    (dict(k=None), L.OC_ERR_INVALID_ARG),
    (dict(kh=0), L.OC_ERR_SHAPE),
    (dict(kh=3), L.OC_ERR_SHAPE),                                                # wider than its rows
    (dict(ld_q=120), L.OC_ERR_SHAPE),
    (dict(ld_qo=132), L.OC_ERR_SHAPE),
    (dict(q=at(0) + 2), L.OC_ERR_INVALID_ARG),
    (dict(ko=at(3) + 8), L.OC_ERR_INVALID_ARG),
    (dict(qo=at(0) + 256), L.OC_ERR_INVALID_ARG),                                # the next row of q
    (dict(qo=at(0), ld_qo=136), L.OC_ERR_INVALID_ARG),                           # in place with another stride
    (dict(qo=at(1)), L.OC_ERR_INVALID_ARG),
    (dict(ko=at(0)), L.OC_ERR_INVALID_ARG),
    (dict(qo=at(1), ko=at(0)), L.OC_ERR_INVALID_ARG),
    (dict(ko=at(2)), L.OC_ERR_INVALID_ARG),
    (dict(q=at(0), ld_q=256, qo=at(0), ld_qo=256, k=at(0) + 128, ld_k=256, ko=at(0) + 128, ld_ko=256),
     L.OC_ERR_INVALID_ARG),                                                      # columns that share channels
    (dict(idx=at(2)), L.OC_ERR_INVALID_ARG),
    (dict(shape=oc.Shape(1, 4, 4, 128, 2, 60, 0, "bf16")), L.OC_ERR_SHAPE),
])
def test_rope_refuses(kw, status):
    assert rope_call(**kw) == status


def test_rope_struct_and_layer_calls_refuse():
    assert C.sizeof(L.oc_rope) == 64
    lib = L.lib()
    sh, cf = oc.Shape(1, 8, 8, 32, 2, 16, 0, "bf16").c(), oc.Cfg("token", r=0.5).c()
    bad, good = oc.Rope((0, 16, 16)).c(), oc.Rope((0, 8, 8)).c()
    w, cache = L.oc_attn_weights(at(0), at(1), at(2), at(3)), L.oc_cache(at(5), 0, 0)
    assert lib.oc_layer_cached_rope(C.byref(sh), C.byref(cf), C.byref(bad), at(4), None, C.byref(w), C.byref(cache),
                                    None, None, at(6), 1 << 40, None) == L.OC_ERR_SHAPE
    assert (cache.valid, cache.step) == (0, 0)
    assert lib.oc_attn_full_rope(C.byref(sh), C.byref(cf), C.byref(bad), at(4), None, C.byref(w), at(5), None, at(6),
                                 1 << 40, None) == L.OC_ERR_SHAPE
    assert lib.oc_attn_reduced_rope(C.byref(sh), C.byref(bad), at(7), at(4), 1, 4, None, C.byref(w), at(5), None,
                                    at(6), 1 << 40, None) == L.OC_ERR_SHAPE
    assert lib.oc_attn_reduced_rope(C.byref(sh), C.byref(good), None, at(4), 1, 4, None, C.byref(w), at(5), None,
                                    at(6), 1 << 40, None) == L.OC_ERR_INVALID_ARG
    with pytest.raises(oc.OmniCacheError):
        oc.Rope((32, 32)).c()
    with pytest.raises(oc.OmniCacheError):
        oc.Rope((0, 32, 32), layout="spiral").c()
    with pytest.raises(oc.OmniCacheError):
        oc.rope_qk(None, None, oc.Rope((0, 32, 32)), oc.Shape(1, 4, 4, 128, 2, 64))


def quant_call(dtype=1, x=at(0), ld=64, n_src=8, K=64, idx=None, rows=8, q=at(1), scale=at(2)):
    return L.lib().oc_quant_rows(dtype, x, ld, n_src, K, idx, rows, q, scale, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), L.OC_ERR_DTYPE),
    (dict(K=60, ld=64), L.OC_ERR_SHAPE),
    (dict(K=0), L.OC_ERR_SHAPE),
    (dict(K=131072, ld=131072), L.OC_ERR_SHAPE),
    (dict(ld=56), L.OC_ERR_SHAPE),
    (dict(ld=68), L.OC_ERR_SHAPE),
    (dict(rows=-1), L.OC_ERR_SHAPE),
    (dict(rows=9), L.OC_ERR_SHAPE),                       # more than there are
    (dict(rows=1 << 30, idx=at(4)), L.OC_ERR_SHAPE),
    (dict(n_src=-1, idx=at(4)), L.OC_ERR_SHAPE),
    (dict(x=None), L.OC_ERR_INVALID_ARG),
    (dict(q=None), L.OC_ERR_INVALID_ARG),
    (dict(scale=None), L.OC_ERR_INVALID_ARG),
    (dict(x=at(0) + 8), L.OC_ERR_INVALID_ARG),
    (dict(q=at(1) + 8), L.OC_ERR_INVALID_ARG),
    (dict(scale=at(2) + 2), L.OC_ERR_INVALID_ARG),
    (dict(idx=at(4) + 1), L.OC_ERR_INVALID_ARG),
    (dict(q=at(0)), L.OC_ERR_INVALID_ARG),                # in place
    (dict(scale=at(1) + 64), L.OC_ERR_INVALID_ARG),
    (dict(idx=at(2)), L.OC_ERR_INVALID_ARG),
])
def test_quant_rows_refuses(kw, status):
    assert quant_call(**kw) == status


def linear_call(dtype=1, rows=4, K=64, N=16, q=at(0), sq=at(1), w=at(2), sw=at(3), bias=None, act=0, idx=None,
                n_out=4, y=at(4), ld_y=16):
    return L.lib().oc_linear_i8(dtype, rows, K, N, q, sq, w, sw, bias, act, idx, n_out, y, ld_y, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=-1), L.OC_ERR_DTYPE),
    (dict(rows=-1), L.OC_ERR_SHAPE),
    (dict(rows=5), L.OC_ERR_SHAPE),
    (dict(n_out=-1, idx=at(5)), L.OC_ERR_SHAPE),
    (dict(K=4), L.OC_ERR_SHAPE),
    (dict(K=131064), L.OC_ERR_SHAPE),                     # its rows hold 131072 elements
    (dict(N=12), L.OC_ERR_SHAPE),
    (dict(N=0), L.OC_ERR_SHAPE),
    (dict(ld_y=8), L.OC_ERR_SHAPE),
    (dict(ld_y=20), L.OC_ERR_SHAPE),
    (dict(act=2), L.OC_ERR_INVALID_ARG),
    (dict(q=None), L.OC_ERR_INVALID_ARG),
    (dict(sq=None), L.OC_ERR_INVALID_ARG),
    (dict(w=None), L.OC_ERR_INVALID_ARG),
    (dict(sw=None), L.OC_ERR_INVALID_ARG),
    (dict(y=None), L.OC_ERR_INVALID_ARG),
    (dict(q=at(0) + 8), L.OC_ERR_INVALID_ARG),
    (dict(sw=at(3) + 4), L.OC_ERR_INVALID_ARG),
    (dict(sq=at(1) + 2), L.OC_ERR_INVALID_ARG),
    (dict(bias=at(6) + 2), L.OC_ERR_INVALID_ARG),
    (dict(y=at(4) + 2), L.OC_ERR_INVALID_ARG),
    (dict(y=at(0)), L.OC_ERR_INVALID_ARG),
    (dict(y=at(3)), L.OC_ERR_INVALID_ARG),
    (dict(bias=at(4)), L.OC_ERR_INVALID_ARG),
    (dict(idx=at(4)), L.OC_ERR_INVALID_ARG),
])
def test_linear_i8_refuses(kw, status):
    assert linear_call(**kw) == status


def test_i8_rows_and_empty_calls():
    f = L.lib().oc_i8_row_bytes
    assert [f(k) for k in (-8, 0, 8, 16, 24, 1536)] == [0, 0, 16, 16, 32, 1536]
    assert quant_call(rows=0, q=None, scale=None) == L.OC_OK and linear_call(rows=0, y=None) == L.OC_OK
    with pytest.raises(oc.OmniCacheError):
        oc.quant_rows(torch.zeros(2, 64))
    with pytest.raises(oc.OmniCacheError):
        oc.linear_i8(*(torch.zeros(2, 64, dtype=torch.int8), torch.zeros(2)) * 2)


def test_norm_gradient_plan_covers_its_rows_and_workspace(native):
    r = native("norm_plan")()
    assert r.returncode == 0, r.stdout[:2000]


def test_calls_leave_shapes_as_they_are():
    """Shapes and positions stay plain values: they can be pickled after a call
    that made their C structs, and equal ones share them."""
    import pickle
    from paper_2607_23844_amd import ops
    for v in (oc.Shape(1, 4, 4, 128, 2, 64), oc.Rope((0, 32, 32)), oc.Rope([0, 32, 32])):
        ops._struct(v)
        assert pickle.loads(pickle.dumps(v)) == v
    a, b = oc.Shape(1, 4, 4, 128, 2, 64), oc.Shape(1, 4, 4, 128, 2, 64, dtype="f32")
    assert ops._struct(a)._obj.dtype == L.OC_BF16 and ops._struct(b)._obj.dtype == L.OC_F32
