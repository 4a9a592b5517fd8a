"""Gradients of norm_gate where a row is not finite and the formulas do not let
that through."""
import pytest
import torch

import paper_2607_23844_amd as oc
from ops_ref import NormGate, check
from test_gpu_norm_gate import BWD, make, setup, shape

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
SIZES = [(70, 328), (1100, 200), (1200, 408), (1100, 704), (1100, 1000), (1100, 1536), (40, 2056), (40, 4104), (20, 8200)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("per", [1, 5, 600])
@pytest.mark.parametrize("rows,C", SIZES)
def test_no_norm_and_infinite_values(rows, C, per, dtype):
    """Without norms n = (h w + b)(1 + s) + t, whose derivative by h does not
    hold h: an infinite x leaves every gradient finite but those of the vectors
    that multiply h, in its channel."""
    x, kw, ref = setup(rows, C, dtype, pre="none", post="none", affine=True, per=per, rs=0.5)
    dh, dn = make(rows, C, dtype, 7), make(rows, C, dtype, 8)
    want = ref.grads(dh, dn)
    x[3, 5], x[rows - 1, C - 1] = float("inf"), float("-inf")
    out = oc.norm_gate_grad(x, shape(C, dtype), dn=dn, dh=dh, **kw)
    for k, v in out.items():
        val, size = (t.reshape(v.shape) for t in want[k])
        ok = torch.ones(v.shape, dtype=torch.bool)
        if k in ("scale", "pre_w"):                      # sum dn a and sum da u, a and u of h
            ok[..., [5, C - 1]] = False
        got = torch.where(ok, v.cpu(), val.to(v.dtype))
        check(got, val, size, BWD + (0 if k in ("dx", "dy") else rows), k)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,C", [(40, 4104), (20, 8200), (70, 328)])
def test_no_norm_after_and_infinite_sublayer_output(rows, C, dtype):
    """post = none: dy = g w H does not hold y (dn NULL, so H is dh)."""
    x, kw, ref = setup(rows, C, dtype, pre="none", post="none", affine=True, per=7, rs=0.5)
    dh = make(rows, C, dtype, 7)
    want = ref.grads(dh)
    kw["y"][3, 5] = float("inf")
    out = oc.norm_gate_grad(x, shape(C, dtype), dh=dh, want=("dx", "dy"), **kw)
    for k in ("dx", "dy"):
        check(out[k], *want[k], BWD, k)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("per", [1, 5, 600])
@pytest.mark.parametrize("rows,C", SIZES)
def test_rows_that_are_not_finite_where_n_has_no_gradient(rows, C, per, dtype):
    """dn NULL: n takes no part, whatever the rows hold.  dx = rs dh, dy and the
    vectors of the norm after follow from H = dh, those of n are zero."""
    x, kw, ref = setup(rows, C, dtype, pre="layer", post="rms", affine=True, per=per, rs=0.5)
    dh = make(rows, C, dtype, 7)
    want = ref.grads(dh)
    x[3, 5], x[rows - 1, C - 1], x[rows // 2] = float("inf"), float("nan"), float("nan")
    out = oc.norm_gate_grad(x, shape(C, dtype), dh=dh, **kw)
    for k in ("scale", "shift", "pre_w", "pre_b"):
        assert (out[k] == 0).all(), k
    for k in ("dx", "dy", "gate", "post_w", "post_b"):
        check(out[k], *(t.reshape(out[k].shape) for t in want[k]), BWD + (0 if k in ("dx", "dy") else rows), k)
