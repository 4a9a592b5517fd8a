"""A workspace that overlaps what the call reads is refused on the host."""
import pytest

import paper_2607_23844_amd as oc
from paper_2607_23844_amd import _lib as L
from test_ops_refusals import at, grad_call, grads, mod

WS = at(9)


@pytest.mark.parametrize("kw", [
    dict(x=WS), dict(y=WS + 256), dict(dh=WS), dict(dn=WS + 256),
    dict(m=mod(WS, None, None)), dict(m=mod(None, WS + 256, None)), dict(m=mod(None, None, WS)),
    dict(post=L.oc_norm(1, 1e-6, WS, None)), dict(pre=L.oc_norm(1, 1e-6, None, WS + 256)),
])
def test_norm_gate_grad_refuses(kw):
    call = dict(rows=400, shape=oc.Shape(1, 1, 1, 64, 1, 16, 0, "f32"), grads=grads())
    assert grad_call(**{**call, **kw}) == L.OC_ERR_INVALID_ARG
    assert b"workspace" in L.lib().oc_last_error()
