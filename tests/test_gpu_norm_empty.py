"""norm_gate of no rows, with every form that the vectors of all rows may have."""
import pytest
import torch

import paper_2607_23844_amd as oc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
C = 64


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("size,grad", [((1, C), (1, C)), ((C,), (1, C)), ((0, C), (0, C))])
def test_vectors_of_all_rows(size, grad, dtype):
    sh = oc.Shape(1, 1, 1, C, 1, 16, 0, "bf16" if dtype == torch.bfloat16 else "f32")
    x = torch.empty(0, C, dtype=dtype, device=DEV)
    v = torch.ones(size, dtype=dtype, device=DEV)
    w = torch.ones(C, dtype=dtype, device=DEV)
    kw = dict(y=x, pre=oc.Norm("layer", 1e-6, w), mod=oc.Mod(v, v, v))
    h, n = oc.norm_gate(x, sh, **kw)
    assert h.shape == n.shape == (0, C)
    out = oc.norm_gate_grad(x, sh, dn=x, dh=x, **kw)
    assert out["dx"].shape == out["dy"].shape == (0, C)
    assert (out["pre_w"] == 0).all()
    for k in ("gate", "scale", "shift"):
        assert out[k].shape == grad and out[k].dtype == torch.float32 and (out[k] == 0).all(), k


def test_vectors_of_given_rows():
    """rows_per_mod given: no rows have no modulation rows, as include/oc.h counts them."""
    sh = oc.Shape(1, 1, 1, C, 1, 16, 0, "f32")
    x = torch.empty(0, C, device=DEV)
    v = torch.ones(0, C, device=DEV)
    assert oc.norm_gate(x, sh, pre=oc.Norm(), mod=oc.Mod(None, v, v, 4))[1].shape == (0, C)
    with pytest.raises(oc.OmniCacheError):
        oc.norm_gate(x, sh, pre=oc.Norm(), mod=oc.Mod(None, torch.ones(1, C, device=DEV), None, 4))
