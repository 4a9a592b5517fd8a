"""Gradients of norm_gate where blocks and teams take several items one after
another, and which gradients a call returns.

Without norms and on small whole numbers every gradient is a whole number below
2^24 that fp32 sums hold exactly in any order (h is at most 12, H 10, dy 40, a
sum over 20001 rows of at most 50 each 1000050), so an item that is lost, doubled
or added to another's rows shows whatever its share of a sum."""
import pytest
import torch

import paper_2607_23844_amd as oc
from ops_ref import NormGate
from test_gpu_norm_gate import shape

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32

# rows, C, rows_per_mod: test_ops_plans.py says which teams they take and that these take more than one item
ITEMS = [
    # teams of 16, 32 and 64 lanes that share a block's item
    (19801, 120, 33), (19801, 200, 33), (9901, 320, 33), (9351, 408, 17), (9351, 704, 17), (4591, 1200, 17),
    # the block as the team
    (901, 1160, 1), (2001, 1600, 1), (8193, 1600, 1), (601, 2504, 1), (301, 4200, 1),
    # teams that take a modulation row each
    (20001, 40, 1), (20001, 200, 2), (13001, 320, 3), (13001, 408, 3), (11001, 704, 5), (2201, 1200, 2),
]


def whole(seed, lo, hi, *s):
    return torch.randint(lo, hi + 1, s, generator=torch.Generator().manual_seed(seed)).float()


def problem(rows, C, per, dtype):
    n_mod = -(-rows // per)

    def to(t):
        return t.to(dtype).to(DEV)

    x, y = to(whole(1, -2, 2, rows, C)), to(whole(2, -2, 2, rows, C))
    gate = whole(3, -1, 1, n_mod, C)
    gate[gate == 1] = 2
    mods = to(torch.cat([gate, whole(4, -1, 1, n_mod, C), whole(5, -1, 1, n_mod, C)], 1))
    vec = []
    for i in range(2):
        w = whole(6 + i, 0, 2, C)
        w[w == 0] = -1
        vec += [to(w), to(whole(8 + i, -1, 1, C))]
    kw = dict(y=y, post=oc.Norm("none", 0.0, *vec[:2]), pre=oc.Norm("none", 0.0, *vec[2:]), res_scale=-1.0,
              mod=oc.Mod(mods[:, :C], mods[:, C:2 * C], mods[:, 2 * C:], per))
    ref = NormGate(x, y, ("none", 0.0, *vec[:2]), ("none", 0.0, *vec[2:]), mods[:, :C], mods[:, C:2 * C],
                   mods[:, 2 * C:], per, -1.0)
    return x, kw, ref, to(whole(10, -2, 2, rows, C)), to(whole(11, -2, 2, rows, C))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,C,per", ITEMS)
def test_sums_over_many_items(rows, C, per, dtype):
    x, kw, ref, dh, dn = problem(rows, C, per, dtype)
    want = ref.grads(dh, dn)
    out = oc.norm_gate_grad(x, shape(C, dtype), dn=dn, dh=dh, **kw)
    assert set(want) == {k for k, v in out.items() if v is not None} == set(out)
    for k, v in out.items():
        assert torch.equal(v.cpu().double(), want[k][0].reshape(v.shape)), k
    # the modulation's alone, and the norms' alone
    for want_only in (("gate", "scale", "shift"), ("post_w", "post_b", "pre_w", "pre_b"), ("dx", "shift", "pre_b")):
        part = oc.norm_gate_grad(x, shape(C, dtype), dn=dn, dh=dh, want=want_only, **kw)
        assert {k for k, v in part.items() if v is not None} == set(want_only)
        for k in want_only:
            assert torch.equal(part[k], out[k]), k


@pytest.mark.parametrize("y", [True, False])
@pytest.mark.parametrize("there", [(), ("gate",), ("scale",), ("shift",), ("gate", "scale", "shift"), ("post_w",),
                                   ("post_b",), ("pre_w",), ("pre_b",), ("gate", "post_w", "post_b", "pre_w", "pre_b")])
def test_which_gradients_are_returned(there, y):
    """Those of the inputs that the call has, no more and no fewer."""
    rows, C = 20, 64
    there = [k for k in there if y or k not in ("gate", "post_w", "post_b")]
    g = torch.Generator().manual_seed(1)

    def make(*s):
        return torch.randn(*s, generator=g).to(DEV)

    v = {k: make(5, C) if k in ("gate", "scale", "shift") else make(C) for k in there}
    kw = dict(pre=oc.Norm("layer", 1e-6, v.get("pre_w"), v.get("pre_b")),
              mod=oc.Mod(v.get("gate"), v.get("scale"), v.get("shift"), 4))
    if y:
        kw.update(y=make(rows, C), post=oc.Norm("rms", 1e-6, v.get("post_w"), v.get("post_b")))
    out = oc.norm_gate_grad(make(rows, C), shape(C, F32), dn=make(rows, C), dh=make(rows, C), **kw)
    assert {k for k, t in out.items() if t is not None} == {"dx", *(["dy"] if y else []), *there}
    for k in there:
        assert out[k].shape == v[k].shape and out[k].dtype == F32, k
