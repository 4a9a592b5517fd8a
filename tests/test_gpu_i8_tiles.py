"""The product of quantised rows on every tile shape that it can pick: rows and
outputs that end inside a tile, K that ends inside a step, both types, each
epilogue, rows to positions."""
import pytest
import torch

import paper_2607_23844_amd as oc
from ops_ref import U32, half_step
from test_gpu_i8 import N_ROUND, make, rnd8

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32

# rows, K, N by tile shape (test_ops_plans.py asserts that each is picked)
TILES = {
    0: [(2747, 72, 4464), (14315, 152, 776), (10837, 520, 1080)],
    1: [(2575, 272, 3856), (13359, 648, 536)],
    2: [(1167, 288, 5096), (8471, 520, 656)],
    3: [(17851, 4312, 840)],
    4: [(629, 656, 3448), (16625, 728, 72)],
    5: [(16789, 16, 168), (12349, 520, 208)],
    6: [(17401, 8, 488), (16781, 560, 168)],
    7: [(16525, 16, 136), (16859, 624, 136)],
    8: [(33, 144, 8), (333, 1544, 1048)],
    9: [(12497, 8, 200), (8429, 616, 72)],
}


def formula(q, s, w, ws, bias, gelu):
    """(value, size) in 64 bits, as ops_ref.linear_i8, on the GPU (the products'
    sums are whole numbers below 2^53)."""
    v = (q.double() @ w.double().t()) * s.double()[:, None] * ws.double()
    size = v.abs()
    if bias is not None:
        v, size = v + bias.double(), size + bias.double().abs()
    if gelu:
        size = 1.13 * size + v.abs() * 50.0
        v = 0.5 * v * (1.0 + torch.tanh((2.0 / torch.pi) ** 0.5 * (v + 0.044715 * v ** 3)))
    return v, size


def hold(got, ref, size, what):
    tol = half_step(got.dtype) * ref.abs() * 1.01 + N_ROUND * U32 * size + 1e-40
    bad = ~((got.double() - ref).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), ref[bad][:4].tolist())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tile,rows,K,N", [(t, *s) for t, sizes in TILES.items() for s in sizes])
def test_tile(tile, rows, K, N, dtype):
    Kp = (K + 15) // 16 * 16
    q, w = rnd8(1, rows, Kp), rnd8(2, N, Kp)
    q[:, K:], w[:, K:] = 0, 0
    # (outputs of a few units, where GELU bends)
    s, ws = make(3, rows).abs() * 0.02 / K ** 0.5, make(4, N).abs() * 0.02
    bias = make(5, N, dtype=dtype)
    for b, act in ((None, "none"), (bias, "none"), (bias, "gelu"), (None, "gelu")):
        ref = formula(q, s, w, ws, b, act == "gelu")
        y = oc.linear_i8(q, s, w, ws, bias=b, act=act, dtype=dtype)
        hold(y, *ref, (act, b is not None))
    # to positions in a wider buffer; every seventh row to none
    total = rows + 40
    idx = torch.randperm(total, generator=torch.Generator().manual_seed(6))[:rows].int()
    idx[::7] = -1
    idx[3::7] = total
    wide = torch.full((total, N + 16), 3.0, dtype=dtype, device=DEV)
    out = oc.linear_i8(q, s, w, ws, bias=bias, act="gelu", out_idx=idx.to(DEV), y=wide[:, 8:8 + N])
    ok = (idx >= 0) & (idx < total)
    y = oc.linear_i8(q, s, w, ws, bias=bias, act="gelu", dtype=dtype)
    at = idx[ok].long().to(DEV)
    assert torch.equal(out[at], y[ok.to(DEV)])
    wide[at, 8:8 + N] = 3
    assert (wide == 3).all()
