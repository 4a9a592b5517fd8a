"""Rotary layers at the ends of fp16: projected pairs inside its range whose
rotation leaves it are saturated like any q and k, on every way that the layers
take (short sequences, the projection's tiles, a pass of its own)."""
import math

import numpy as np
import pytest
import torch

import paper_2607_23844_amd as oc
from ops_ref import grid_pos
from parity import TOL, rel_err, to_f64
from test_gpu_rope import attention

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
GRID = dict(F=3, H=6, W=10)
BIG = 60000.0          # (60000, 60000) turned by an eighth of a turn is (0, 84853)


def first_pair(rp):
    """The channels of the first pair of the first axis that has any (its frequency is 1)."""
    start = 0
    for n in rp.dims:
        if n:
            return {"pairs": (start, start + 1), "halves": (start, start + n // 2),
                    "split": (start // 2, start // 2 + sum(rp.dims) // 2)}[rp.layout]
        start += n


def large_pairs(rp, L, n_seq, heads, dh, C=128):
    """Head 0 has k = (BIG, BIG) in the first pair where its q is 0, the last head
    q = (BIG, BIG) after its scaling where k is 0: the formula's scores do not
    hold these channels, an infinity among them would be one times 0."""
    sh = oc.Shape(**GRID, C=C, heads=heads, head_dim=dh)
    hd, n = heads * dh, sh.F * sh.N
    g = torch.Generator().manual_seed(L + dh)
    W64 = {k: torch.randn(hd, C, generator=g, dtype=torch.float64) / C ** 0.5 for k in ("wq", "wk", "wv")}
    W64["wo"] = torch.randn(C, hd, generator=g, dtype=torch.float64) / hd ** 0.5
    x = torch.randn(n_seq * L, C, generator=g)
    x[:, 0] = 1.0
    a, b = first_pair(rp)
    last = (heads - 1) * dh
    for c in (a, b):
        for k in ("wq", "wk"):
            W64[k][c] = 0
            W64[k][last + c] = 0
        W64["wk"][c, 0] = BIG
        W64["wq"][last + c, 0] = BIG * dh ** 0.5 / math.log2(math.e)
    W = {k: v.bfloat16().to(DEV) for k, v in W64.items()}
    W64 = {k: v.cpu().double().numpy() for k, v in W.items()}
    x = x.bfloat16()
    idx = torch.randint(0, n, (n_seq * L,), generator=g, dtype=torch.int32)
    pos = grid_pos(idx, sh.H, sh.W)
    # some rows do leave the range: angle = position at frequency 1
    ang = pos[:, next(i for i, d in enumerate(rp.dims) if d)]
    assert (BIG * 1.05 * (ang.cos().abs() + ang.sin().abs()) > 70000).any()
    y, _ = oc.attn_reduced(x.to(DEV), n_seq, L, W, sh, rope=rp, kept_idx=idx.to(DEV))
    ref = np.concatenate([attention(x[i:i + L].double().numpy(), None, pos[i:i + L], W64, heads, dh, rp)
                          for i in range(0, n_seq * L, L)])
    y = to_f64(y).reshape(ref.shape)
    assert np.isfinite(y).all()
    assert rel_err(y, ref, "bf16") <= TOL["bf16"]


ROPES = [oc.Rope((16, 24, 24)), oc.Rope((16, 24, 24), layout="halves"), oc.Rope((14, 10, 22), layout="halves"),
         oc.Rope((0, 32, 32), layout="split")]


@pytest.mark.parametrize("rp", ROPES)
@pytest.mark.parametrize("L,n_seq", [(25, 11), (64, 3)])
def test_short_sequences(rp, L, n_seq):
    large_pairs(rp, L, n_seq, 3, 64)


@pytest.mark.parametrize("rp", ROPES)
@pytest.mark.parametrize("heads", [2, 24])
def test_projection_tiles_of_heads_of_64(rp, heads):
    large_pairs(rp, 300, 1, heads, 64)


@pytest.mark.parametrize("heads,dh,rp", [
    (5, 72, oc.Rope((24, 24, 24))), (5, 72, oc.Rope((24, 24, 24), layout="halves")),
    (3, 96, oc.Rope((32, 32, 32), layout="halves")), (7, 80, oc.Rope((14, 10, 22), layout="halves")),
    (3, 128, oc.Rope((32, 48, 48), layout="halves")), (4, 128, oc.Rope((44, 42, 42), layout="halves")),
])
def test_other_heads(heads, dh, rp):
    large_pairs(rp, 90, 3, heads, dh)
