"""The operators around a sublayer on tensors of more than 2^31 elements: rows
at both ends and around the border against the same rows by themselves."""
import pytest
import torch

import paper_2607_23844_amd as oc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


@pytest.fixture(autouse=True)
def freed():
    yield
    torch.cuda.empty_cache()


def fill(*s):
    return torch.empty(*s, dtype=BF, device=DEV).normal_(generator=torch.Generator(device=DEV).manual_seed(5))


def ends(rows, width):
    at = (1 << 31) // width
    return sorted({0, 1, at - 1, at, at + 1, rows - 2, rows - 1})


def test_norms_and_their_gradients():
    rows, C = 1100001, 2048
    sh = oc.Shape(1, 1, 1, C, 1, 16)
    x, y = fill(rows, C), fill(rows, C)
    kw = dict(post=oc.Norm("rms"), pre=oc.Norm("layer"), res_scale=0.5)
    h, n = oc.norm_gate(x, sh, y=y, **kw)
    g = oc.norm_gate_grad(x, sh, dn=h, y=y, want=("dx", "dy"), **kw)
    for r in ends(rows, C):
        h1, n1 = oc.norm_gate(x[r:r + 1], sh, y=y[r:r + 1], **kw)
        # one row takes another team of threads: sums in another order, a step of bf16 at most
        assert ((h[r] - h1[0]).abs() <= 2.0 ** -7 * h1[0].abs()).all(), r
        assert ((n[r] - n1[0]).abs() <= 2.0 ** -7 * n1[0].abs() + 1e-4).all(), r
        g1 = oc.norm_gate_grad(x[r:r + 1], sh, dn=h[r:r + 1], y=y[r:r + 1], want=("dx", "dy"), **kw)
        for k in ("dx", "dy"):
            assert ((g[k][r] - g1[k][0]).abs() <= 2.0 ** -7 * g1[k][0].abs() + 1e-4).all(), (k, r)


@pytest.mark.parametrize("rp", [oc.Rope((48, 40, 40)), oc.Rope((44, 42, 42), layout="halves")])
def test_rotation(rp):
    rows, heads, dh = 530001, 32, 128
    sh = oc.Shape(3, 30, 40, heads * dh, heads, dh)
    q = fill(rows, heads, dh)
    pos = torch.randint(0, 1 << 20, (rows, 3), generator=torch.Generator(device=DEV).manual_seed(6), device=DEV,
                        dtype=torch.int32)
    out, _ = oc.rope_qk(q, None, rp, sh, pos=pos)
    for r in ends(rows, heads * dh):
        assert torch.equal(out[r], oc.rope_qk(q[r:r + 1], None, rp, sh, pos=pos[r:r + 1])[0][0]), r


def test_quantised_rows_and_product():
    rows, K, N = 600001, 64, 4096
    x = fill(rows, 4096)
    q, s = oc.quant_rows(x)
    for r in ends(rows, 4096):
        q1, s1 = oc.quant_rows(x[r:r + 1])
        assert torch.equal(q[r], q1[0]) and torch.equal(s[r], s1[0]), r
    q, s = q[:, :K].contiguous(), s
    w, ws = oc.quant_rows(fill(N, K))
    out = x                                          # [rows, N], written from the end
    idx = torch.arange(rows - 1, -1, -1, dtype=torch.int32, device=DEV)
    oc.linear_i8(q, s, w, ws, out_idx=idx, y=out)
    for r in ends(rows, N):
        want = oc.linear_i8(q[rows - 1 - r:rows - r], s[rows - 1 - r:rows - r], w, ws)
        assert torch.equal(out[r], want[0]), r
