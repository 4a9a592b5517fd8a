"""Norms fused with gate, modulation and residual, and their gradients,
against the formulas in 64 bits (tests/ops_ref.py)."""
import pytest
import torch

import paper_2607_23844_amd as oc
from ops_ref import NormGate, U32, check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# Roundings of the longest chain, forward: a sum over C <= 16384 channels adds at
# most 64 in a row in a lane and 14 across lanes; twice that for mean and
# deviation, again for the norm before; the rest is a few per element.
FWD = 2 * 2 * 80 + 40
BWD = 2 * FWD      # the same again for the means of the gradients


def make(rows, C, dtype, seed=0, **kw):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, C, generator=g, **kw)).to(dtype).to(DEV)


def shape(C, dtype):
    return oc.Shape(1, 1, 1, C, 1, 16, 0, "bf16" if dtype == torch.bfloat16 else "f32")


def setup(rows, C, dtype, pre="layer", post="none", affine=False, y=True, per=None, gate=True, rs=1.0, eps=1e-6):
    """(call keywords, the formulas)"""
    x, yy = make(rows, C, dtype, 1) * 2, make(rows, C, dtype, 2) if y else None
    vec = []
    for k in range(4):
        vec.append((make(1, C, torch.float32, 10 + k)[0] * 0.2 + (1 - k % 2)).to(dtype) if affine else None)
    po = oc.Norm(post, eps, vec[0], vec[1]) if y else None
    pr = oc.Norm(pre, eps, vec[2], vec[3])
    m = gt = sc = sh = None
    if per is not None:
        n_mod = -(-rows // per)
        wide = make(max(n_mod, 1), 3 * C, dtype, 5)[:n_mod]
        gt = wide[:, :C] if gate and y else None
        sc, sh = wide[:, C:2 * C], wide[:, 2 * C:]
        m = oc.Mod(gt, sc, sh, per)
    kw = dict(y=yy, post=po, pre=pr, mod=m, res_scale=rs if y else 1.0)
    ref = NormGate(x, yy, (post, eps, vec[0], vec[1]) if y else ("none", 0, None, None), (pre, eps, vec[2], vec[3]),
                   gt, sc, sh, per, rs if y else 1.0)
    return x, kw, ref


CASES = [
    # rows, C, dtype, options
    (1, 8, torch.bfloat16, {}),
    (1, 8, torch.float32, dict(pre="rms", per=1)),
    (3, 16, torch.bfloat16, dict(per=3, affine=True, post="layer")),
    (5, 72, torch.float32, dict(per=2, post="rms", affine=True, rs=0.5)),
    (333, 1536, torch.bfloat16, dict(per=333, pre="rms", post="rms", affine=True, rs=0.7071)),
    (1021, 320, torch.float32, dict(per=256, rs=-1.25)),
    (1021, 320, torch.bfloat16, dict(per=100, y=False)),
    (257, 1160, torch.bfloat16, dict(per=1, post="layer")),
    (70, 2056, torch.float32, dict(per=7, post="rms", affine=True)),
    (41, 4104, torch.bfloat16, dict(per=41, post="rms", affine=True)),
    (9, 16384, torch.float32, dict(per=4, post="layer", affine=True)),
    (5, 16392, torch.bfloat16, dict(per=5, post="rms", affine=True)),
    (2500, 64, torch.bfloat16, dict(per=625, gate=False)),
    (130, 136, torch.float32, dict(pre="none", post="none", per=64)),
    (40, 136, torch.bfloat16, dict(pre="none", post="rms")),
    (20000, 40, torch.bfloat16, dict(per=3, affine=True)),
    # many rows: every team of lanes, with modulation rows that share items, fill them and are taken alone
    (1100, 200, torch.float32, dict(per=300, affine=True, post="rms")),
    (1100, 320, torch.bfloat16, dict(per=1100, affine=True, post="layer", rs=0.5)),
    (1501, 320, torch.float32, dict(per=5, affine=True, post="rms")),
    (1100, 408, torch.bfloat16, dict(per=37, post="rms", pre="rms")),
    (1300, 704, torch.float32, dict(per=650, affine=True)),
    (1030, 1000, torch.bfloat16, dict(per=1, affine=True, post="rms")),
    (1030, 1000, torch.float32, dict(per=17, post="layer")),
    (1100, 1536, torch.bfloat16, dict(per=9, affine=True, post="rms")),
    (2100, 1536, torch.float32, dict(per=700, affine=True, post="rms")),
    (1030, 2000, torch.bfloat16, dict(per=515, affine=True, post="layer")),
    (4, 64, torch.float32, dict(per=3, affine=True, post="rms")),
    (600, 8200, torch.bfloat16, dict(per=250, affine=True, post="rms")),
]
IDS = [f"{r}x{c}-{str(t)[6:]}-{i}" for i, (r, c, t, _) in enumerate(CASES)]


@pytest.mark.parametrize("rows,C,dtype,opt", CASES, ids=IDS)
def test_forward(rows, C, dtype, opt):
    x, kw, ref = setup(rows, C, dtype, **opt)
    h, n = oc.norm_gate(x, shape(C, dtype), **kw)
    if kw["y"] is not None:
        check(h, ref.h, ref.h_size, FWD, "h")
    else:
        assert h is x
    check(n, ref.n, ref.n_size, FWD, "n")


@pytest.mark.parametrize("rows,C,dtype,opt", CASES, ids=IDS)
def test_gradients(rows, C, dtype, opt):
    x, kw, ref = setup(rows, C, dtype, **opt)
    dh, dn = make(rows, C, dtype, 7), make(rows, C, dtype, 8)
    out = oc.norm_gate_grad(x, shape(C, dtype), dn=dn, dh=dh, **kw)
    want = ref.grads(dh, dn)
    for k, v in out.items():
        if v is None:
            continue
        # sums over rows: at most `rows` more roundings in a row
        check(v, *(t.reshape(v.shape) for t in want[k]), BWD + (0 if k in ("dx", "dy") else rows), k)
    assert out["dx"] is not None and (out["dy"] is None) == (kw["y"] is None)
    # either of the incoming gradients alone, and a part of the outgoing ones
    for a, b in ((dh, None), (None, dn)):
        only = oc.norm_gate_grad(x, shape(C, dtype), dn=b, dh=a, want=("dx",), **kw)
        w = ref.grads(a, b)["dx"]
        check(only["dx"], *w, BWD, "dx alone")
        assert [k for k, v in only.items() if v is not None] == ["dx"]


def test_gradients_against_differences():
    """Central differences of the kernel against those of the formulas at the
    same step (their truncation is the same), and these against the gradient."""
    rows, C, step = 6, 72, 2.0 ** -6
    opt = dict(per=2, post="rms", pre="layer", affine=True, rs=0.5, eps=1e-3)
    x, kw, ref = setup(rows, C, torch.float32, **opt)
    sh = shape(C, torch.float32)
    dh, dn = make(rows, C, torch.float32, 7), make(rows, C, torch.float32, 8)
    got = oc.norm_gate_grad(x, sh, dn=dn, dh=dh, **kw)
    vec = kw["post"], kw["pre"], kw["mod"]

    def at(leaf, by):
        """kernel's and formulas' (sum of outputs times dh, dn), and the kernel's rounding bound"""
        p, q, m = oc.Norm(**vars(vec[0])), oc.Norm(**vars(vec[1])), oc.Mod(**vars(vec[2]))
        xx, yy = x, kw["y"]
        if leaf == "dx":
            xx = x + by
        elif leaf == "dy":
            yy = yy + by
        elif leaf in ("gate", "scale", "shift"):
            for k in ("gate", "scale", "shift"):
                v = getattr(m, k)
                setattr(m, k, (v + by if k == leaf else v).contiguous())
        else:
            o, k = (p if leaf[:4] == "post" else q), leaf[-1]
            setattr(o, k, getattr(o, k) + by)
        h, n = oc.norm_gate(xx, sh, y=yy, post=p, pre=q, mod=m, res_scale=0.5)
        r = NormGate(xx, yy, (p.kind, p.eps, p.w, p.b), (q.kind, q.eps, q.w, q.b), m.gate, m.scale, m.shift, 2, 0.5)
        cd, cn = dh.cpu().double(), dn.cpu().double()
        f = float((h.cpu().double() * cd + n.cpu().double() * cn).sum())
        e = float((r.h * cd + r.n * cn).sum())
        tol = float(((r.h.abs() + FWD * r.h_size) * cd.abs() + (r.n.abs() + FWD * r.n_size) * cn.abs()).sum()) * U32
        return f, e, tol

    for leaf, grad in got.items():
        by = make(*grad.reshape(-1, C).shape, torch.float32, 30).reshape(grad.shape) * step
        (f1, e1, t1), (f0, e0, t0) = at(leaf, by), at(leaf, -by)
        assert abs((f1 - f0) - (e1 - e0)) <= t1 + t0, leaf
        along = 2 * float((grad.cpu().double() * by.cpu().double()).sum())
        fine = [at(leaf, by / 64)[1] - at(leaf, -by / 64)[1]][0] * 64     # (by / 64: 4096 times less truncation)
        size = ref.grads(dh, dn)[leaf][1].reshape(grad.shape)
        tol = 2 * float((size * by.cpu().double().abs()).sum()) * (BWD + rows) * U32
        # by / 64 is added to fp32 inputs: half a step of values up to 8 each, as far as the difference goes
        moved = 2 * 64 * float(size.sum()) * 8 * U32
        assert abs(along - fine) <= tol + moved + abs(fine) * 2e-3, leaf


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_in_place(dtype):
    x, kw, _ = setup(50, 328, dtype, per=25, post="rms", affine=True)
    sh = shape(328, dtype)
    h, n = oc.norm_gate(x, sh, **kw)
    x2, y2 = x.clone(), kw["y"].clone()
    kw["y"] = y2
    h2, n2 = oc.norm_gate(x2, sh, h=x2, n=y2, **kw)
    assert h2 is x2 and n2 is y2 and torch.equal(h, h2) and torch.equal(n, n2)


def test_parts_of_the_result():
    x, kw, _ = setup(50, 328, torch.bfloat16, per=50, post="rms", affine=True)
    sh = shape(328, torch.bfloat16)
    h, n = oc.norm_gate(x, sh, **kw)
    assert torch.equal(oc.norm_gate(x, sh, n=False, **kw)[0], h)
    assert torch.equal(oc.norm_gate(x, sh, h=False, **kw)[1], n)
    # any leading dimensions
    kw["y"] = kw["y"].view(5, 10, 328)
    h3, n3 = oc.norm_gate(x.view(5, 10, 328), sh, **kw)
    assert h3.shape == (5, 10, 328) and torch.equal(h3.view(50, 328), h) and torch.equal(n3.view(50, 328), n)


@pytest.mark.parametrize("C", [328, 2048, 4104])
def test_not_finite_rows_stay_in_their_row(C):
    x, kw, _ = setup(70, C, torch.bfloat16, per=70, post="layer")
    sh = shape(C, torch.bfloat16)
    h, n = oc.norm_gate(x, sh, **kw)
    x[3, 5], x[40, 1], kw["y"][66, C - 1] = float("nan"), float("inf"), float("-inf")
    h2, n2 = oc.norm_gate(x, sh, **kw)
    ok = torch.ones(70, dtype=torch.bool)
    ok[[3, 40, 66]] = False
    assert torch.equal(h[ok], h2[ok]) and torch.equal(n[ok], n2[ok])
    assert n2[[3, 40, 66]].isnan().all() and h2[66].isnan().all()
    assert h2[3, 5].isnan() and h2[40, 1].isinf() and h2[3].isnan().sum() == 1


def test_zero_rows_and_zero_deviation():
    sh = shape(64, torch.float32)
    x = torch.zeros(0, 64, device=DEV)
    w = torch.ones(64, device=DEV)
    h, n = oc.norm_gate(x, sh, y=x, pre=oc.Norm("rms", 1e-6, w))
    assert h.shape == n.shape == (0, 64)
    # sums over no rows are zero
    out = oc.norm_gate_grad(x, sh, dn=x, y=x, pre=oc.Norm("rms", 1e-6, w), post=oc.Norm("layer", 1e-6, w, w))
    assert out["dx"].shape == (0, 64) and all((out[k] == 0).all() for k in ("pre_w", "post_w", "post_b"))
    # a row without deviation: eps keeps it finite
    c = torch.full((2, 64), 3.0, device=DEV)
    assert torch.equal(oc.norm_gate(c, sh, pre=oc.Norm("layer", 1e-6))[1], torch.zeros_like(c))


def test_largest_finite_bf16_and_small_values():
    """Rounding up to an infinity only where the value rounds to it."""
    sh = shape(64, torch.bfloat16)
    x = torch.full((2, 64), 3.0e38, device=DEV).bfloat16()
    h, _ = oc.norm_gate(x, sh, y=x, n=False, res_scale=0.0)
    assert torch.equal(h, x)
    h, _ = oc.norm_gate(x, sh, y=x, n=False)
    assert h.isinf().all()


def test_same_results_every_time_and_on_another_stream():
    x, kw, _ = setup(3001, 320, torch.bfloat16, per=700, post="rms", affine=True)
    sh = shape(320, torch.bfloat16)
    dh, dn = make(3001, 320, torch.bfloat16, 7), make(3001, 320, torch.bfloat16, 8)
    first = oc.norm_gate(x, sh, **kw), oc.norm_gate_grad(x, sh, dn=dn, dh=dh, **kw)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        again = oc.norm_gate(x, sh, **kw), oc.norm_gate_grad(x, sh, dn=dn, dh=dh, **kw)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first[0], again[0]))
    assert all(torch.equal(first[1][k], again[1][k]) for k in first[1])


def test_captured_and_replayed():
    x, kw, _ = setup(777, 320, torch.bfloat16, per=111, post="rms", affine=True)
    sh = shape(320, torch.bfloat16)
    dh, dn = make(777, 320, torch.bfloat16, 7), make(777, 320, torch.bfloat16, 8)
    ws = torch.empty(oc.norm_gate_grad_workspace_bytes(sh, 777, 111), dtype=torch.uint8, device=DEV)

    def call():
        return [*oc.norm_gate(x, sh, **kw), *oc.norm_gate_grad(x, sh, dn=dn, dh=dh, ws=ws, **kw).values()]

    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = call()
    for i in range(4):
        x.copy_(make(777, 320, torch.bfloat16, 40 + i))
        g.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in out]
        eager = call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, eager)), i
