"""Rows quantised to 8 bits and the product of quantised matrices."""
import pytest
import torch

import paper_2607_23844_amd as oc
from ops_ref import check, d, linear_i8, quant

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# The sum's conversion, two scales, the bias: 4 roundings; GELU: its cube, sum and
# factor 4, exponential, sum, quotient and product 5.
N_ROUND = 4 + 9
BF, F32 = torch.bfloat16, torch.float32


def make(seed, *s, dtype=F32):
    return torch.randn(*s, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


def rnd8(seed, *s):
    return torch.randint(-127, 128, s, generator=torch.Generator().manual_seed(seed), dtype=torch.int8).to(DEV)


def ids(n, total, seed=3):
    return torch.randperm(total, generator=torch.Generator().manual_seed(seed))[:n].int().to(DEV)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,K", [(1, 8), (3, 24), (333, 1536), (77, 320), (500, 64), (9, 4104), (5, 6144), (2, 40000),
                                    (2000, 200)])
def test_quantised_rows(rows, K, dtype):
    x = make(1, rows, K, dtype=dtype)
    x[:, 3::97] *= 20
    q, s = oc.quant_rows(x)
    rq, rs = quant(x)
    assert q.shape == (rows, (K + 15) // 16 * 16) and q.dtype == torch.int8
    assert torch.equal(d(q)[:, :K], rq) and not q[:, K:].any()
    assert torch.equal(s.cpu(), rs)
    # retained rows, also twice and in any order, of a wider buffer
    wide = make(2, rows, K + 16, dtype=dtype)
    idx = torch.cat([ids(rows, rows), ids(rows, rows, 4)[:7]])
    q2, s2 = oc.quant_rows(wide[:, 8:8 + K], row_idx=idx)
    rq, rs = quant(wide[:, 8:8 + K][idx.long()])
    assert torch.equal(d(q2)[:, :K], rq) and torch.equal(s2.cpu(), rs)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_ties_go_to_the_even_number(dtype):
    """max|x| = 127 c makes every x = (n + 1/2) c a tie; max|x| = m makes m / 2
    one (63.5)."""
    n = torch.arange(-126, 127).double()
    x = torch.zeros(6, 256, dtype=torch.float64)
    x[:3, 0], x[:3, 1:254] = 127.0, n + 0.5
    x[1] *= 2.0 ** -100
    x[2] *= 2.0 ** 110
    for r, m in ((3, 1.0), (4, 1.0 + 2 ** -7), (5, 1.9921875)):
        x[r, 0], x[r, 1], x[r, 2] = m, m / 2, -m / 2
    x = x.to(dtype).to(DEV)
    rq, rs = quant(x)
    assert (rq[0, 1:254] % 2 == 0).all() and (rq[3:, 1] == 64).all()      # (64 is the even one)
    q, s = oc.quant_rows(x)
    assert torch.equal(d(q), rq) and torch.equal(s.cpu(), rs)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_all_quotients(dtype):
    """Every bf16 fraction of many maxima, from the smallest subnormal numbers
    to the largest."""
    vals = torch.arange(1, 0x7F80, dtype=torch.int32).to(torch.int16).view(BF)    # every positive value
    rows = []
    for i in range(0, len(vals), 331):
        top = vals[i]
        lo = max(0, i - 8 * 128 - 256)
        r = vals[lo:i + 1].double()
        r = torch.cat([r, torch.zeros(1408 - len(r), dtype=torch.float64)])
        rows.append(r * torch.where(torch.arange(len(r)) % 2 == 0, 1.0, -1.0))
        assert r.max() == top.double()
    x = torch.stack(rows).to(dtype).to(DEV)
    q, s = oc.quant_rows(x)
    rq, rs = quant(x)
    assert torch.equal(d(q), rq) and torch.equal(s.cpu(), rs)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("K", [64, 2056])
def test_rows_of_zeros_and_not_finite_rows(dtype, K):
    x = make(1, 6, K, dtype=dtype)
    x[1] = 0
    x[2, K - 1], x[3, 0], x[4, 5] = float("nan"), float("inf"), float("-inf")
    q, s = oc.quant_rows(x)
    assert not q[1:5].any() and s[1] == 0 and s[2:5].isnan().all()
    w, ws = oc.quant_rows(make(2, 16, K, dtype=dtype))
    y = oc.linear_i8(q, s, w, ws, dtype=F32)
    assert (y[1] == 0).all() and y[2:5].isnan().all() and y[[0, 5]].isfinite().all()


def test_rows_outside_are_left_as_they_were():
    x = make(1, 10, 64)
    idx = torch.tensor([3, -1, 10, 9, 1 << 30, -(1 << 31)], dtype=torch.int32, device=DEV)
    q, s = torch.full((6, 64), 5, dtype=torch.int8, device=DEV), torch.full((6,), 7.0, device=DEV)
    oc.quant_rows(x, row_idx=idx, q=q, scale=s)
    rq, rs = quant(x[[3, 9]])
    assert torch.equal(d(q)[[0, 3]], rq) and torch.equal(s[[0, 3]].cpu(), rs)
    assert (q[[1, 2, 4, 5]] == 5).all() and (s[[1, 2, 4, 5]] == 7).all()


SIZES = [(1, 16, 8), (1, 1536, 1536), (2, 72, 40), (7, 320, 1280), (13, 1024, 512), (16, 2048, 72), (17, 4096, 136),
         (33, 6144, 64), (40, 128, 4096), (64, 1152, 1152), (100, 264, 328), (333, 1536, 1536), (1021, 200, 1000),
         (2500, 64, 72), (130, 40000, 24), (600, 512, 2048)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,K,N", SIZES)
def test_product(rows, K, N, dtype):
    Kp = (K + 15) // 16 * 16
    q, w = rnd8(1, rows, Kp), rnd8(2, N, Kp)
    q[:, K:], w[:, K:] = 0, 0
    s, ws = make(3, rows).abs() * 0.01, make(4, N).abs() * 0.01
    bias = make(5, N, dtype=dtype)
    for act, b in (("none", None), ("gelu", bias)):
        y = oc.linear_i8(q, s, w, ws, bias=b, act=act, dtype=dtype)
        assert y.dtype == dtype and y.shape == (rows, N)
        check(y, *linear_i8(q, s, w, ws, b, act), N_ROUND, act)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,K,N", [(1, 1024, 8), (16, 1032, 2048), (5, 1016, 2048), (5, 2048, 2056), (20, 320, 1000),
                                      (32, 1536, 2056), (32, 6144, 1544), (17, 1024, 24), (32, 72, 4096), (17, 200, 4104)])
def test_product_of_few_rows(rows, K, N, dtype):
    test_product(rows, K, N, dtype)


@pytest.mark.parametrize("rows", [1, 16, 200])
def test_sums_are_exact_integers(rows):
    """The largest sums that fit (-128 too), and sums that fp32 would not hold."""
    K = 131056
    q, w = torch.full((rows, K), -128, dtype=torch.int8, device=DEV), torch.full((24, K), -128, dtype=torch.int8, device=DEV)
    w[1] = 127
    w[2, ::2] = 127
    one, ones = torch.ones(rows, device=DEV), torch.ones(24, device=DEV)
    y = oc.linear_i8(q, one, w, ones, dtype=F32)
    want = (d(q)[:1] @ d(w).t()).float()
    assert torch.equal(y.cpu(), want.expand(rows, 24))
    q[:, 1:] = 0
    w[3, 0] = 1
    assert torch.equal(oc.linear_i8(q, one, w, ones, dtype=F32)[:, 3].cpu(), torch.full((rows,), -128.0))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,N", [(5, 64), (90, 72), (300, 520)])
def test_rows_to_their_positions(rows, N, dtype):
    K = 64
    q, w, s, ws = rnd8(1, rows, K), rnd8(2, N, K), make(3, rows).abs() * 0.01, make(4, N).abs() * 0.01
    ref = oc.linear_i8(q, s, w, ws, dtype=dtype)
    idx = ids(rows, rows + 50)
    idx[2], idx[4] = -1, rows + 50
    wide = torch.full((rows + 50, N + 16), 3.0, dtype=dtype, device=DEV)
    y = oc.linear_i8(q, s, w, ws, out_idx=idx, y=wide[:, 8:8 + N])
    ok = torch.ones(rows, dtype=torch.bool, device=DEV)
    ok[[2, 4]] = False
    assert torch.equal(y[idx[ok].long()], ref[ok])
    rest = torch.ones(rows + 50, dtype=torch.bool, device=DEV)
    rest[idx[ok].long()] = False
    assert (y[rest] == 3).all() and (wide[:, :8] == 3).all() and (wide[:, 8 + N:] == 3).all()
    # without positions: the first rows of a longer y
    long = torch.full((rows + 3, N), 3.0, dtype=dtype, device=DEV)
    oc.linear_i8(q, s, w, ws, y=long)
    assert torch.equal(long[:rows], ref) and (long[rows:] == 3).all()


def test_empty():
    x = torch.empty(0, 64, dtype=BF, device=DEV)
    q, s = oc.quant_rows(x)
    assert q.shape == (0, 64) and s.shape == (0,)
    w, ws = oc.quant_rows(make(1, 16, 64))
    assert oc.linear_i8(q, s, w, ws).shape == (0, 16)


def test_quantised_product_is_near_the_product():
    """x w^T from quantised x and w: each factor off by half a step of its row."""
    x, w = make(1, 50, 320, dtype=BF), make(2, 64, 320, dtype=BF)
    q, s = oc.quant_rows(x)
    wq, ws = oc.quant_rows(w)
    y = oc.linear_i8(q, s, wq, ws, dtype=F32)
    sx, sw = d(s)[:, None], d(ws)
    # |x w - q w'| <= |x| half a step of w + |w'| half a step of x, summed; fp32 rounding is far below
    tol = 0.5 * (d(x).abs().sum(1, keepdim=True) * sw + (d(w).abs().sum(1) + 320 * 0.5 * sw) * sx) * 1.001
    assert ((d(y) - d(x) @ d(w).t()).abs() <= tol).all()


def test_captured_replayed_and_other_stream():
    x, idx = make(1, 500, 320, dtype=BF), ids(200, 500).sort().values.int()
    w, ws = oc.quant_rows(make(2, 136, 320, dtype=BF))
    y = torch.zeros(500, 136, dtype=BF, device=DEV)

    def call(out):
        return oc.linear_i8(*oc.quant_rows(x, row_idx=idx), w, ws, act="gelu", out_idx=idx, y=out)

    ref = call(y.clone())
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        other = call(torch.zeros_like(y))
    torch.cuda.synchronize()
    assert torch.equal(ref, other)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(y)
    for i in range(3):
        x.copy_(make(10 + i, 500, 320, dtype=BF))
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, call(torch.zeros_like(y)))
