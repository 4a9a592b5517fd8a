"""Rotary positions with several axes against 64 bits: the rotation by itself,
and inside the reduced, the cached and the uncached attention layer."""
import numpy as np
import pytest
import torch

import paper_2607_23844_amd as oc
from oc_synth import small_workload
from ops_ref import check, d, grid_pos, rope
from parity import TOL, check_output_bars, dev_tensor, rel_err, shapes, to_f64, weights_dev, weights_f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# The angle is off by half a step of a fraction of at most half a turn (pi
# roundings), cosine and sine by 4 units in the last place (8), product, sum and
# difference by 3.
N_ROUND = 15


def make(seed, *s, dtype=torch.float32):
    return torch.randn(*s, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


def ids(n, total, seed=3):
    return torch.randperm(total, generator=torch.Generator().manual_seed(seed))[:n].sort().values.int().to(DEV)


GRID = dict(F=3, H=6, W=10)
CASES = [
    # heads, k_heads, head_dim, rope
    (2, 2, 64, oc.Rope((16, 24, 24))),
    (24, 24, 64, oc.Rope((0, 32, 32))),
    (3, 1, 72, oc.Rope((24, 24, 24), layout="halves")),
    (3, 3, 64, oc.Rope((16, 16, 16), layout="halves", theta=100.0)),          # 16 channels left alone
    (2, 2, 64, oc.Rope((16, 24, 24), layout="halves", scale=(0.5, 1.0, 2.0))),
    (5, 5, 128, oc.Rope((44, 42, 42), layout="halves")),                      # odd numbers of pairs
    (1, 4, 16, oc.Rope((2, 0, 6), layout="halves")),
    (4, 2, 80, oc.Rope((20, 30, 30), layout="split", shared=True)),
    (2, 2, 96, oc.Rope((32, 32, 16), layout="split", shared=True, origin=(7, -3, 100))),
    (2, 2, 48, oc.Rope((48, 0, 0), shared=True, origin=(1 << 30, 0, 0))),
    (1, 1, 32, oc.Rope((0, 0, 2))),
    (7, 7, 128, oc.Rope((0, 64, 64), layout="split", theta=1e6)),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_rotation(case, dtype):
    heads, kh, dh, rp = CASES[case]
    sh = oc.Shape(**GRID, C=heads * dh, heads=heads, head_dim=dh, dtype="bf16" if dtype == torch.bfloat16 else "f32")
    n = 180
    for rows, idx in ((n, None), (1, None), (77, ids(77, n))):
        q, k = make(1, rows, heads, dh, dtype=dtype), make(2, rows, kh, dh, dtype=dtype)
        pos = grid_pos(idx if idx is not None else torch.arange(rows), 6, 10)
        for inv in (False, True):
            qo, ko = oc.rope_qk(q, k, rp, sh, kept_idx=idx, inverse=inv)
            check(qo, *rope(q, pos, rp, inv), N_ROUND, "q")
            check(ko, *rope(k, pos, rp, inv), N_ROUND, "k")
    rot = sum(rp.dims)
    assert torch.equal(qo[..., rot:], q[..., rot:])          # channels past the axes are copied


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["pairs", "halves", "split"])
def test_given_positions_far_and_negative(layout, dtype):
    sh = oc.Shape(1, 1, 1, 4 * 64, 4, 64, 0, "bf16" if dtype == torch.bfloat16 else "f32")
    pos = torch.tensor([[0, 0, 0], [1 << 20, 12345, -7], [-(1 << 31), (1 << 31) - 1, 5], [99991, -99991, 1 << 24]],
                       dtype=torch.int32, device=DEV).repeat(9, 1)[:33]
    rp = oc.Rope((16, 24, 24), layout=layout)
    q, k = make(1, 33, 4, 64, dtype=dtype), make(2, 33, 2, 64, dtype=dtype)
    qo, ko = oc.rope_qk(q, k, rp, sh, pos=pos)
    check(qo, *rope(q, pos, rp), N_ROUND, "q")
    check(ko, *rope(k, pos, rp), N_ROUND, "k")
    assert torch.equal(qo[0], q[0])


ODD = oc.Rope((22, 26, 22), layout="halves")      # halves of 11, 13 and 11: no run of four channels


@pytest.mark.parametrize("rp", [oc.Rope((24, 24, 24)), oc.Rope((24, 24, 24), layout="halves"), ODD])
def test_columns_of_a_projected_buffer_and_in_place(rp):
    sh = oc.Shape(**GRID, C=4 * 72, heads=4, head_dim=72)
    buf = make(5, 180, 6 * 72 + 8, dtype=torch.bfloat16)
    q, k = buf[:, :4 * 72].unflatten(1, (4, 72)), buf[:, 4 * 72:5 * 72].unflatten(1, (1, 72))
    qo, ko = oc.rope_qk(q, k, rp, sh)
    q1, k1 = oc.rope_qk(q.contiguous(), k.contiguous(), rp, sh)
    assert torch.equal(qo, q1) and torch.equal(ko, k1)
    rest = buf[:, 5 * 72:].clone()
    oc.rope_qk(q, k, rp, sh, q_out=q, k_out=k)
    assert torch.equal(q, q1) and torch.equal(k, k1) and torch.equal(buf[:, 5 * 72:], rest)
    # one of the two alone, out of place into columns
    out = torch.zeros_like(buf)
    oc.rope_qk(None, k1, rp, sh, k_out=out[:, 4 * 72:5 * 72].unflatten(1, (1, 72)), inverse=True)
    assert torch.equal(out[:, :4 * 72], torch.zeros_like(out[:, :4 * 72])) and out[:, 4 * 72:5 * 72].any()


@pytest.mark.parametrize("rp", [oc.Rope((16, 24, 24)), ODD])
def test_rows_without_a_token_are_left_alone(rp):
    sh = oc.Shape(**GRID, C=144, heads=2, head_dim=72)
    q, k = make(1, 5, 2, 72, dtype=torch.bfloat16), make(2, 5, 2, 72, dtype=torch.bfloat16)
    idx = torch.tensor([179, -1, 180, 3, -(1 << 31)], dtype=torch.int32, device=DEV)
    qo, ko = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    oc.rope_qk(q, k, rp, sh, kept_idx=idx, q_out=qo, k_out=ko)
    full = oc.rope_qk(q[[0, 3]], k[[0, 3]], rp, sh, kept_idx=idx[[0, 3]])
    assert torch.equal(qo[[0, 3]], full[0]) and torch.equal(ko[[0, 3]], full[1])
    assert (qo[[1, 2, 4]] == 7).all() and (ko[[1, 2, 4]] == 7).all()


def test_not_finite_values_stay_in_their_pair():
    sh = oc.Shape(**GRID, C=64, heads=1, head_dim=64)
    rp = oc.Rope((8, 8, 8), layout="halves")
    q = make(1, 180, 1, 64, dtype=torch.bfloat16)
    ref = oc.rope_qk(q, None, rp, sh)[0]
    q[70, 0, 2], q[70, 0, 40], q[71, 0, 63] = float("inf"), float("nan"), float("-inf")
    out = oc.rope_qk(q, None, rp, sh)[0]
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[70, 0, [2, 6, 40]] = True
    bad[71, 0, 63] = True
    assert torch.equal(out[~bad], ref[~bad])
    assert out[71, 0, 63] == float("-inf") and out[70, 0, 40].isnan()


@pytest.mark.parametrize("rp", [oc.Rope((48, 40, 40)), oc.Rope((48, 40, 40), layout="halves"), ODD])
def test_many_rows_and_heads(rp):
    """Blocks of several rows, more heads than one of them holds at a time."""
    sh = oc.Shape(3, 30, 31, 33 * 128, 33, 128)
    q, k = make(1, 2790, 33, 128, dtype=torch.bfloat16), make(2, 2790, 7, 128, dtype=torch.bfloat16)
    idx = torch.randint(-40, 2830, (2790,), generator=torch.Generator().manual_seed(5)).int().to(DEV)
    qo, ko = oc.rope_qk(q, k, rp, sh, kept_idx=idx, q_out=q.clone(), k_out=k.clone())
    ok = (idx >= 0) & (idx < 2790)
    pos = grid_pos(idx[ok], 30, 31)
    check(qo[ok], *rope(q[ok], pos, rp), N_ROUND, "q")
    check(ko[ok], *rope(k[ok], pos, rp), N_ROUND, "k")
    assert torch.equal(qo[~ok], q[~ok]) and torch.equal(ko[~ok], k[~ok])


def test_gradient_is_the_transpose():
    """<R x, y> = <x, R^T y>: each side off by its outputs' errors."""
    sh = oc.Shape(**GRID, C=3 * 64, heads=3, head_dim=64, dtype="f32")
    rp = oc.Rope((16, 24, 24), layout="split", shared=True)
    x, y = make(1, 180, 3, 64), make(2, 180, 3, 64)
    rx, ry = oc.rope_qk(x, None, rp, sh)[0], oc.rope_qk(y, None, rp, sh, inverse=True)[0]
    pos = grid_pos(torch.arange(180), 6, 10)
    tol = sum(float(((1 + N_ROUND) * 2.0 ** -24 * rope(a, pos, rp)[1] * d(b).abs()).sum()) for a, b in ((x, y), (y, x)))
    assert abs(float((d(rx) * d(y)).sum()) - float((d(x) * d(ry)).sum())) <= tol


def test_captured_replayed_and_other_stream():
    sh = oc.Shape(**GRID, C=24 * 64, heads=24, head_dim=64)
    rp = oc.Rope((0, 32, 32))
    idx = ids(77, 180)
    q, k = make(1, 77, 24, 64, dtype=torch.bfloat16), make(2, 77, 24, 64, dtype=torch.bfloat16)
    ref = oc.rope_qk(q, k, rp, sh, kept_idx=idx)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        other = oc.rope_qk(q, k, rp, sh, kept_idx=idx)
    torch.cuda.synchronize()
    assert torch.equal(ref[0], other[0]) and torch.equal(ref[1], other[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = oc.rope_qk(q, k, rp, sh, kept_idx=idx)
    for i in range(3):
        q.copy_(make(20 + i, 77, 24, 64, dtype=torch.bfloat16))
        idx.copy_(ids(77, 180, 30 + i))
        g.replay()
        torch.cuda.synchronize()
        eager = oc.rope_qk(q, k, rp, sh, kept_idx=idx)
        assert torch.equal(out[0], eager[0]) and torch.equal(out[1], eager[1])


# ---------------------------------------------------------------------------
# inside the layer
# ---------------------------------------------------------------------------

def attention(X, ctx, pos, W, heads, dh, rp):
    """One sequence in 64 bits: q and k of its tokens turned, context rows not."""
    A = np.concatenate([X, ctx]) if ctx is not None else X
    n = len(X)
    q, k, v = (torch.from_numpy(A @ W[w].T).view(len(A), heads, dh) for w in ("wq", "wk", "wv"))
    q, k = q.clone(), k.clone()
    q[:n], k[:n] = rope(q[:n], pos, rp)[0], rope(k[:n], pos, rp)[0]
    s = torch.matmul(q.transpose(0, 1), k.permute(1, 2, 0)) / dh ** 0.5
    o = torch.matmul(s.softmax(-1), v.transpose(0, 1)).transpose(0, 1).reshape(len(A), heads * dh)
    return o.numpy() @ W["wo"].T


def bars(y, ref, dtype, what):
    check_output_bars(rel_err(y, ref, dtype), rel_err(y, ref), dtype, what)


LAYERS = [
    ("token", dict(F=1, H=16, W=16, C=64, heads=2, head_dim=32, dtype="bf16", r=0.5, n_ctx=5), oc.Rope((0, 16, 16))),
    ("token", dict(F=1, H=16, W=16, C=64, heads=1, head_dim=64, dtype="f32", r=0.5, n_ctx=3),
     oc.Rope((0, 24, 24), layout="halves")),
    ("frame", dict(F=5, H=8, W=8, C=72, heads=1, head_dim=72, dtype="bf16", r_frame=0.4),
     oc.Rope((24, 24, 24), layout="halves")),
    ("frame", dict(F=6, H=8, W=8, C=64, heads=2, head_dim=32, dtype="bf16", r_frame=0.34, patch_k=2),
     oc.Rope((8, 12, 12))),
    ("block", dict(F=9, H=8, W=8, C=128, heads=2, head_dim=64, dtype="bf16", r=0.5), oc.Rope((64, 0, 0))),
    ("block", dict(F=70, H=4, W=4, C=64, heads=1, head_dim=64, dtype="f32", r=0.5), oc.Rope((64, 0, 0), layout="split")),
    ("frame_token", dict(F=5, H=8, W=8, C=64, heads=2, head_dim=32, dtype="bf16", r=0.5, r_frame=0.4),
     oc.Rope((8, 12, 12), layout="split", shared=True)),
]


@pytest.mark.parametrize("i", range(len(LAYERS)), ids=[f"{g}-{k['dtype']}-{i}" for i, (g, k, _) in enumerate(LAYERS)])
def test_layer(i):
    gran, kw, rp = LAYERS[i]
    wl = small_workload(gran, n_steps=2, seed=20 + i, **kw)
    sh, cf, _, _ = shapes(wl)
    W, W64 = weights_dev(wl), weights_f64(wl)
    dt = kw["dtype"]
    ctx = dev_tensor(wl, wl.ctx) if wl.n_ctx else None
    ctx64 = wl.f64(wl.ctx) if wl.n_ctx else None
    cache, plain = oc.LayerCache(sh, DEV), oc.LayerCache(sh, DEV)
    prev = None
    for s in range(2):
        x, x64 = dev_tensor(wl, wl.steps[s]), wl.f64(wl.steps[s]).reshape(sh.F * sh.N, sh.C)
        y, y_ctx, tr = oc.layer_cached(x, W, cache, sh, cf, ctx=ctx, trace=True, rope=rp)
        _, _, tp = oc.layer_cached(x, W, plain, sh, cf, ctx=ctx, trace=True)
        for k in ("kept_idx", "cached_idx", "restore_map", "node_idx"):
            assert torch.equal(tr[k], tp[k]), k              # the decisions do not depend on the rotation
        y = to_f64(y).reshape(sh.F * sh.N, sh.C)
        kept = tr["kept_idx"].cpu().long().numpy()
        pl = oc.plan(sh, cf)
        if gran == "frame" and cf.patch_k > 1:
            seqs = [kept[kept // sh.N == f] for f in range(sh.F)]
        else:
            seqs = list(kept.reshape(pl.n_seq, pl.seq_len))
        outs = [attention(x64[q], ctx64, grid_pos(torch.from_numpy(q), sh.H, sh.W), W64, sh.heads, sh.head_dim, rp)
                for q in seqs if len(q)]
        ref = np.concatenate([o[:len(q)] for o, q in zip(outs, [q for q in seqs if len(q)])])
        bars(y[np.concatenate(seqs)], ref, dt, "retained rows")
        if ctx is not None:
            bars(to_f64(y_ctx), outs[0][len(seqs[0]):], dt, "context rows")
        cached = tr["cached_idx"].cpu().long().numpy()
        if s == 1:
            assert np.array_equal(y[cached], prev[cached])   # restored from the step before
        prev = y
    # the uncached layer, against the same formulas on a few sequences
    yf, _ = oc.attn_full(x, W, sh, cf, ctx=ctx, rope=rp)
    yf = to_f64(yf).reshape(sh.F * sh.N, sh.C)
    groups = [np.arange(sh.F) * sh.N + n for n in (0, 5)] if gran == "block" else \
        [f * sh.N + np.arange(sh.N) for f in (0, sh.F - 1)]
    for q in groups:
        ref = attention(x64[q], ctx64, grid_pos(torch.from_numpy(q), sh.H, sh.W), W64, sh.heads, sh.head_dim, rp)
        bars(yf[q], ref[:len(q)], dt, "uncached rows")


def reduced(rp, L, n_seq, heads, dh, n_ctx=0, C=128):
    """attn_reduced of random rows, some of them without a token (not turned), against 64 bits."""
    sh = oc.Shape(**GRID, C=C, heads=heads, head_dim=dh, n_ctx=n_ctx)
    n, hd = sh.F * sh.N, heads * dh
    g = torch.Generator().manual_seed(L)
    W64 = {k: torch.randn(hd, C, generator=g, dtype=torch.float64) / C ** 0.5 for k in ("wq", "wk", "wv")}
    W64["wo"] = torch.randn(C, hd, generator=g, dtype=torch.float64) / hd ** 0.5
    W = {k: v.bfloat16().to(DEV) for k, v in W64.items()}
    W64 = {k: v.cpu().double().numpy() for k, v in W.items()}
    x = torch.randn(n_seq * L, C, generator=g).bfloat16()
    ctx = torch.randn(n_ctx, C, generator=g).bfloat16() if n_ctx else None
    idx = torch.randint(0, n, (n_seq * L,), generator=g, dtype=torch.int32)
    idx[::7] = n
    idx[3::11] = -1
    y, yc = oc.attn_reduced(x.to(DEV), n_seq, L, W, sh, ctx=None if ctx is None else ctx.to(DEV), rope=rp,
                            kept_idx=idx.to(DEV))
    there = (idx >= 0) & (idx < n)
    pos = grid_pos(torch.where(there, idx, 0).long(), sh.H, sh.W)
    pos[~there] = 0   # (the angle at the origin is nothing)
    c64 = None if ctx is None else ctx.double().numpy()
    ref = np.concatenate([attention(x[i:i + L].double().numpy(), c64, pos[i:i + L], W64, heads, dh, rp)
                          for i in range(0, n_seq * L, L)])
    y = to_f64(y if yc is None else torch.cat([y, yc])).reshape(ref.shape)
    # The computation's error by the layer's bar.  Beside it the outputs' rounding, at most 2^-8 of a value, so 2^-8 of
    # the largest one in the unadjusted error (among millions of outputs that is 6 times their RMS: 0.0235).
    assert rel_err(y, ref, "bf16") <= TOL["bf16"]
    assert rel_err(y, ref) <= TOL["bf16"] + 2.0 ** -8 * np.abs(ref).max() / np.sqrt(np.mean(ref * ref))


@pytest.mark.parametrize("L,n_seq,n_ctx", [(300, 1, 21), (90, 3, 0), (40, 7, 0)])
@pytest.mark.parametrize("heads,dh,rp", [
    (5, 72, oc.Rope((24, 24, 24))), (5, 72, oc.Rope((24, 24, 24), layout="halves")),
    (3, 128, oc.Rope((32, 48, 48), layout="halves")), (5, 64, oc.Rope((0, 32, 32), layout="split")),
    (6, 48, oc.Rope((16, 8, 8))), (3, 96, oc.Rope((32, 32, 32), layout="halves")),
    (7, 80, oc.Rope((14, 10, 22))), (9, 32, oc.Rope((8, 8, 16), layout="halves")), (17, 16, oc.Rope((0, 8, 8))),
    (4, 128, oc.Rope((40, 40, 8), layout="split", shared=True)), (4, 64, oc.Rope((64, 0, 0))),
])
def test_reduced_sequences(L, n_seq, n_ctx, heads, dh, rp):
    """Heads and halves inside and across the tiles of the projection."""
    reduced(rp, L, n_seq, heads, dh, n_ctx)


@pytest.mark.parametrize("C,L,n_seq,n_ctx,heads,dh", [(1536, 2048, 1, 333, 24, 64), (1152, 256, 12, 0, 16, 72),
                                                      (320, 90, 222, 0, 5, 64), (640, 512, 16, 0, 10, 64),
                                                      (1024, 128, 4, 0, 8, 128), (1152, 16, 150, 0, 16, 72)])
@pytest.mark.parametrize("layout", ["pairs", "halves"])
def test_large_projections(layout, C, L, n_seq, n_ctx, heads, dh):
    """The large tiles' rotation."""
    reduced(oc.Rope((16, 24, 24), layout=layout), L, n_seq, heads, dh, n_ctx, C)


@pytest.mark.parametrize("L,n_seq", [(1, 130), (3, 43), (25, 11), (64, 3)])
@pytest.mark.parametrize("rp", [oc.Rope((64, 0, 0)), oc.Rope((16, 24, 24), layout="halves", shared=True),
                                oc.Rope((14, 10, 22)), oc.Rope((14, 10, 22), layout="halves"),
                                oc.Rope((6, 0, 4), layout="split")])
def test_short_sequences(rp, L, n_seq):
    """Heads of 64 and few tokens a sequence; rows without a token are not turned."""
    reduced(rp, L, n_seq, 3, 64)


def test_staged_calls_and_runner_match_the_layer_call():
    from paper_2607_23844_amd import runner
    gran, kw, rp = LAYERS[0]
    wl = small_workload(gran, n_steps=2, seed=20, **kw)
    sh, cf, _, _ = shapes(wl)
    W, ctx = weights_dev(wl), dev_tensor(wl, wl.ctx)
    ws = oc.workspace(sh, cf, DEV)
    cache = oc.LayerCache(sh, DEV)
    run = runner.LayerRunner(sh, cf, W, DEV, ctx=ctx, rope=rp)
    for s in range(2):
        x = dev_tensor(wl, wl.steps[s])
        y, y_ctx, tr = oc.layer_cached(x, W, cache, sh, cf, ctx=ctx, trace=True, rope=rp)
        assert torch.equal(run(x), y) and torch.equal(run.y_ctx, y_ctx)
    nm, ni = oc.match(x, sh, cf, ws)
    kept, _, rmap = oc.select(nm, ni, sh, cf, ws)
    yk, yc = oc.attn_reduced(oc.gather(x, kept, sh, cf), 1, kept.numel(), W, sh, ctx=ctx, rope=rp, kept_idx=kept)
    out = oc.restore(yk, rmap, sh, cache_y=y, y=y.clone())
    assert torch.equal(out, y) and torch.equal(yc, y_ctx)
    # no rotation: the call without it
    a, _ = oc.attn_full(x, W, sh, cf, ctx=ctx)
    b = runner.FullRunner(sh, cf, W, DEV, ctx=ctx)
    assert torch.equal(a, b(x))


def test_layer_captured_and_replayed():
    gran, kw, rp = LAYERS[3]
    wl = small_workload(gran, n_steps=2, seed=23, **kw)
    sh, cf, _, _ = shapes(wl)
    W, ws = weights_dev(wl), oc.workspace(sh, cf, DEV)
    cache, eager = oc.LayerCache(sh, DEV), oc.LayerCache(sh, DEV)
    x = dev_tensor(wl, wl.steps[0])
    for c in (cache, eager):
        oc.layer_cached(x, W, c, sh, cf, ws=ws, rope=rp)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        oc.layer_cached(x, W, cache, sh, cf, ws=ws, rope=rp)
    for i in range(3):
        x.copy_(dev_tensor(wl, wl.steps[i % 2]) * (1 + i))
        g.replay()
        torch.cuda.synchronize()
        oc.layer_cached(x, W, eager, sh, cf, rope=rp)
        assert torch.equal(cache.y, eager.y)
