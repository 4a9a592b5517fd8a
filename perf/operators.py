"""The operators between and around a denoiser's sublayers, as they are timed.

A case is one call (or the two calls that always go together) through the
public entry points: the norms around a sublayer fused with gate, modulation
and residual, and their gradients; the rotation of q and k by the positions
of the retained tokens on the time / height / width grid; and the product in
8-bit integers of rows quantised on the spot.  `run` computes the same in
elementary torch operations unless `own` is set; `exact` is the definition in
64 bits.
"""
import math

import torch

own = False            # True: the library's entry points; False: their plain form

OUTLIER = 20.0         # a few channels of a residual stream stand this far above the rest
EPS = 1e-6


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _norm(name, rows, C, dtype="bf16", pre="layer", post="none", affine=False, y=True, rows_per_mod=0, gate=True,
          res_scale=1.0, grad=False):
    """rows_per_mod: rows that share a modulation row (gate, scale, shift); 0: none."""
    d = dict(op="norm_grad" if grad else "norm", rows=rows, C=C, dtype=dtype, pre=pre, post=post if y else "none",
             affine=affine, y=y, rows_per_mod=rows_per_mod, gate=gate and y and rows_per_mod > 0,
             res_scale=res_scale if y else 1.0)
    return dict(d, name=name) if name else d


def _rope(name, F, H, W, heads, k_heads, head_dim, dims, keep=1.0, dtype="bf16", layout="pairs", shared=False,
          inverse=False, fused=False, far=0):
    """keep: fraction of the grid's tokens retained; fused: q and k are columns
    of one projected buffer; far > 0: positions in [0, far) given per row."""
    d = dict(op="rope", F=F, H=H, W=W, heads=heads, k_heads=k_heads, head_dim=head_dim, d_t=dims[0], d_h=dims[1],
             d_w=dims[2], keep=keep, dtype=dtype, layout=layout, shared=shared, inverse=inverse, fused=fused, far=far)
    return dict(d, name=name) if name else d


def _linear(name, tokens, rows, K, N, dtype="bf16", bias=True, act="none", scatter=False):
    """rows of `tokens` rows are quantised (all of them in place when equal)
    and multiplied; scatter: written back at their positions."""
    d = dict(op="linear", tokens=tokens, rows=rows, K=K, N=N, dtype=dtype, bias=bias, act=act, scatter=scatter)
    return dict(d, name=name) if name else d


def listed():
    return [
        # one pooled token: the smallest call, where launches and latency count
        _norm("norm_one_row", 1, 1536, rows_per_mod=1),
        # 333 text tokens with norms before and after the sublayer, each with its weights, and a scaled residual
        _norm("norm_context_sandwich", 333, 1536, pre="rms", post="rms", affine=True, rows_per_mod=333,
              res_scale=0.7071),
        # 64 x 64 image tokens after the attention: gate, residual, layer norm, modulation
        _norm("norm_image", 4096, 1536, rows_per_mod=4096),
        # 25 frames of 72 x 128 tokens kept in fp32, a modulation row for each frame
        _norm("norm_video_f32", 230400, 320, dtype="f32", rows_per_mod=9216),
        # training: 16 frames of 16 x 16 tokens with a modulation row for each frame
        _norm("norm_grad_frames", 4096, 1152, rows_per_mod=256, grad=True),
        # training: a whole video level with weights on both norms
        _norm("norm_grad_video", 230400, 320, pre="rms", post="rms", affine=True, rows_per_mod=9216, grad=True),
        # the 2048 tokens that a Token Cache retained of 64 x 64, height and width axes
        _rope("rope_retained", 1, 64, 64, 24, 24, 64, (0, 32, 32), keep=0.5),
        # a video level's q and k inside the projected buffer, three axes in halves
        _rope("rope_video_fused", 25, 72, 128, 5, 5, 64, (16, 24, 24), layout="halves", fused=True),
        # the gradient at far positions, fp32, an odd number of rows, part of the head unrotated
        _rope("rope_grad_far_f32", 1, 1, 1021, 16, 16, 72, (16, 24, 24), dtype="f32", layout="split", shared=True,
              inverse=True, far=1 << 20),
        # a time step's modulation vectors: one row, bound by the weights
        _linear("linear_one_row", 1, 1, 1536, 9216),
        # the retained half of the tokens through an output projection, back to their positions
        _linear("linear_retained", 4096, 2048, 1536, 1536, bias=False, scatter=True),
        # image and text tokens through the first feed-forward product
        _linear("linear_ffn_up", 4429, 4429, 1536, 6144, act="gelu"),
    ]


def _log(rng, lo, hi, step=1):
    """A whole multiple of step in [lo, hi], spread over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return int(min(hi // step, max(-(-lo // step), round(v / step)))) * step


def _split_axes(rng, head_dim, axes):
    """Even shares of a head for `axes` axes (time, height, width), maybe not all of it."""
    left = head_dim if rng.random() < 0.7 else 2 * rng.randint(axes, head_dim // 2)
    cut = sorted(rng.sample(range(1, left // 2), axes - 1)) if axes > 1 else []
    parts = [2 * (b - a) for a, b in zip([0] + cut, cut + [left // 2])]
    return tuple([0] * (3 - axes) + parts) if axes > 1 else rng.choice([(parts[0], 0, 0), (0, 0, parts[0])])


def _draw_once(rng):
    op = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "rope", "rope", "linear", "linear"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op in ("norm", "norm_grad"):
        C = _log(rng, 64, 4096, 8)
        rows = _log(rng, 1, 230400)
        per = rng.choice([0, 1, rows, rows, -(-rows // rng.randint(2, 25)), rng.randint(1, rows)])
        return _norm(None, rows, C, dtype=dtype, pre=rng.choice(["layer", "layer", "rms"]),
                     post=rng.choice(["none", "none", "rms", "layer"]), affine=rng.random() < 0.5,
                     y=rng.random() < 0.8, rows_per_mod=per, gate=rng.random() < 0.8,
                     res_scale=rng.choice([1.0, 1.0, 0.5, 0.7071]), grad=op == "norm_grad")
    if op == "rope":
        dh = rng.choice([16, 32, 48, 64, 64, 64, 72, 80, 96, 128])
        heads = _log(rng, 1, max(1, 1536 // dh))
        k_heads = rng.choice([heads, heads, 1])
        F, H, W = rng.choice([1, rng.randint(2, 25)]), _log(rng, 1, 72), _log(rng, 1, 128)
        layout = rng.choice(["pairs", "pairs", "halves", "split"])
        return _rope(None, F, H, W, heads, k_heads, dh, _split_axes(rng, dh, rng.choice([1, 2, 3, 3])),
                     keep=rng.choice([1.0, 0.75, 0.5, 0.25]), dtype=dtype, layout=layout,
                     shared=layout == "split" or rng.random() < 0.2, inverse=rng.random() < 0.4,
                     fused=rng.random() < 0.5, far=rng.choice([0, 0, 0, 1 << 20]))
    tokens = _log(rng, 1, 36864)
    rows = tokens if rng.random() < 0.5 else max(1, int(tokens * rng.choice([0.75, 0.5, 0.25])))
    return _linear(None, tokens, rows, _log(rng, 64, 6144, 8), _log(rng, 64, 6144, 8), dtype=dtype,
                   bias=rng.random() < 0.5, act=rng.choice(["none", "none", "gelu"]), scatter=rng.random() < 0.5)


def draw(rng):
    most = [work(c) for c in listed()]
    while True:
        c = _draw_once(rng)
        w = work(c)
        if w["bytes"] <= max(m["bytes"] for m in most) and w["flops"] <= max(m["flops"] for m in most):
            return c


def _esz(c):
    return 2 if c["dtype"] == "bf16" else 4


def _n_mod(c):
    return -(-c["rows"] // c["rows_per_mod"]) if c["rows_per_mod"] else 0


def _n_kept(c):
    return max(1, int(c["F"] * c["H"] * c["W"] * c["keep"]))


def work(c):
    """Every input read once, every output written once, and the operations of the formulas."""
    e = _esz(c)
    if c["op"] in ("norm", "norm_grad"):
        rc = c["rows"] * c["C"]
        vec = _n_mod(c) * c["C"] * (2 + c["gate"])                                 # modulation
        par = c["C"] * c["affine"] * (2 + 2 * (c["post"] != "none"))    # weights and biases
        if c["op"] == "norm":
            return {"bytes": (rc * (4 if c["y"] else 2) + vec + par) * e, "flops": rc * (16 if c["y"] else 9)}
        return {"bytes": (rc * (6 if c["y"] else 4) + vec + par) * e + (vec + par) * 4,
                "flops": rc * (40 if c["y"] else 22)}
    if c["op"] == "rope":
        n = _n_kept(c) * (c["heads"] + c["k_heads"])
        rot = c["d_t"] + c["d_h"] + c["d_w"]
        return {"bytes": 2 * n * c["head_dim"] * e + _n_kept(c) * (12 if c["far"] else 4 * (c["keep"] < 1)),
                "flops": 3 * n * rot}
    return {"bytes": c["rows"] * (c["K"] + c["N"]) * e + c["N"] * (c["K"] + 4 + c["bias"] * e)
            + 4 * (c["rows"] < c["tokens"]) * c["rows"], "flops": 2 * c["rows"] * c["K"] * c["N"]}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _dt(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _stream_rows(g, rows, C, dt):
    """Rows of a residual stream: normal, with every 97th channel far above the rest."""
    x = torch.randn((rows, C), generator=g, device="cuda")
    x[:, 5::97] *= OUTLIER
    return x.to(dt)


def _inputs(c, seed):
    """The tensors of a case, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _dt(c)

    def randn(*shape, scale=1.0, mean=0.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale + mean).to(dt)

    if c["op"] in ("norm", "norm_grad"):
        rows, C, M = c["rows"], c["C"], _n_mod(c)
        s = {"x": _stream_rows(g, rows, C, dt), "y": randn(rows, C, scale=2.0) if c["y"] else None}
        # the vectors of one modulation product, next to each other in a row of it
        vec = randn(M, 3 * C, scale=0.3) if M else None
        s["gate"] = vec[:, :C] if c["gate"] else None
        s["scale"] = vec[:, C:2 * C] if M else None
        s["shift"] = vec[:, 2 * C:] if M else None
        for k, has in (("pre", True), ("post", c["post"] != "none")):
            s[k + "_w"] = randn(C, scale=0.1, mean=1.0) if c["affine"] and has else None
            s[k + "_b"] = randn(C, scale=0.1) if c["affine"] and has else None
        if c["op"] == "norm_grad":
            s["dn"] = randn(rows, C)
            s["dh"] = randn(rows, C, scale=0.5)
        return s
    if c["op"] == "rope":
        n, dh = _n_kept(c), c["head_dim"]
        FN = c["F"] * c["H"] * c["W"]
        if c["fused"]:
            buf = randn(n, (c["heads"] + 2 * c["k_heads"]) * dh)
            q = buf[:, :c["heads"] * dh].unflatten(1, (c["heads"], dh))
            k = buf[:, c["heads"] * dh:(c["heads"] + c["k_heads"]) * dh].unflatten(1, (c["k_heads"], dh))
        else:
            q, k = randn(n, c["heads"], dh), randn(n, c["k_heads"], dh)
        s = {"q": q, "k": k, "idx": None, "pos": None}
        if c["far"]:
            s["pos"] = torch.randint(0, c["far"], (n, 3), generator=g, device="cuda", dtype=torch.int32)
        elif n < FN:
            s["idx"] = torch.randperm(FN, generator=g, device="cuda")[:n].sort().values.to(torch.int32)
        return s
    s = {"x": _stream_rows(g, c["tokens"], c["K"], dt), "w": randn(c["N"], c["K"], scale=c["K"] ** -0.5),
         "bias": randn(c["N"], scale=0.1) if c["bias"] else None, "idx": None, "y": None}
    if c["rows"] < c["tokens"]:
        s["idx"] = torch.randperm(c["tokens"], generator=g, device="cuda")[:c["rows"]].sort().values.to(torch.int32)
    if c["scatter"]:
        s["y"] = randn(c["tokens"], c["N"])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["op"] == "linear":
        # the weights are quantised once
        w = s.pop("w")
        if own:
            import paper_2607_23844_amd as oc
            s["wq"], s["ws"] = oc.quant_rows(w)
        else:
            s["wq"], s["ws"] = _quant(w)
    if own:
        import paper_2607_23844_amd as oc
        if case["op"] in ("norm", "norm_grad"):
            s["shape"] = oc.Shape(1, 1, 1, case["C"], 1, 16, 0, case["dtype"])
            s["pre"] = oc.Norm(case["pre"], EPS, s["pre_w"], s["pre_b"])
            s["post"] = oc.Norm(case["post"], EPS, s["post_w"], s["post_b"]) if case["y"] else None
            s["mod"] = oc.Mod(s["gate"], s["scale"], s["shift"], case["rows_per_mod"]) if _n_mod(case) else None
        elif case["op"] == "rope":
            s["shape"] = oc.Shape(case["F"], case["H"], case["W"], case["heads"] * case["head_dim"], case["heads"],
                                  case["head_dim"], 0, case["dtype"])
            s["rope"] = oc.Rope((case["d_t"], case["d_h"], case["d_w"]), layout=case["layout"], shared=case["shared"])
    return s


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------

def _normed(v, kind, w, b):
    """(normalised rows, their 1/deviation, with weights)"""
    if kind == "none":
        return v, None, v
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    r = 1.0 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
    u = v * r
    a = u
    if w is not None:
        a = a * w
    if b is not None:
        a = a + b
    return u, r, a


def _mod_rows(v, c):
    """A modulation vector for every row, in 32 bits."""
    if v is None or v.shape[0] == 1:
        return _f(v)
    m = torch.arange(c["rows"], device=v.device) // c["rows_per_mod"]
    return v.float()[m]


def _f(t):
    return None if t is None else t.float()


def _norm_plain(s, c):
    dt = _dt(c)
    h = x = s["x"].float()
    if c["y"]:
        z = _normed(s["y"].float(), c["post"], _f(s["post_w"]), _f(s["post_b"]))[2]
        g = _mod_rows(s["gate"], c)
        h = c["res_scale"] * x + (z if g is None else g * z)
    n = _normed(h, c["pre"], _f(s["pre_w"]), _f(s["pre_b"]))[2]
    if c["rows_per_mod"]:
        n = n * (1.0 + _mod_rows(s["scale"], c)) + _mod_rows(s["shift"], c)
    return {"h": h.to(dt), "n": n.to(dt)} if c["y"] else {"n": n.to(dt)}


def _norm_back(dv, u, r, kind):
    """Gradient of a normalisation from that of its normalised rows."""
    if kind == "none":
        return dv
    d = dv - u * (dv * u).mean(1, keepdim=True)
    if kind == "layer":
        d = d - dv.mean(1, keepdim=True)
    return d * r


def _mod_sum(d, c):
    """Sums over the rows that share a modulation row."""
    n, per = _n_mod(c), c["rows_per_mod"]
    if n * per > c["rows"]:
        d = torch.cat([d, d.new_zeros((n * per - c["rows"], c["C"]))])
    return d.view(n, per, c["C"]).sum(1)


def _norm_grad_plain(s, c):
    dt = _dt(c)
    x, dn, out = s["x"].float(), s["dn"].float(), {}
    h = x
    if c["y"]:
        v, ry, z = _normed(s["y"].float(), c["post"], _f(s["post_w"]), _f(s["post_b"]))
        g = _mod_rows(s["gate"], c)
        h = c["res_scale"] * x + (z if g is None else g * z)
    u, rh, a = _normed(h, c["pre"], _f(s["pre_w"]), _f(s["pre_b"]))
    da = dn
    if c["rows_per_mod"]:
        out["scale"], out["shift"] = _mod_sum(dn * a, c), _mod_sum(dn, c)
        da = dn * (1.0 + _mod_rows(s["scale"], c))
    if c["affine"]:
        out["pre_w"], out["pre_b"] = (da * u).sum(0), da.sum(0)
        da = da * s["pre_w"].float()
    dh = s["dh"].float() + _norm_back(da, u, rh, c["pre"])
    out["dx"] = (c["res_scale"] * dh).to(dt)
    if c["y"]:
        dz = dh
        if g is not None:
            out["gate"] = _mod_sum(dh * z, c)
            dz = dh * g
        if s["post_w"] is not None:
            out["post_w"], out["post_b"] = (dz * v).sum(0), dz.sum(0)
            dz = dz * s["post_w"].float()
        out["dy"] = _norm_back(dz, v, ry, c["post"]).to(dt)
    return {k: out[k] for k in sorted(out)}


def _pairs(c):
    """(first channel, second channel, axis, exponent) of every rotated pair."""
    dims = (c["d_t"], c["d_h"], c["d_w"])
    total, out, off = sum(dims), [], 0
    for a, d in enumerate(dims):
        for i in range(d // 2):
            p = off // 2 + i
            if c["layout"] == "pairs":
                lo, hi = 2 * p, 2 * p + 1
            elif c["layout"] == "halves":
                lo, hi = off + i, off + i + d // 2
            else:
                lo, hi = p, p + total // 2
            out.append((lo, hi, a, 2.0 * p / total if c["shared"] else 2.0 * i / d))
        off += d
    return out


def _positions(s, c):
    """[rows, 3] positions (frame, row, column)."""
    if s["pos"] is not None:
        return s["pos"].long()
    t = s["idx"].long() if s["idx"] is not None else torch.arange(c["F"] * c["H"] * c["W"], device=s["q"].device)
    n = t % (c["H"] * c["W"])
    return torch.stack([t // (c["H"] * c["W"]), n // c["W"], n % c["W"]], 1)


def _rope_plain(s, c):
    dt, pr = _dt(c), _pairs(c)
    dev = s["q"].device
    lo, hi, ax = (torch.tensor([p[i] for p in pr], device=dev) for i in range(3))
    f = torch.tensor([10000.0 ** -p[3] for p in pr], device=dev, dtype=torch.float64)
    angle = _positions(s, c)[:, ax].double() * f                 # far positions: the angle in 64 bits
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if c["inverse"]:
        sin = -sin
    res = []
    for t in (s["q"], s["k"]):
        v = t.float()
        o = v.clone()
        a, b = v[..., lo], v[..., hi]
        o[..., lo] = a * cos - b * sin
        o[..., hi] = a * sin + b * cos
        res.append(o.to(dt))
    return {"q": res[0], "k": res[1]}


def _quant(x):
    """Whole numbers (in fp32) and the scale of every row; quotients next to a
    border in 64 bits, ties to the even number."""
    top = x.abs().amax(1, keepdim=True).float()
    d = x.double() * 127.0 / torch.where(top > 0, top, torch.ones_like(top)).double()
    return torch.round(d).float(), top[:, 0] / 127.0


def _gelu(v):
    return 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))


def _linear_plain(s, c):
    x = s["x"] if s["idx"] is None else s["x"][s["idx"].long()]
    q, sx = _quant(x)
    v = (q @ s["wq"].t()) * sx[:, None] * s["ws"]
    if s["bias"] is not None:
        v = v + s["bias"].float()
    if c["act"] == "gelu":
        v = _gelu(v)
    v = v.to(_dt(c))
    if not c["scatter"]:
        return v
    rows = s["idx"].long() if s["idx"] is not None else torch.arange(c["rows"], device=v.device)
    s["y"][rows] = v
    return s["y"]


# ---------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------

def _run_own(s, c):
    import paper_2607_23844_amd as oc
    if c["op"] == "norm":
        h, n = oc.norm_gate(s["x"], s["shape"], y=s["y"], post=s["post"], pre=s["pre"], mod=s["mod"],
                            res_scale=c["res_scale"])
        return {"h": h, "n": n} if c["y"] else {"n": n}
    if c["op"] == "norm_grad":
        g = oc.norm_gate_grad(s["x"], s["shape"], dn=s["dn"], dh=s["dh"], y=s["y"], post=s["post"], pre=s["pre"],
                              mod=s["mod"], res_scale=c["res_scale"])
        return {k: g[k] for k in sorted(g) if g[k] is not None}
    if c["op"] == "rope":
        q, k = oc.rope_qk(s["q"], s["k"], s["rope"], s["shape"], kept_idx=s["idx"], pos=s["pos"],
                          inverse=c["inverse"])
        return {"q": q, "k": k}
    q, sx = oc.quant_rows(s["x"], row_idx=s["idx"])
    out_idx = s["idx"] if c["scatter"] else None
    return oc.linear_i8(q, sx, s["wq"], s["ws"], bias=s["bias"], act=c["act"], out_idx=out_idx, y=s["y"],
                        dtype=_dt(c))


def run(state):
    c = state["case"]
    if own:
        return _run_own(state, c)
    return {"norm": _norm_plain, "norm_grad": _norm_grad_plain, "rope": _rope_plain, "linear": _linear_plain}[c["op"]](
        state, c)


# ---------------------------------------------------------------------------
# 64 bits
# ---------------------------------------------------------------------------

def _norm64(v, kind, w, b):
    if kind == "layer":
        v = (v - v.mean(-1, keepdim=True)) / (v.var(-1, unbiased=False, keepdim=True) + EPS).sqrt()
    elif kind == "rms":
        v = v / (v.square().mean(-1, keepdim=True) + EPS).sqrt()
    v = v if w is None else v * w
    return v if b is None else v + b


def _norm_exact(c, s, grad):
    """The definition; gradients by differentiating it."""
    t = {k: v.double().requires_grad_(grad) for k, v in s.items()
         if v is not None and k not in ("dn", "dh")}
    per = c["rows_per_mod"]

    def spread(v):
        return None if v is None else v.repeat_interleave(per, 0)[:c["rows"]]

    gate, scale, shift = (spread(t.get(k)) for k in ("gate", "scale", "shift"))
    h = t["x"]
    if c["y"]:
        z = _norm64(t["y"], c["post"], t.get("post_w"), t.get("post_b"))
        h = c["res_scale"] * h + (z if gate is None else gate * z)
    n = _norm64(h, c["pre"], t.get("pre_w"), t.get("pre_b"))
    if scale is not None:
        n = n + n * scale + shift
    if not grad:
        return {"h": h, "n": n} if c["y"] else {"n": n}
    torch.autograd.backward([h, n], [s["dh"].double(), s["dn"].double()])
    out = {("d" + k if k in ("x", "y") else k): v.grad for k, v in t.items()}
    return {k: out[k] for k in sorted(out)}


def _rope_exact(c, s):
    """Pairs as complex numbers, turned."""
    pos, out = _positions(s, c).double(), {}
    for name in ("q", "k"):
        v = s[name].double()
        o = v.clone()
        for lo, hi, a, e in _pairs(c):
            ang = pos[:, a] * 10000.0 ** -e
            turn = torch.polar(torch.ones_like(ang), -ang if c["inverse"] else ang)[:, None]
            w = torch.complex(v[..., lo], v[..., hi]) * turn
            o[..., lo], o[..., hi] = w.real, w.imag
        out[name] = o
    return out


def _linear_exact(c, s):
    def q64(x):
        x = x.double()
        top = x.abs().amax(1, keepdim=True)
        return torch.where(top > 0, torch.round(x * 127.0 / top), torch.zeros_like(x)), top / 127.0

    x = s["x"] if s["idx"] is None else s["x"].index_select(0, s["idx"].long())
    q, sx = q64(x)
    w, sw = q64(s["w"])
    v = torch.mm(q, w.t().contiguous()) * (sx * sw.t())
    if s["bias"] is not None:
        v += s["bias"].double()
    if c["act"] == "gelu":
        v = v / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))
    if not c["scatter"]:
        return v
    return v if s["idx"] is None else s["y"].double().index_copy(0, s["idx"].long(), v)


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] in ("norm", "norm_grad"):
        return _norm_exact(case, s, case["op"] == "norm_grad")
    if case["op"] == "rope":
        return _rope_exact(case, s)
    return _linear_exact(case, s)
