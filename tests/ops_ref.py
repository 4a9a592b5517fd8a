"""The operators around a sublayer in 64 bits on the CPU, plainly from their
formulas, with a bound on the error of their evaluation in 32 bits.

Bounds: every quantity carries (value, size), where size bounds the magnitudes
that its evaluation adds up (the formula on absolute values); an evaluation in
fp32 whose longest chain has n roundings is off by at most n 2^-24 size, to
first order.
"""
import torch

U32 = 2.0 ** -24


def half_step(dtype):
    return {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}[dtype]


def d(t):
    return None if t is None else t.detach().cpu().double()


def norm(v, size, kind, eps):
    """(normalised, its size, 1/deviation)"""
    if kind == "none":
        return v, size, torch.ones_like(v[:, :1])
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
        size = size + size.mean(1, keepdim=True)
    r = 1.0 / torch.sqrt((v * v).mean(1, keepdim=True) + eps)
    # the deviation's own relative error: that of the squares, at most size r each
    rel = (v.abs() * size).mean(1, keepdim=True) * r * r
    return v * r, size * r + v.abs() * r * (1.0 + rel), r


def spread(v, rows, per):
    return None if v is None else v.repeat_interleave(per, 0)[:rows]


class NormGate:
    """z = post(y), h = rs x + g z, n = pre(h)(1 + s) + t and its gradients."""

    def __init__(self, x, y=None, post=("none", 0.0, None, None), pre=("none", 0.0, None, None), gate=None, scale=None,
                 shift=None, per=None, rs=1.0):
        self.rows, self.C = x.shape
        self.per = per or max(self.rows, 1)
        self.n_mod = -(-self.rows // self.per)
        one, zero = torch.ones(1, self.C, dtype=torch.float64), torch.zeros(1, self.C, dtype=torch.float64)

        def vec(v, other):
            return other if v is None else d(v).reshape(-1, self.C)

        self.g, self.s, self.t = (one if v is None and i == 0 else zero if v is None else
                                  spread(vec(v, None), self.rows, self.per) for i, v in enumerate((gate, scale, shift)))
        self.rs, self.post, self.pre = rs, post, pre
        self.pw, self.pb = vec(post[2], one), vec(post[3], zero)
        self.w, self.b = vec(pre[2], one), vec(pre[3], zero)
        x = d(x)
        self.has_y = y is not None
        self.h, self.h_size = x, x.abs()
        if self.has_y:
            y = d(y)
            self.v, self.v_size, self.ry = norm(y, y.abs(), post[0], post[1])
            self.z = self.v * self.pw + self.pb
            self.z_size = self.v_size * self.pw.abs() + self.pb.abs()
            self.h = rs * x + self.g * self.z
            self.h_size = abs(rs) * x.abs() + self.g.abs() * self.z_size
        self.u, self.u_size, self.r = norm(self.h, self.h_size, pre[0], pre[1])
        self.a = self.u * self.w + self.b
        self.a_size = self.u_size * self.w.abs() + self.b.abs()
        self.n = self.a * (1.0 + self.s) + self.t
        self.n_size = self.a_size * (1.0 + self.s.abs()) + self.t.abs()

    def _back(self, dv, dv_size, u, u_size, r, kind):
        if kind == "none":
            return dv, dv_size
        o = dv - u * (dv * u).mean(1, keepdim=True)
        z = dv_size + u_size * (dv_size * u_size).mean(1, keepdim=True) * 3.0
        if kind == "layer":
            o = o - dv.mean(1, keepdim=True)
            z = z + dv_size.mean(1, keepdim=True)
        rel = (u.abs() * u_size).mean(1, keepdim=True)     # (of r)
        return o * r, z * r * (1.0 + rel)

    def _groups(self, v):
        pad = self.n_mod * self.per - self.rows
        v = torch.cat([v, torch.zeros(pad, self.C, dtype=v.dtype)]) if pad else v
        return v.view(self.n_mod, self.per, self.C).sum(1)

    def grads(self, dh=None, dn=None):
        """{name: (value, size)}"""
        zero = torch.zeros(self.rows, self.C, dtype=torch.float64)
        dh, dn = zero if dh is None else d(dh), zero if dn is None else d(dn)
        out = {"scale": (self._groups(dn * self.a), self._groups(dn.abs() * self.a_size)),
               "shift": (self._groups(dn), self._groups(dn.abs()))}
        da, da_size = dn * (1.0 + self.s), dn.abs() * (1.0 + self.s.abs())
        out["pre_w"] = ((da * self.u).sum(0), (da_size * self.u_size).sum(0))
        out["pre_b"] = (da.sum(0), da_size.sum(0))
        H, H_size = self._back(da * self.w, da_size * self.w.abs(), self.u, self.u_size, self.r, self.pre[0])
        H, H_size = H + dh, H_size + dh.abs()
        out["dx"] = (self.rs * H, abs(self.rs) * H_size)
        if self.has_y:
            out["gate"] = (self._groups(H * self.z), self._groups(H_size * self.z_size))
            dz, dz_size = H * self.g, H_size * self.g.abs()
            out["post_w"] = ((dz * self.v).sum(0), (dz_size * self.v_size).sum(0))
            out["post_b"] = (dz.sum(0), dz_size.sum(0))
            out["dy"] = self._back(dz * self.pw, dz_size * self.pw.abs(), self.v, self.v_size, self.ry, self.post[0])
        return out


def rope_pairs(dims, layout, shared):
    """[(first channel, second channel, axis, exponent of 1 / theta)]"""
    out, start, P = [], 0, sum(dims) // 2
    for a, n in enumerate(dims):
        for i in range(n // 2):
            p = start // 2 + i
            ab = {"pairs": (2 * p, 2 * p + 1), "halves": (start + i, start + n // 2 + i), "split": (p, p + P)}[layout]
            out.append((*ab, a, p / P if shared else 2 * i / n))
        start += n
    return out


def rope(v, pos, rp, inverse=False):
    """v [rows, heads, head_dim] turned by positions [rows, 3] under an
    oc.Rope: (value, size)."""
    v, pos = d(v), d(pos)
    o, z = v.clone(), v.abs()
    for a, b, axis, e in rope_pairs(rp.dims, rp.layout, rp.shared):
        ang = ((pos[:, axis] + rp.origin[axis]) * rp.scale[axis] * rp.theta ** -e)[:, None]
        c, s = ang.cos(), -ang.sin() if inverse else ang.sin()
        o[..., a], o[..., b] = v[..., a] * c - v[..., b] * s, v[..., a] * s + v[..., b] * c
        z[..., a] = z[..., b] = v[..., a].abs() + v[..., b].abs()
    return o, z


def grid_pos(tokens, H, W):
    t = d(tokens).long()
    return torch.stack([t // (H * W), t % (H * W) // W, t % (H * W) % W], 1).double()


def check(got, ref, size, roundings, what):
    """|got - ref| <= the output's own rounding + roundings 2^-24 size."""
    got = got.detach().cpu()
    tol = half_step(got.dtype) * ref.abs() * 1.01 + roundings * U32 * size + 1e-40
    err = (got.double() - ref).abs()
    bad = ~(err <= tol)
    assert not bad.any(), (what, int(bad.sum()), float((err / tol).nan_to_num(1e30).max()),
                           got[bad][:4].tolist(), ref[bad][:4].tolist())


def quant(x):
    """(whole numbers, scales) of rows in 64 bits: the quotient 127 x / max|x|
    as a fraction of whole numbers would round it (doubles keep it apart from
    every tie that it is not: the values have at most 24 bits)."""
    x = d(x)
    top = x.abs().amax(1, keepdim=True)
    q = torch.where(top > 0, x * 127.0 / torch.where(top > 0, top, torch.ones_like(top)), torch.zeros_like(x))
    return q.round(), (top[:, 0].float() / 127.0)


def gelu(v):
    return 0.5 * v * (1.0 + torch.tanh((2.0 / torch.pi) ** 0.5 * (v + 0.044715 * v ** 3)))


def linear_i8(q, s, w, ws, bias=None, act="none"):
    """(value, size) of the product of quantised rows."""
    acc = d(q).float().double() @ d(w).t()
    v = acc * d(s)[:, None] * d(ws)
    size = v.abs()
    if bias is not None:
        v, size = v + d(bias), size + d(bias).abs()
    if act == "gelu":
        # |gelu'| <= 1.13; beside that the factor's own evaluation, whose exponent
        # 2 sqrt(2/pi) (v + 0.044715 v^3) is off by a few roundings of itself (it counts where the
        # factor is neither 0 nor 1: |v| below 8, an exponent below 50)
        size = 1.13 * size + v.abs() * 50.0
        v = gelu(v)
    return v, size
