"""The operators of paper_2103_07454_amd.nn in 64 bits on the CPU, with bounds of what 32-bit kernels may be off.

Forward values and gradients are written out from the formulas (not taken from automatic differentiation); each comes with an
elementwise bound derived from the rounding errors of a computation that holds sums in 32 bits: n terms summed in any order are off
by at most n * 2^-24 times the sum of their magnitudes, a rounding to p bits by 2^-p of the value (and half the smallest
subnormal), a library function by 8 units of 2^-24.
"""
import math

import torch

U32 = 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
#: Half the spacing of the subnormals.
TINY = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
FUNCTION = 8 * U32


def rounding(x, dtype):
    return UNIT[dtype] * x.abs() + TINY[dtype]


def act(kind, g):
    """Activation, slope and curvature bound (of the slope's change with g)."""
    if kind == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    if kind == "gelu":
        cdf = 0.5 * torch.erfc(-g / math.sqrt(2))
        return g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        th = torch.tanh(c * (g + 0.044715 * g ** 3))
        return 0.5 * g * (1 + th), 0.5 * (1 + th) + 0.5 * g * (1 - th * th) * c * (1 + 3 * 0.044715 * g * g)
    return g.clamp(min=0), (g > 0).double()


def ffn(kind, dtype, x, wg, wu, wd, dy=None):
    """{name: (value, bound)} of one worker's block; all arguments in 64 bits."""
    T, D = x.shape
    F = wg.shape[0]
    m = lambda a, b: a @ b
    g, u = m(x, wg.t()), m(x, wu.t())
    eg, eu = D * U32 * m(x.abs(), wg.t().abs()), D * U32 * m(x.abs(), wu.t().abs())
    a, s = act(kind, g)
    # |act'| and |act''| of all four stay below 1.2; ReLU's slope jumps where g's sign is not certain
    ea = 1.2 * eg + FUNCTION * (g.abs() + a.abs())
    es = 1.2 * eg + FUNCTION * (1 + g.abs() * 2) if kind != "relu" else (g.abs() <= eg).double()
    h = a * u
    eh = ea * u.abs() + a.abs() * eu + ea * eu + 2 * U32 * h.abs()
    eh = eh + rounding(h.abs() + eh, dtype)
    y = m(h, wd.t())
    ey = m(eh, wd.t().abs()) + F * U32 * m(h.abs() + eh, wd.t().abs())
    out = dict(y=(y, ey + rounding(y.abs() + ey, dtype)))
    if dy is not None:
        dh = m(dy, wd)
        edh = D * U32 * m(dy.abs(), wd.abs())

        def product(*terms):
            """A product of (value, error) pairs, and its rounding to the type."""
            v, lo, hi = 1.0, 1.0, 1.0
            for t, e in terms:
                v, lo, hi = v * t, lo * t.abs(), hi * (t.abs() + e)
            e = hi - lo + 4 * U32 * hi
            return v, e + rounding(v.abs() + e, dtype)

        dg, edg = product((dh, edh), (u, eu), (s, es))
        du, edu = product((dh, edh), (a, ea))
        for name, pairs, n in (("dx", ((dg, edg, wg), (du, edu, wu)), 2 * F), ("dw_gate", ((dg.t(), edg.t(), x),), T),
                               ("dw_up", ((du.t(), edu.t(), x),), T), ("dw_down", ((dy.t(), None, h),), T)):
            v = e = 0.0
            for p, ep, q in pairs:
                v = v + m(p, q)
                if ep is None:
                    e = e + m(p.abs(), eh) + n * U32 * m(p.abs(), q.abs() + eh)
                else:
                    e = e + m(ep, q.abs()) + n * U32 * m(p.abs() + ep, q.abs())
            out[name] = (v, e + rounding(v.abs() + e, dtype))
    return out


def unit(kind, z, eps):
    if kind == "layer":
        z = z - z.mean(-1, keepdim=True)
    inv = 1 / torch.sqrt((z * z).mean(-1, keepdim=True) + eps)
    return z * inv, inv


def unit_gradient(kind, d, u, inv):
    r = d - u * (d * u).mean(-1, keepdim=True)
    if kind == "layer":
        r = r - d.mean(-1, keepdim=True)
    return r * inv


def blocknorm(kind, t, *, eps, alpha, beta, gate_rows):
    """Values of one worker's norms from `t`, tensors by name in 64 bits (absent ones left out); gradients where it has d_out or
    d_normed.  Second, the magnitudes that errors scale with: the same expressions with every term's magnitude, before any cancel."""
    r = alpha * t["residual"]
    rows = r.shape[0]
    out, size = {}, {}
    size_r = r.abs()
    ub = inv_b = None
    after = t.get("branch")
    if after is not None:
        if "post" in t:
            ub, inv_b = unit(kind, after, eps)
            after = ub * t["post"] + t.get("post_bias", 0.0)
        gate = t["gate"][torch.arange(rows) // gate_rows] if "gate" in t else torch.ones_like(after)
        size_after = after.abs() if "post" not in t else ub.abs() * t["post"].abs() + abs(t.get("post_bias", torch.zeros(())))
        size_r = size_r + abs(beta) * gate.abs() * size_after
        r = r + beta * gate * after
    out["residual"], size["residual"] = r, size_r
    ur = None
    if "pre" in t:
        ur, inv_r = unit(kind, r, eps)
        out["normed"] = ur * t["pre"] + t.get("pre_bias", 0.0)
        # r' itself is off by its magnitude's share, and so is its mean
        unit_size = (size_r + size_r.mean(-1, keepdim=True)) * inv_r
        size["normed"] = (unit_size + ur.abs()) * t["pre"].abs() + abs(t.get("pre_bias", torch.zeros(())))
    if "d_out" not in t and "d_normed" not in t:
        return out, size

    def gradient_size(d, u, inv, u_size):
        return inv * (d + d.mean(-1, keepdim=True) + u_size * (d * u_size).mean(-1, keepdim=True))

    dr = t.get("d_out", torch.zeros_like(r))
    size_dr = dr.abs()
    if "pre" in t:
        dn = t.get("d_normed", torch.zeros_like(r))
        out["d_pre"], size["d_pre"] = (dn * ur).sum(0), (dn.abs() * unit_size).square().sum(0).sqrt()
        if "pre_bias" in t:
            out["d_pre_bias"], size["d_pre_bias"] = dn.sum(0), dn.square().sum(0).sqrt()
        dr = dr + unit_gradient(kind, dn * t["pre"], ur, inv_r)
        size_dr = size_dr + gradient_size((dn * t["pre"]).abs(), ur, inv_r, unit_size)
    out["d_residual"], size["d_residual"] = alpha * dr, abs(alpha) * size_dr
    if after is not None:
        if "gate" in t:
            which = torch.arange(rows) // gate_rows
            out["d_gate"] = torch.zeros_like(t["gate"]).index_add_(0, which, beta * dr * after)
            size["d_gate"] = torch.zeros_like(t["gate"]).index_add_(0, which, (beta * size_dr * size_after).square()).sqrt()
        da = beta * gate * dr
        size_da = abs(beta) * gate.abs() * size_dr
        if "post" in t:
            b = t["branch"].abs()
            ub_size = (b + b.mean(-1, keepdim=True)) * inv_b
            out["d_post"], size["d_post"] = (da * ub).sum(0), (size_da * ub_size).square().sum(0).sqrt()
            if "post_bias" in t:
                out["d_post_bias"], size["d_post_bias"] = da.sum(0), size_da.square().sum(0).sqrt()
            da = unit_gradient(kind, da * t["post"], ub, inv_b)
            size_da = gradient_size(size_da * t["post"].abs(), ub, inv_b, ub_size)
        out["d_branch"], size["d_branch"] = da, size_da
    return out, size
