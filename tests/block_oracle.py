"""The block operators (include/rk_block.h) from their definitions in 64 bits, on the CPU, with
the error bounds that their 32-bit sums and one rounding of each output allow.

Every function returns 64-bit tensors.  A bound is the largest error an output may have: half a
unit in the last place of its type, and for a 32-bit sum of n terms (n + a few) * 2^-24 times
the sum of the terms' absolute values.
"""
import math

import torch

GROUP = 32
U32 = 2.0 ** -24
# unit roundoff, smallest subnormal / 2, largest finite value
ROUND = {torch.float32: (2.0 ** -24, 2.0 ** -150), torch.float16: (2.0 ** -11, 2.0 ** -25),
         torch.bfloat16: (2.0 ** -8, 2.0 ** -134)}


def rounding(ref, dtype):
    u, tiny = ROUND[dtype]
    return ref.abs() * u + tiny


def d(t):
    return t.detach().cpu().double()


def layer_norm(x, w, b, eps):
    mean = x.mean(1, keepdim=True)
    var = ((x - mean) ** 2).mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    xh = (x - mean) * rstd
    w = torch.ones(x.shape[1], dtype=torch.float64) if w is None else w
    b = torch.zeros(x.shape[1], dtype=torch.float64) if b is None else b
    return xh * w + b, mean[:, 0], rstd[:, 0]


def layer_norm_grads(dy, x, mean, rstd, w):
    xh = (x - mean[:, None]) * rstd[:, None]
    v = dy if w is None else dy * w
    dx = rstd[:, None] * (v - v.mean(1, keepdim=True) - xh * (v * xh).mean(1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def ckpt_step(x):
    """[rows, groups]: the exponent e of each group's step, by counting up from the smallest."""
    rows, cols = x.shape
    pad = torch.zeros(rows, -cols % GROUP, dtype=torch.float64)
    top = torch.cat([x, pad], 1).view(rows, -1, GROUP).abs().amax(2)
    e = torch.full_like(top, -126.0)
    while True:
        more = (top > 127 * torch.exp2(e)) & (e < 122)
        if not more.any():
            return e
        e = torch.where(more, e + 1, e)


def ckpt(x, dtype):
    """(codes [rows, cols], e [rows, groups], values [rows, cols]) of the checkpoint of x (finite), x of type dtype."""
    rows, cols = x.shape
    e = ckpt_step(x)
    wide = e.repeat_interleave(GROUP, 1)[:, :cols]
    step = torch.exp2(wide)
    limit = torch.where(64 * step > torch.finfo(dtype).max, 63.0, 127.0).double()
    q = torch.round(x / step)  # ties to even
    q = torch.minimum(torch.maximum(q, -limit), limit)
    return q, e, q * step


def act(g, kind):
    """(act(g), act'(g))"""
    if kind == "silu":
        s = torch.sigmoid(g)
        return g * s, s + g * s * (1 - s)
    below = 0.5 * torch.erfc(-g / math.sqrt(2))
    return g * below, below + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def act_error(g, kind):
    """Relative error of the 32-bit act and act' terms at g: e^t and erfc(t) turn an error of t's rounding
    into one of |t| (t^2) times as much; a few roundings besides."""
    return (g.abs() + 16) * 4 * U32 if kind == "silu" else (g * g + 16) * 4 * U32


def gated(x, wg, wu, kind):
    g, u = x @ wg.t(), x @ wu.t()
    return act(g, kind)[0] * u, g, u


def gated_grads(dh, x, wg, wu, kind, g, u):
    """(dx, dwg, dwu, h) with g and u given."""
    a, s = act(g, kind)
    dg, du = dh * u * s, dh * a
    return dg @ wg + du @ wu, dg.t() @ x, du.t() @ x, a * u


# bounds ------------------------------------------------------------------------------------

def sum_bound(terms_abs_sum, n):
    return (n + 8) * U32 * terms_abs_sum


def layer_norm_bounds(x, w, b, eps, dtype):
    """Bounds of y, mean and rstd."""
    n = x.shape[1]
    y, mean, rstd = layer_norm(x, w, b, eps)
    m_err = sum_bound(x.abs().mean(1), n)
    xc = x - mean[:, None]
    # variance: (x - m)^2 with m off by m_err (second order in the mean), 32-bit squares and sum
    var = (xc ** 2).mean(1)
    v_err = sum_bound(var, n) + m_err ** 2 + 4 * U32 * (xc.abs() * x.abs().amax(1, keepdim=True)).mean(1)
    r_err = rstd ** 3 * 0.5 * v_err * 1.5 + 4 * U32 * rstd
    w = torch.ones(n, dtype=torch.float64) if w is None else w
    bb = torch.zeros(n, dtype=torch.float64) if b is None else b
    y_err = w.abs() * (rstd[:, None] * (m_err[:, None] + U32 * x.abs()) + xc.abs() * r_err[:, None]) \
        + 4 * U32 * (w * xc * rstd[:, None]).abs() + 2 * U32 * (y.abs() + bb.abs())
    return y_err + rounding(y, dtype), m_err + U32 * mean.abs() + 1e-45, r_err


def layer_norm_grad_bounds(dy, x, mean, rstd, w, dtype, wdtype):
    """Bounds of dx, dw and db, with mean and rstd as given."""
    rows, n = x.shape
    dx, dw, db = layer_norm_grads(dy, x, mean, rstd, w)
    xh = (x - mean[:, None]) * rstd[:, None]
    e_xh = 4 * U32 * (xh.abs() + (mean * rstd).abs()[:, None])
    v = dy if w is None else dy * w
    e_s = sum_bound((v * xh).abs().mean(1, keepdim=True), n) + (v.abs() * e_xh).mean(1, keepdim=True)
    e = sum_bound(v.abs().mean(1, keepdim=True), n) + xh.abs() * e_s + e_xh * (v * xh).mean(1, keepdim=True).abs()
    e = rstd[:, None].abs() * (e + 4 * U32 * (v.abs() + v.mean(1, keepdim=True).abs()
                                              + (xh * (v * xh).mean(1, keepdim=True)).abs()))
    e_dw = sum_bound((dy * xh).abs().sum(0), rows) + (dy.abs() * e_xh).sum(0)
    return (e + rounding(dx, dtype), e_dw + rounding(dw, wdtype), sum_bound(dy.abs().sum(0), rows) + rounding(db, wdtype))


def gated_bounds(x, wg, wu, kind, dtype):
    """Bounds of h, g and u before their rounding (g and u in 32 bits), and h rounded."""
    n = x.shape[1]
    h, g, u = gated(x, wg, wu, kind)
    eg, eu = sum_bound(x.abs() @ wg.abs().t(), n), sum_bound(x.abs() @ wu.abs().t(), n)
    a, s = act(g, kind)
    # |act'| <= 1.13, and so is its slope's effect over eg
    e = 1.2 * eg * (u.abs() + eu) + a.abs() * eu + (a * u).abs() * act_error(g, kind)
    return e + rounding(h, dtype), eg, eu


def gated_grad_bounds(dh, x, wg, wu, kind, g, u, dtype, eg=0.0, eu=0.0, fine=False):
    """Bounds of dx, dwg, dwu and h for g and u that may be off by eg and eu (0: as given).  fine: dg and du
    enter the products in two parts, and lose the square of a rounding only."""
    ud = ROUND[dtype][0] ** (2 if fine else 1)
    dx, dwg, dwu, h = gated_grads(dh, x, wg, wu, kind, g, u)
    a, s = act(g, kind)
    ae = act_error(g, kind)
    dg, du = dh * u * s, dh * a
    # the slope's terms may cancel: bound by their absolute values (each at most about 1 + |g| / 2)
    slope_abs = 1.0 + 0.5 * g.abs()
    # |act''| <= 1
    e_dg = dh.abs() * (u.abs() * (ae * slope_abs + eg) + eu * (s.abs() + eg)) + ud * dg.abs() + ROUND[dtype][1]
    e_du = dh.abs() * (a.abs() * ae + 1.2 * eg) + ud * du.abs() + ROUND[dtype][1]
    n, rows = g.shape[1], x.shape[0]
    e_dx = e_dg @ wg.abs() + e_du @ wu.abs() + sum_bound(dg.abs() @ wg.abs() + du.abs() @ wu.abs(), 2 * n)
    e_wg = e_dg.t() @ x.abs() + sum_bound(dg.abs().t() @ x.abs(), rows)
    e_wu = e_du.t() @ x.abs() + sum_bound(du.abs().t() @ x.abs(), rows)
    e_h = 1.2 * eg * (u.abs() + eu) + a.abs() * eu + (a * u).abs() * ae
    return (e_dx * 1.01 + rounding(dx, dtype), e_wg * 1.01 + rounding(dwg, dtype), e_wu * 1.01 + rounding(dwu, dtype),
            e_h + rounding(h, dtype))


def worst(got, ref, bound):
    """Largest error over its bound (at most 1 when all is well; NaN counts as infinite)."""
    if ref.numel() == 0:
        return 0.0
    r = (d(got) - ref).abs() / bound
    return float(torch.nan_to_num(r, nan=math.inf).max())
