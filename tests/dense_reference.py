"""The dense operators' definitions in 64 bits on the CPU, and how far a result in fp32 arithmetic may be from them.

Every bound follows from the arithmetic: U is fp32's rounding unit, UT the output type's; a sum of n terms in any order is within
depth * U * sum |terms|, with the depth of the order that is used or n; the matrix instructions' accumulation is allowed
2 U a term, since it may truncate."""
import math

import torch

U = 2.0 ** -24
UT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}      # half the smallest step
SILU, GELU, RELU = 0, 1, 2


def rounding(y, dtype):
    """Of one rounding to dtype, of values near y."""
    return y.abs() * UT[dtype] * 1.01 + TINY[dtype]


def act(g, kind):
    if kind == SILU:
        return g * torch.sigmoid(g)
    if kind == GELU:
        return 0.5 * g * torch.special.erfc(-g / math.sqrt(2.0))
    return g.clamp(min=0.0)


def slope(g, kind):
    if kind == SILU:
        s = torch.sigmoid(g)
        return s + g * s * torch.sigmoid(-g)
    if kind == GELU:
        return 0.5 * torch.special.erfc(-g / math.sqrt(2.0)) + g * torch.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)
    return (g > 0).double()


def quantize(x):
    """(q, scale) by the definition, each of its fp32 operations rounded as fp32 rounds."""
    x = x.float().cpu()
    top = x.abs().amax(1) if x.shape[0] else x.new_zeros(0)
    bad = ~torch.isfinite(x).all(1)
    none = ~bad & (top < 2.0 ** -100)
    most = torch.full_like(top, 127.0)          # (torch divides by or into a number through its reciprocal)
    to, scale = most / top, top / most
    q = torch.round(x * to[:, None])
    q[bad | none] = 0.0
    scale[none], scale[bad] = 0.0, float("nan")
    return q.to(torch.int8), scale


def int8_product(a, b):
    return a.cpu().double() @ b.cpu().double().t()       # exact: below 2^53


def int8_matmul(a, sa, b, sb, bias, dtype):
    """(out, bound)"""
    y = int8_product(a, b) * (sa.cpu().double()[:, None] * sb.cpu().double()[None])
    out = y if bias is None else y + bias.cpu().double()[None]
    # the sum's conversion, the scales' product and theirs: three roundings; the addition's one
    return out, y.abs() * 3.1 * U + out.abs() * U + rounding(out, dtype)


def norm(x, gamma, beta, eps, dtype):
    """(y, mean, rstd) and the bounds of the three; dtype None: y not rounded at the end."""
    x = x.cpu().double()
    n = x.shape[1]
    g = torch.ones(n).double() if gamma is None else gamma.cpu().double()
    b = torch.zeros(n).double() if beta is None else beta.cpu().double()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    var = d.square().mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(var + eps)
    y = d * rstd * g + b
    depth = n / 64 + 64          # of a thread's chain, a wave's tree and a workgroup's
    e_mean = (depth + 1) * U * x.abs().mean(1, keepdim=True)
    # the mean's error moves every difference and adds its square to the variance; a difference's rounding counts twice in its square
    e_rstd = rstd * (0.5 * (depth + 4) * U + 0.5 * e_mean.square() * rstd.square() + 3 * U)
    e_y = g.abs() * (rstd * (e_mean + d.abs() * U) + d.abs() * e_rstd) * 1.01 + 3 * U * (y.abs() + b.abs())
    if dtype is not None:
        e_y = e_y + rounding(y, dtype)
    return (y, mean[:, 0], rstd[:, 0]), (e_y, e_mean[:, 0] + 1e-45, e_rstd[:, 0])


def norm_back(dy, x, gamma, mean, rstd, dtype, p_dtype):
    """(dx, dgamma, dbeta) and their bounds."""
    dy, x = dy.cpu().double(), x.cpu().double()
    rows, n = x.shape
    g = torch.ones(n).double() if gamma is None else gamma.cpu().double()
    m, r = mean.cpu().double()[:, None], rstd.cpu().double()[:, None]
    xh, p = (x - m) * r, dy * g
    s1, s2 = p.mean(1, keepdim=True), (p * xh).mean(1, keepdim=True)
    dx = r * (p - s1 - xh * s2)
    depth = n / 64 + 72
    e = r * (4 * U * p.abs() + depth * U * p.abs().mean(1, keepdim=True) + xh.abs() * depth * U * (p * xh).abs().mean(1, keepdim=True)
             + 8 * U * (xh * s2).abs() + 4 * U * s1.abs()) * 1.01
    dg, db = (dy * xh).sum(0), dy.sum(0)
    down = rows / 32 + 128
    e_g = (down + 4) * U * (dy * xh).abs().sum(0)
    e_b = down * U * dy.abs().sum(0)
    return (dx, dg, db), (e + rounding(dx, dtype), e_g + rounding(dg, p_dtype), e_b + rounding(db, p_dtype))


def _gate(g, u, e_g, e_u, kind):
    """act(g) u and its bound but for the final rounding.  The slopes of all three are below 1.13; act in fp32 is within 8 roundings of |g|."""
    h = act(g, kind) * u
    return h, (u.abs() + e_u) * (1.13 * e_g + 8 * U * g.abs()) + act(g, kind).abs() * e_u + 2 * U * h.abs()


def gated(x, wg, wu, kind, dtype):
    """(h, g, u) and their bounds."""
    x, wg, wu = (t.cpu().double() for t in (x, wg, wu))
    g, u = x @ wg.t(), x @ wu.t()
    k = x.shape[1]
    e_g, e_u = 2 * k * U * (x.abs() @ wg.abs().t()), 2 * k * U * (x.abs() @ wu.abs().t())
    h, e_h = _gate(g, u, e_g, e_u, kind)
    return (h, g, u), (e_h + rounding(h, dtype), e_g + rounding(g, dtype), e_u + rounding(u, dtype))


def int8_gated(a, sa, wg, sg, wu, su, kind, dtype):
    g = int8_product(a, wg) * (sa.cpu().double()[:, None] * sg.cpu().double()[None])
    u = int8_product(a, wu) * (sa.cpu().double()[:, None] * su.cpu().double()[None])
    h, e = _gate(g, u, 3.1 * U * g.abs(), 3.1 * U * u.abs(), kind)
    return h, e + rounding(h, dtype)


def gated_back(dh, x, wg, wu, g, u, kind, dtype):
    """(dx, dwg, dwu) and their bounds: dg and du are rounded to the block's type before the products."""
    dh, x, wg, wu, g, u = (t.cpu().double() for t in (dh, x, wg, wu, g, u))
    dg, du = dh * u * slope(g, kind), dh * act(g, kind)
    # fp32: the slope within 16 roundings of 1 + |g|, then two products; then the type's rounding
    e_dg = 16 * U * (dh * u).abs() * (1 + g.abs()) + rounding(dg, dtype)
    e_du = 12 * U * (dh * g).abs() + rounding(du, dtype)
    dx, dwg, dwu = dg @ wg + du @ wu, dg.t() @ x, du.t() @ x
    m, f = dg.shape
    e_dx = e_dg @ wg.abs() + e_du @ wu.abs() + 4 * f * U * (dg.abs() @ wg.abs() + du.abs() @ wu.abs()) * 1.01
    e_wg = e_dg.t() @ x.abs() + 2 * m * U * (dg.abs().t() @ x.abs()) * 1.01
    e_wu = e_du.t() @ x.abs() + 2 * m * U * (du.abs().t() @ x.abs()) * 1.01
    return (dx, dwg, dwu), (e_dx + rounding(dx, dtype), e_wg + rounding(dwg, dtype), e_wu + rounding(dwu, dtype))


def assert_within(got, want, bound, what):
    got = got.cpu().double()
    assert got.shape == want.shape, what
    assert torch.isfinite(got).all(), f"{what}: not finite"
    off = (got - want).abs() - bound
    assert not (off > 0).any(), f"{what}: {int((off > 0).sum())} of {off.numel()} out of bounds, worst by {float(off.max())}"
