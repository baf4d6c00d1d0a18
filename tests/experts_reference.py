"""Definitions in 64 bits on the CPU of routing and of the products with 4-bit weights, and how far a result in fp32 arithmetic may be from them
(dense_reference says how the bounds are formed)."""
import math

import torch

from dense_reference import U, _gate, rounding

SOFTMAX, SIGMOID = 0, 1


def levels_of(q, cols):
    """uint8 [..][rows][cols] from rows of words: value 2 j of eight in bits 4 j, value 2 j + 1 in bits 16 + 4 j."""
    words = q.cpu().contiguous().view(torch.int32).long()
    out = torch.empty(*words.shape[:-1], words.shape[-1] * 8, dtype=torch.uint8)
    for v in range(8):
        out[..., v::8] = (words >> (4 * (v // 2) + 16 * (v % 2)) & 15).to(torch.uint8)
    return out[..., :cols]


def quantize(w, group, zeros, scale_dtype):
    """(levels, scale, zero) by the definition, each of its fp32 operations rounded as fp32 rounds."""
    w = w.float().cpu()
    rows, cols = w.shape
    groups = (cols + group - 1) // group
    part = torch.nn.functional.pad(w, (0, groups * group - cols)).view(rows, groups, group)
    bad = ~torch.isfinite(part).all(2)
    low, high = part.amin(2).clamp(max=0.0), part.amax(2).clamp(min=0.0)
    span, most = (high - low, 15.0) if zeros else (torch.maximum(-low, high), 7.0)
    scale = (span / torch.full_like(span, most)).to(scale_dtype)
    scale[bad | ~torch.isfinite(scale)] = float("nan")
    s = scale.float()
    none = ~(s > 0)
    zero = torch.full_like(s, 8.0)
    if zeros:
        zero = torch.where(none, zero, torch.round(-low / s).clamp(0, 15))
    level = torch.where(none[..., None], zero[..., None].expand_as(part), (torch.round(part / s[..., None]) + zero[..., None]).clamp(0, 15))
    level = level.nan_to_num(0.0).to(torch.uint8).view(rows, -1)[:, :cols]
    return level, scale.t().contiguous(), zero.t().to(torch.uint8).contiguous() if zeros else None


def values(w):
    """A matrix's values, its scales and its zero points by row and column, in 64 bits."""
    by_column = lambda t: t.cpu().double().repeat_interleave(w.group, 0)[:w.cols].t()      # noqa: E731
    s = by_column(w.scale)
    z = torch.full_like(s, 8.0) if w.zero is None else by_column(w.zero)
    return (levels_of(w.q, w.cols).double() - z) * s, s, z


def product(x, e_x, w, dtype):
    """x w^T and its bound but for the output's rounding.  e_x: x's own."""
    v, s, z = values(w)
    x = x.cpu().double()
    y = x @ v.t()
    n = x.shape[1]
    a = x.abs() + e_x
    # a group's sum: of levels less zeros, or (bf16) of 16 + level and -(16 + zero), whose sums twice as many terms form; then the groups' sums (of at
    # least 32 values) with their scales after one another, at most 16 shares of them and 8 waves', a scale's product and the last addition
    most = (v.abs() if dtype is torch.float16 else (levels_of(w.q, w.cols).double() + z + 32.0) * s.abs())
    depth = 2 * (1 if dtype is torch.float16 else 2) * min(n, w.group) + n / 32 + 32
    return y, depth * U * (a @ most.t()) + e_x @ v.abs().t()


def linear(x, w, bias, out_dtype):
    y, e = product(x, torch.zeros(x.shape).double(), w, x.dtype)
    if bias is not None:
        y = y + bias.cpu().double()
    return y, e + U * y.abs() + rounding(y, out_dtype)


def gated(x, wg, wu, act, out_dtype):
    none = torch.zeros(x.shape).double()
    g, e_g = product(x, none, wg, x.dtype)
    u, e_u = product(x, none, wu, x.dtype)
    h, e = _gate(g, u, e_g, e_u, act)
    return h, e + rounding(h, out_dtype)


def one(w, e):
    return type(w)(w.q[e], w.scale[e], None if w.zero is None else w.zero[e], w.cols, w.group)


def experts(x, chosen, weights, wg, wu, wd, act, out_dtype):
    T, k = chosen.shape
    E, N = wd.q.shape[0], wd.rows
    y, e_y = torch.zeros(T, N).double(), torch.zeros(T, N).double()
    weights = weights.cpu().double()
    for e in range(E):
        for s in range(k):
            rows = (chosen[:, s].cpu() == e).nonzero()[:, 0]
            if rows.numel() == 0:
                continue
            h, e_h = gated(x[rows.to(x.device)], one(wg, e), one(wu, e), act, x.dtype)
            p, e_p = product(h, e_h, one(wd, e), x.dtype)
            w = weights[rows, s, None]
            y[rows] += w * p
            e_y[rows] += w.abs() * (e_p + (k + 2) * U * (p.abs() + e_p))
    return y, e_y + rounding(y, out_dtype)


def route(logits, k, bias=None, score=SOFTMAX, groups=1, kept=1, top=1, renorm=True, factor=1.0):
    """(experts, weights) of each token, one after the other, by the definition."""
    logits = logits.cpu().double()
    T, E = logits.shape
    chosen, weights = torch.full((T, k), -1, dtype=torch.int32), torch.zeros(T, k).double()
    b = torch.zeros(E).double() if bias is None else bias.cpu().double()
    for t in range(T):
        row = logits[t]
        if torch.isnan(row).any() or (score == SOFTMAX and (row == math.inf).any()):
            weights[t] = math.nan
            continue
        if (row == -math.inf).all():
            continue
        p = torch.softmax(row, 0) if score == SOFTMAX else torch.sigmoid(row)
        c = (p + b).tolist()
        open_ = [e for e in range(E) if row[e] > -math.inf and c[e] > -math.inf]
        if groups > 1:
            size = E // groups
            of = []
            for g in range(groups):
                mine = sorted((c[e] for e in open_ if e // size == g), reverse=True)[:top]
                of.append(sum(mine) if mine else -math.inf)
            stay = sorted(range(groups), key=lambda g: (-of[g], g))[:kept]
            open_ = [e for e in open_ if e // size in stay]
        best = sorted(open_, key=lambda e: (-c[e], e))[:k]
        w = p[best]
        if renorm:
            w = w / w.sum() if w.sum() > 0 else torch.zeros_like(w)
        chosen[t, :len(best)] = torch.tensor(best, dtype=torch.int32)
        weights[t, :len(best)] = w * factor
    return chosen, weights


def lists(chosen, E):
    flat = chosen.reshape(-1).tolist()
    of = [[] for _ in range(E)]
    for i, e in enumerate(flat):
        if 0 <= e < E:
            of[e].append(i)
    offsets, order = [0], []
    for mine in of:
        order += mine
        offsets.append(len(order))
    return torch.tensor(offsets, dtype=torch.int32), torch.tensor(order + [-1] * (len(flat) - len(order)), dtype=torch.int32)


def weights_of(logits, chosen, score, renorm, factor):
    """The weights of the experts chosen as a function of the logits, for differentiation: slots without one are 0."""
    E = logits.shape[1]
    p = torch.softmax(logits, 1) if score == SOFTMAX else torch.sigmoid(logits)
    there = (chosen >= 0) & (chosen < E)
    w = torch.where(there, p.gather(1, chosen.long().clamp(0, E - 1)), torch.zeros(()).double())
    if renorm:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / torch.where(total > 0, total, 1.0), torch.zeros(()).double())
    return w * factor


def route_back(dweights, logits, chosen, score, renorm, factor, dtype):
    """(dlogits, bound) by the definition."""
    l, d, chosen = logits.cpu().double(), dweights.cpu().double() * factor, chosen.cpu()
    E = l.shape[1]
    there = (chosen >= 0) & (chosen < E)
    at = chosen.long().clamp(0, E - 1)
    p = torch.softmax(l, 1) if score == SOFTMAX else torch.sigmoid(l)
    none = torch.zeros(()).double()
    w = torch.where(there, p.gather(1, at), none)
    d = torch.where(there, d, none)
    dense = score == SOFTMAX and not renorm
    if renorm:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
    dot = (d * w).sum(1, keepdim=True) if renorm or dense else 0.0 * d[:, :1]
    reach = (d.abs() * w).sum(1, keepdim=True) if renorm or dense else dot
    # a score's relative error: its exponent's argument is rounded, the exponential within 2 units, sums of 16 terms a lane and 6 steps, a division
    finite = l.masked_fill(~torch.isfinite(l), 0.0)
    rel = (64.0 + 4.0 * finite.abs().amax(1, keepdim=True)) * U
    if dense:
        e = torch.zeros_like(l).scatter_add_(1, at, d)
        size = torch.zeros_like(l).scatter_add_(1, at, d.abs())
        dl, bound = p * (e - dot), rel * p * (size + reach)
    else:
        rest = 1.0 - torch.sigmoid(l.gather(1, at)) if score == SIGMOID else torch.ones_like(w)
        dl = torch.zeros_like(l).scatter_add_(1, at, torch.where(there, w * (d - dot) * rest, none))
        bound = torch.zeros_like(l).scatter_add_(1, at, torch.where(there, rel * w * (d.abs() + reach) * rest, none))
    return dl, bound + 2.0 ** -149 + rounding(dl, dtype)
