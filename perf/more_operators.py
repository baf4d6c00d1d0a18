"""Timed passes through routing to experts, 4-bit linear layers and the experts' gated blocks on 4-bit weights.

``listed`` names the passes, ``draw`` makes more of the same ranges, ``prepare`` makes what a program holds before the call
and ``run`` is one pass: through the library where ``own`` is set, else in elementary torch operations.  ``exact`` is the definition in
64 bits.  Operators:

    route       scores of logits, the chosen experts of each token with their weights, and the tokens of each expert as a list
    route_back  the logits' gradient from the weights'
    linear      y = x w^T with 4-bit weights, a scale (and a zero point) for each row and group of columns
    gated       act(x wg^T) * (x wu^T) on such weights
    experts     y[t] = sum over the token's experts e of weight * (act(x wg_e^T) * (x wu_e^T)) wd_e^T on such weights
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # a decoding step's one token to 8 of 64 experts: latency alone
        {"name": "route, one token", "op": "route", "tokens": 1, "experts": 64, "chosen": 8, "score": "softmax", "bias": False, "groups": 1, "kept": 1,
         "top": 1, "renorm": True, "type": "bf16"},
        # a training batch, sigmoid scores with a bias for balance, 4 of 8 groups of experts by their two best
        {"name": "route, 16384 tokens, groups", "op": "route", "tokens": 16384, "experts": 256, "chosen": 8, "score": "sigmoid", "bias": True, "groups": 8,
         "kept": 4, "top": 2, "renorm": True, "type": "fp32"},
        # gradients of a small batch, odd sizes
        {"name": "route back, odd", "op": "route_back", "tokens": 1013, "experts": 60, "chosen": 5, "score": "sigmoid", "renorm": True, "type": "f16"},
        # gradients of a training batch whose weights are the scores themselves
        {"name": "route back, 16384 tokens", "op": "route_back", "tokens": 16384, "experts": 256, "chosen": 8, "score": "softmax", "renorm": False,
         "type": "fp32"},
        # one token through a square layer: a decoding step, bound by latency and by reading the weights
        {"name": "linear, one token", "op": "linear", "tokens": 1, "inner": 4096, "outer": 4096, "group": 128, "zeros": False, "bias": False, "type": "bf16"},
        # a few requests at once through a layer of odd sizes, short groups with zero points, a bias
        {"name": "linear, 13 tokens, odd", "op": "linear", "tokens": 13, "inner": 1037, "outer": 1531, "group": 32, "zeros": True, "bias": True, "type": "f16"},
        # a long prompt through a large layer
        {"name": "linear, 4096 tokens", "op": "linear", "tokens": 4096, "inner": 8192, "outer": 8192, "group": 128, "zeros": False, "bias": False,
         "type": "bf16"},
        # the served feed-forward layer's front for one token
        {"name": "gated, one token", "op": "gated", "tokens": 1, "inner": 4096, "hidden": 8192, "group": 64, "zeros": True, "act": "silu", "type": "bf16"},
        # a short prompt, odd sizes
        {"name": "gated, 200 tokens, odd", "op": "gated", "tokens": 200, "inner": 2040, "hidden": 5001, "group": 128, "zeros": False, "act": "gelu",
         "type": "f16"},
        # one token through 8 of 64 experts
        {"name": "experts, one token", "op": "experts", "tokens": 1, "experts": 64, "chosen": 8, "width": 2048, "hidden": 1024, "group": 128,
         "zeros": False, "act": "silu", "type": "bf16"},
        # a few requests at once, odd sizes
        {"name": "experts, 24 tokens, odd", "op": "experts", "tokens": 24, "experts": 30, "chosen": 3, "width": 1100, "hidden": 777, "group": 32,
         "zeros": True, "act": "silu", "type": "f16"},
        # a long prompt: most experts are met, some by many more tokens than others
        {"name": "experts, 4096 tokens", "op": "experts", "tokens": 4096, "experts": 64, "chosen": 8, "width": 2048, "hidden": 1024, "group": 128,
         "zeros": False, "act": "silu", "type": "bf16"},
    ]


def _size(rng, low, high):
    """Spread evenly over the logarithm; half of the sizes are multiples of 64, as widths mostly are, the others as they fall."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    return max(low, n // 64 * 64) if rng.random() < 0.5 else n


MOST = 2 * 4096 * 8192 * 8192       # operations of the largest listed pass


def draw(rng):
    op = rng.choice(("route", "route_back", "linear", "gated", "experts"))
    if op in ("route", "route_back"):
        case = {"op": op, "tokens": _size(rng, 1, 16384), "score": rng.choice(("softmax", "sigmoid")), "renorm": rng.random() < 0.6,
                "type": rng.choice(sorted(TYPES))}
        groups = rng.choice((1, 1, 2, 4, 8)) if op == "route" else 1
        case["experts"] = groups * rng.randint(2, 256 // groups)
        kept = rng.randint(1, groups)
        case["chosen"] = rng.randint(1, min(8, case["experts"] // groups * kept))
        if op == "route":
            case.update(bias=rng.random() < 0.5, groups=groups, kept=kept, top=rng.choice((1, 2)))
        return case
    case = {"op": op, "group": rng.choice((32, 64, 128)), "zeros": rng.random() < 0.5, "type": rng.choice(("f16", "bf16"))}
    tokens = _size(rng, 1, 4096) if rng.random() < 0.6 else _size(rng, 1, 64)
    if op == "experts":
        case.update(experts=rng.randint(2, 64), width=_size(rng, 128, 2048), hidden=_size(rng, 128, 1024), act=rng.choice(("silu", "gelu")))
        case["chosen"] = rng.randint(1, min(8, case["experts"]))
        return {**case, "tokens": tokens}
    inner, outer = _size(rng, 128, 8192), _size(rng, 128, 8192)
    if op == "linear":
        case.update(inner=inner, outer=outer, bias=rng.random() < 0.5)
        return {**case, "tokens": tokens}
    case.update(inner=inner, hidden=outer, act=rng.choice(("silu", "gelu")))
    return {**case, "tokens": max(1, min(tokens, MOST // (4 * inner * outer)))}


# ---- what a program holds -----------------------------------------------------------------------------------------------


def _packed(levels):
    """Levels 0 .. 15 [..][rows][cols], eight to a word of 32 bits: of each eight value 2 j in bits 4 j .. 4 j + 3 and value 2 j + 1 in bits
    16 + 4 j .. 19 + 4 j.  Rows stand at multiples of 64 bytes."""
    cols = levels.shape[-1]
    words = (cols + 7) // 8
    held = (words + 15) // 16 * 16
    full = torch.nn.functional.pad(levels, (0, held * 8 - cols)).view(*levels.shape[:-1], held, 8)
    low, high = full[..., 0::2], full[..., 1::2]
    four = torch.stack((low[..., 0] | low[..., 1] << 4, low[..., 2] | low[..., 3] << 4, high[..., 0] | high[..., 1] << 4, high[..., 2] | high[..., 3] << 4), -1)
    return four.reshape(*levels.shape[:-1], held * 4)[..., :words * 4]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device="cuda") * std

    def inputs(rows, cols):
        # activations: rows of different size and mean, a few columns much larger than the others
        x = normal(rows, cols)
        x *= torch.exp(normal(rows, 1, std=0.3))
        x *= 1.0 + 7.0 * (torch.rand(cols, generator=gen, device="cuda") < 0.01)
        x += normal(rows, 1, std=0.1)
        return x.to(kind)

    def weights4(rows, cols, count=None):
        # levels as a normal distribution leaves them, scales that vary by a few tenths, zero points near the middle
        many = 1 if count is None else count
        groups = (cols + case["group"] - 1) // case["group"]
        scale = (torch.exp(normal(many, groups, rows, std=0.2)) / (2.6 * math.sqrt(cols))).to(kind)
        zero = torch.randint(6, 11, (many, groups, rows), generator=gen, device="cuda", dtype=torch.int32).to(torch.uint8) if case["zeros"] else None
        q = []
        for e in range(many):
            centre = 8.0 if zero is None else zero[e].repeat_interleave(case["group"], 0)[:cols].t()
            q.append(_packed((normal(rows, cols, std=2.6).round() + centre).clamp(0, 15).to(torch.uint8)))
        words = q[0].shape[1]
        held = torch.zeros(many, rows, (words + 63) // 64 * 64, dtype=torch.uint8, device="cuda")
        for e in range(many):
            held[e, :, :words] = q[e]
        held = held[:, :, :words]
        if count is None:
            return held[0], scale[0], None if zero is None else zero[0]
        return held, scale, zero

    kind, op = TYPES[case["type"]], case["op"]
    s = {"case": dict(case)}
    if op in ("route", "route_back"):
        # some experts are liked by all tokens
        t, e, k = case["tokens"], case["experts"], case["chosen"]
        s["logits"] = (normal(t, e, std=1.5) + normal(e, std=0.5)).to(kind)
        if op == "route":
            s["bias"] = normal(e, std=0.05) if case["bias"] else None
        else:
            p = _scores(s["logits"].double(), case["score"])
            s["experts"] = torch.sort(p, dim=1, descending=True, stable=True).indices[:, :k].to(torch.int32).contiguous()
            s["dweights"] = normal(t, k)
        return s
    if op == "linear":
        s["x"] = inputs(case["tokens"], case["inner"])
        s["w"] = weights4(case["outer"], case["inner"])
        s["bias"] = normal(case["outer"], std=0.1) if case["bias"] else None
    elif op == "gated":
        s["x"] = inputs(case["tokens"], case["inner"])
        s["wg"], s["wu"] = weights4(case["hidden"], case["inner"]), weights4(case["hidden"], case["inner"])
    else:
        t, e, k, d, f = case["tokens"], case["experts"], case["chosen"], case["width"], case["hidden"]
        s["x"] = inputs(t, d)
        s["wg"], s["wu"], s["wd"] = weights4(f, d, e), weights4(f, d, e), weights4(d, f, e)
        p = torch.softmax(normal(t, e, std=1.5) + normal(e, std=0.5), 1)
        top = torch.sort(p, dim=1, descending=True, stable=True)
        s["experts"] = top.indices[:, :k].to(torch.int32).contiguous()
        s["weights"] = (top.values[:, :k] / top.values[:, :k].sum(1, keepdim=True)).contiguous()
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------------


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2007_14178_amd import binding as xb
    case = s["case"]
    op = case["op"]
    if op in ("route", "route_back"):
        score = {"softmax": xb.SCORE_SOFTMAX, "sigmoid": xb.SCORE_SIGMOID}[case["score"]]
        if op == "route_back":
            return xb.xnor_route_bwd(s["dweights"], s["logits"], s["experts"], score=score, renorm=case["renorm"])
        experts, weights = xb.xnor_route_fwd(s["logits"], case["chosen"], bias=s["bias"], score=score, groups=case["groups"], groups_kept=case["kept"],
                                             group_top=case["top"], renorm=case["renorm"])
        offsets, order = xb.xnor_route_lists(experts, case["experts"])
        return experts, weights, offsets, order
    if op == "linear":
        return xb.xnor_int4_linear(s["x"], xb.Int4(*s["w"], case["inner"], case["group"]), s["bias"])
    act = {"silu": xb.ACT_SILU, "gelu": xb.ACT_GELU}[case["act"]]
    inner = case["inner"] if op == "gated" else case["width"]
    wg, wu = xb.Int4(*s["wg"], inner, case["group"]), xb.Int4(*s["wu"], inner, case["group"])
    if op == "gated":
        return xb.xnor_int4_gated(s["x"], wg, wu, act)
    return xb.xnor_int4_experts(s["x"], s["experts"], s["weights"], wg, wu, xb.Int4(*s["wd"], case["hidden"], case["group"]), act)


def _scores(logits, score):
    if score == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-logits))
    e = torch.exp(logits - logits.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True)


def _best(c, n):
    """The n largest of each row, the lowest index first among equals."""
    return torch.sort(c, dim=1, descending=True, stable=True).indices[:, :n]


def _unpacked(w, cols, group):
    """The fp32 weights that packed levels, scales and zero points stand for."""
    q, scale, zero = w
    four = q.view(q.shape[0], -1, 4)
    nibbles = torch.stack((four & 15, four >> 4), -1).view(q.shape[0], -1, 2, 4)        # [word][low or high half][j]
    levels = nibbles.transpose(2, 3).reshape(q.shape[0], -1)[:, :cols].float()
    by_column = lambda t: t.float().repeat_interleave(group, 0)[:cols].t()      # noqa: E731
    return (levels - (8.0 if zero is None else by_column(zero))) * by_column(scale)


def _act(g, act):
    if act == "silu":
        return g / (1.0 + torch.exp(-g))
    return 0.5 * g * (1.0 + torch.erf(g * math.sqrt(0.5)))


def _of(w, e):
    return w[0][e], w[1][e], None if w[2] is None else w[2][e]


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    if op == "route":
        # in 64 bits: which of two nearly equal scores is the larger decides whole numbers
        t, n, k = case["tokens"], case["experts"], case["chosen"]
        p = _scores(s["logits"].double(), case["score"])
        c = p if s["bias"] is None else p + s["bias"].double()
        if case["groups"] > 1:
            size = n // case["groups"]
            of_group = torch.sort(c.view(t, case["groups"], size), dim=2, descending=True).values[:, :, :min(case["top"], size)].sum(2)
            kept = torch.zeros_like(of_group).scatter_(1, _best(of_group, case["kept"]), 1.0)
            c = torch.where(kept.repeat_interleave(size, 1) > 0, c, torch.full_like(c, -math.inf))
        experts = _best(c, k)
        w = p.gather(1, experts)
        if case["renorm"]:
            w = w / w.sum(1, keepdim=True)
        flat = experts.reshape(-1)
        order = torch.sort(flat, dim=0, stable=True).indices
        offsets = torch.zeros(n + 1, dtype=torch.int64, device=flat.device)
        offsets[1:] = (flat[:, None] == torch.arange(n, device=flat.device)).sum(0).cumsum(0)
        return experts.int(), w.float(), offsets.int(), order.int()
    if op == "route_back":
        kind, experts = s["logits"].dtype, s["experts"].long()
        p = _scores(s["logits"].float(), case["score"])
        chosen, dw = p.gather(1, experts), s["dweights"]
        if case["renorm"]:
            total = chosen.sum(1, keepdim=True)
            dw = (dw - (dw * chosen).sum(1, keepdim=True) / total) / total
        dp = torch.zeros_like(p).scatter_(1, experts, dw)
        if case["score"] == "sigmoid":
            return (dp * p * (1.0 - p)).to(kind)
        return (p * (dp - (dp * p).sum(1, keepdim=True))).to(kind)
    x, kind, group = s["x"].float(), s["x"].dtype, case["group"]
    if op == "linear":
        y = x @ _unpacked(s["w"], case["inner"], group).t()
        return (y if s["bias"] is None else y + s["bias"]).to(kind)
    if op == "gated":
        g, u = x @ _unpacked(s["wg"], case["inner"], group).t(), x @ _unpacked(s["wu"], case["inner"], group).t()
        return (_act(g, case["act"]) * u).to(kind)
    # the tokens of one expert after the other, as a program has it that multiplies with an expert at a time
    d, f, k = case["width"], case["hidden"], case["chosen"]
    flat = s["experts"].reshape(-1).long()
    order = torch.sort(flat, dim=0, stable=True).indices
    counts = (flat[:, None] == torch.arange(case["experts"], device=flat.device)).sum(0).tolist()
    pairs = torch.empty(flat.shape[0], d, device=x.device)
    at = 0
    for e, n in enumerate(counts):
        if n == 0:
            continue
        mine = order[at:at + n]
        at += n
        xe = x[mine // k]
        h = _act(xe @ _unpacked(_of(s["wg"], e), d, group).t(), case["act"]) * (xe @ _unpacked(_of(s["wu"], e), d, group).t())
        pairs[mine] = h @ _unpacked(_of(s["wd"], e), f, group).t()
    return (pairs.view(-1, k, d) * s["weights"][:, :, None]).sum(1).to(kind)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------


def work(case):
    e = 4 if case["type"] == "fp32" else 2
    t = case["tokens"]
    if case["op"] == "route":
        n, k = case["experts"], case["chosen"]
        return {"bytes": t * n * e + 12 * t * k + 4 * n + (4 * n if case["bias"] else 0), "flops": 20 * t * n}
    if case["op"] == "route_back":
        n, k = case["experts"], case["chosen"]
        return {"bytes": 2 * t * n * e + 8 * t * k, "flops": 10 * t * n}

    def held(rows, cols):
        return rows * (cols + 1) // 2 + rows * ((cols + case["group"] - 1) // case["group"]) * (3 if case["zeros"] else 2)
    if case["op"] == "linear":
        k, n = case["inner"], case["outer"]
        return {"bytes": 2 * t * k + held(n, k) + 2 * t * n + (4 * n if case["bias"] else 0), "flops": 2 * t * k * n}
    if case["op"] == "gated":
        k, f = case["inner"], case["hidden"]
        return {"bytes": 2 * t * k + 2 * held(f, k) + 2 * t * f, "flops": 4 * t * k * f}
    n, k, d, f = case["experts"], case["chosen"], case["width"], case["hidden"]
    met = n * (1.0 - (1.0 - k / n) ** t)         # experts that at least one of the tokens has chosen, were all liked alike
    return {"bytes": int(4 * t * d + 8 * t * k + met * (2 * held(f, d) + held(d, f))), "flops": 6 * t * k * d * f}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------


def _exact_weights(w, cols, group):
    """Column by column of the words' bits."""
    q, scale, zero = w
    words = q.contiguous().view(torch.int32).long()
    out = torch.empty(q.shape[0], words.shape[1] * 8, dtype=torch.float64, device=q.device)
    for v in range(8):
        out[:, v::8] = (words >> (4 * (v // 2) + 16 * (v % 2)) & 15).double()
    out = out[:, :cols]
    for j in range(scale.shape[0]):
        part = out[:, j * group:(j + 1) * group]
        part -= 8.0 if zero is None else zero[j].double()[:, None]
        part *= scale[j].double()[:, None]
    return out


def _exact_gate(g, act):
    return g * torch.sigmoid(g) if act == "silu" else 0.5 * g * torch.special.erfc(-g / math.sqrt(2.0))


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("route", "route_back"):
        logits = s["logits"].double()
        p = torch.sigmoid(logits) if case["score"] == "sigmoid" else torch.softmax(logits, 1)
        t, n, k = case["tokens"], case["experts"], case["chosen"]
        if op == "route_back":
            p.requires_grad_(True)
            w = p.gather(1, s["experts"].long())
            if case["renorm"]:
                w = w / w.sum(1, keepdim=True)
            (dp,) = torch.autograd.grad(w, p, s["dweights"].double())
            p = p.detach()
            return dp * p * torch.sigmoid(-logits) if case["score"] == "sigmoid" else p * dp - p * (p * dp).sum(1, keepdim=True)
        c = p.clone() if s["bias"] is None else p + s["bias"].double()
        size = n // case["groups"]
        if case["groups"] > 1:
            left = c.view(t, case["groups"], size).clone()
            of_group = torch.zeros(t, case["groups"], dtype=torch.float64, device=c.device)
            for _ in range(min(case["top"], size)):
                best = left.max(2)
                of_group += best.values
                left.scatter_(2, best.indices[:, :, None], -math.inf)
            out = torch.ones(t, case["groups"], dtype=torch.bool, device=c.device)
            for _ in range(case["kept"]):
                most = of_group.amax(1, keepdim=True)
                first = (of_group == most).int().argmax(1, keepdim=True)
                out.scatter_(1, first, False)
                of_group.scatter_(1, first, -math.inf)
            c[out.repeat_interleave(size, 1)] = -math.inf
        places = torch.arange(n, device=c.device)
        experts = torch.empty(t, k, dtype=torch.int64, device=c.device)
        for i in range(k):
            experts[:, i] = torch.where(c == c.amax(1, keepdim=True), places, n).amin(1)
            c.scatter_(1, experts[:, i:i + 1], -math.inf)
        w = p.gather(1, experts)
        if case["renorm"]:
            w = w / w.sum(1, keepdim=True)
        pairs = torch.arange(t * k, device=c.device)
        order = torch.argsort(experts.reshape(-1) * (t * k) + pairs)
        offsets = torch.searchsorted(experts.reshape(-1)[order], torch.arange(n + 1, device=c.device))
        return experts.int(), w, offsets.int(), order.int()
    x, group = s["x"].double(), case["group"]
    if op == "linear":
        y = torch.matmul(x, _exact_weights(s["w"], case["inner"], group).t())
        return y if s["bias"] is None else y + s["bias"].double()
    if op == "gated":
        g, u = (torch.matmul(x, _exact_weights(s[w], case["inner"], group).t()) for w in ("wg", "wu"))
        return _exact_gate(g, case["act"]) * u
    y = torch.zeros(case["tokens"], case["width"], dtype=torch.float64, device=x.device)
    for e in range(case["experts"]):
        # (an expert stands at most once among a token's)
        share = torch.where(s["experts"] == e, s["weights"].double(), 0.0).sum(1)
        rows = (s["experts"] == e).any(1).nonzero()[:, 0]
        if rows.numel() == 0:
            continue
        g, u = (torch.matmul(x[rows], _exact_weights(_of(s[w], e), case["width"], group).t()) for w in ("wg", "wu"))
        y[rows] += share[rows, None] * torch.matmul(_exact_gate(g, case["act"]) * u, _exact_weights(_of(s["wd"], e), case["hidden"], group).t())
    return y
