"""Timed passes through the dense operators: the 8-bit linear layer, layer norm and the gated feed-forward block.

``listed`` names the passes, ``draw`` makes more of the same ranges, ``prepare`` makes what a program holds before the call
and ``run`` is one pass: through the library where ``own`` is set, else in elementary torch operations in 32 bits.  ``exact``
is the definition in 64 bits.  Operators:

    int8_linear  y = quantised(x) w^T with a scale per token and channel, from real tokens and 8-bit weights
    norm         layer norm, forward (with the statistics that the backward pass takes) or backward
    int8_gated   layer norm, quantisation and the gated block on 8-bit weights: the front of a served feed-forward layer
    gated        the gated block in 16 bits, forward (with what the backward pass takes) or backward
"""
import math

import torch

own = False

EPS = 1e-5
TYPES = {"fp32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # one token through a square layer: a decoding step, bound by latency and by reading the weights
        {"name": "linear, one token", "op": "int8_linear", "tokens": 1, "inner": 4096, "outer": 4096, "type": "bf16", "bias": False},
        # a few requests at once through a layer of odd sizes, with a bias
        {"name": "linear, 13 tokens, odd", "op": "int8_linear", "tokens": 13, "inner": 1037, "outer": 1531, "type": "f16", "bias": True},
        # the positions and channels of 128 images of 28 x 28 with 512 channels, as a pointwise layer in fp32
        {"name": "linear, image positions", "op": "int8_linear", "tokens": 100352, "inner": 512, "outer": 512, "type": "fp32", "bias": True},
        # prompts of a large batch through a large layer
        {"name": "linear, 16384 tokens", "op": "int8_linear", "tokens": 16384, "inner": 8192, "outer": 8192, "type": "bf16", "bias": False},
        # the norm of one token in a decoding step: latency alone
        {"name": "norm, one token", "op": "norm", "back": False, "rows": 1, "cols": 4096, "type": "bf16", "params": "bf16"},
        # the norm in front of a layer, a training batch
        {"name": "norm, 16384 rows", "op": "norm", "back": False, "rows": 16384, "cols": 4096, "type": "f16", "params": "fp32"},
        # gradients of a small fp32 layer of odd sizes
        {"name": "norm back, odd", "op": "norm", "back": True, "rows": 1000, "cols": 1111, "type": "fp32", "params": "fp32"},
        # gradients of a training batch
        {"name": "norm back, 16384 rows", "op": "norm", "back": True, "rows": 16384, "cols": 4096, "type": "bf16", "params": "fp32"},
        # the served feed-forward layer's front for one token
        {"name": "8-bit gated, one token", "op": "int8_gated", "tokens": 1, "inner": 4096, "hidden": 8192, "act": "silu", "type": "bf16"},
        # ... and for a prompt
        {"name": "8-bit gated, 2000 tokens", "op": "int8_gated", "tokens": 2000, "inner": 4096, "hidden": 8192, "act": "silu", "type": "f16"},
        # the training forward pass of a small layer of odd sizes
        {"name": "gated, odd", "op": "gated", "back": False, "tokens": 777, "inner": 1001, "hidden": 2501, "act": "gelu", "type": "f16"},
        # gradients of a training batch
        {"name": "gated back, 8192 tokens", "op": "gated", "back": True, "tokens": 8192, "inner": 4096, "hidden": 8192, "act": "silu", "type": "bf16"},
    ]


def _size(rng, low, high):
    """Spread evenly over the logarithm; half of the sizes are multiples of 64, as widths mostly are, the others as they fall."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    return max(low, n // 64 * 64) if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(("int8_linear", "norm", "int8_gated", "gated"))
    if op == "norm":
        return {"op": op, "back": rng.random() < 0.5, "rows": _size(rng, 1, 16384), "cols": _size(rng, 64, 8192), "type": rng.choice(sorted(TYPES)),
                "params": "fp32"}
    case = {"op": op, "tokens": _size(rng, 1, 16384), "inner": _size(rng, 256, 8192)}
    if op == "int8_linear":
        case.update(outer=_size(rng, 256, 8192), type=rng.choice(sorted(TYPES)), bias=rng.random() < 0.5)
        return case
    case.update(hidden=_size(rng, 256, 8192), act=rng.choice(("silu", "gelu")), type=rng.choice(("f16", "bf16")))
    case["tokens"] = min(case["tokens"], 8192)
    if op == "gated":
        case["back"] = rng.random() < 0.5
        case["inner"] = min(case["inner"], 4096)
    elif case["tokens"] < 64:
        case["type"] = "bf16"
    return case


def _rows16(w):
    """8-bit rows on a stride of 16 bytes, as the library lays out what it quantises."""
    n, k = w.shape
    held = torch.zeros(n, (k + 15) // 16 * 16, dtype=torch.int8, device=w.device)
    held[:, :k] = w
    return held[:, :k]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device="cuda") * std

    def tokens(rows, cols, kind):
        # activations: rows of different size and mean, a few columns much larger than the others
        x = normal(rows, cols)
        x *= torch.exp(normal(rows, 1, std=0.3))
        x *= 1.0 + 7.0 * (torch.rand(cols, generator=gen, device="cuda") < 0.01)
        x += normal(rows, 1, std=0.1)
        return x.to(kind)

    def weights8(rows, cols):
        w = torch.randint(-127, 128, (rows, cols), generator=gen, device="cuda", dtype=torch.int32).to(torch.int8)
        return _rows16(w), torch.exp(normal(rows, std=0.2)) / (73.0 * math.sqrt(cols))

    kind, op = TYPES[case["type"]], case["op"]
    s = {"case": dict(case)}
    if op == "int8_linear":
        s["x"] = tokens(case["tokens"], case["inner"], kind)
        s["w"], s["w_scale"] = weights8(case["outer"], case["inner"])
        s["bias"] = normal(case["outer"], std=0.1) if case["bias"] else None
    elif op == "norm":
        n, c, params = case["rows"], case["cols"], TYPES[case["params"]]
        s["x"] = tokens(n, c, kind)
        s["gamma"], s["beta"] = (1.0 + normal(c, std=0.1)).to(params), normal(c, std=0.1).to(params)
        if case["back"]:
            s["dy"] = normal(n, c).to(kind)
            x = s["x"].float()
            s["mean"] = x.mean(1)
            s["rstd"] = 1.0 / torch.sqrt((x - s["mean"][:, None]).square().mean(1) + EPS)
    elif op == "int8_gated":
        s["x"] = tokens(case["tokens"], case["inner"], kind)
        s["gamma"], s["beta"] = 1.0 + normal(case["inner"], std=0.1), normal(case["inner"], std=0.1)
        s["wg"], s["wg_scale"] = weights8(case["hidden"], case["inner"])
        s["wu"], s["wu_scale"] = weights8(case["hidden"], case["inner"])
    else:
        m, k, f = case["tokens"], case["inner"], case["hidden"]
        s["x"] = normal(m, k).to(kind)
        s["wg"], s["wu"] = normal(f, k, std=k ** -0.5).to(kind), normal(f, k, std=k ** -0.5).to(kind)
        if case["back"]:
            s["dh"] = normal(m, f).to(kind)
            # what the forward pass left: of the products' distribution
            s["g"], s["u"] = normal(m, f).to(kind), normal(m, f).to(kind)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------------


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2007_14178_amd import binding as xb
    case = s["case"]
    op = case["op"]
    if op == "int8_linear":
        return xb.xnor_int8_linear(s["x"], s["w"], s["w_scale"], s["bias"])
    if op == "norm":
        if case["back"]:
            return xb.xnor_layer_norm_bwd(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"])
        return xb.xnor_layer_norm_fwd(s["x"], s["gamma"], s["beta"], EPS)
    act = {"silu": xb.ACT_SILU, "gelu": xb.ACT_GELU}[case["act"]]
    if op == "int8_gated":
        q, scale = xb.xnor_layer_norm_fwd_int8(s["x"], s["gamma"], s["beta"], EPS)
        return xb.xnor_int8_gated(q, scale, s["wg"], s["wg_scale"], s["wu"], s["wu_scale"], act, out_dtype=s["x"].dtype)
    if case["back"]:
        return xb.xnor_gated_bwd(s["dh"], s["x"], s["wg"], s["wu"], s["g"], s["u"], act)
    return xb.xnor_gated_fwd(s["x"], s["wg"], s["wu"], act, want_pre=True)


def _quantise(x):
    top = x.abs().amax(1, keepdim=True)
    most = torch.full_like(top, 127.0)      # (a division by or of a number is not rounded as one of two tensors is)
    return torch.round(x * (most / top)), top / most


def _norm(x, gamma, beta):
    mean = x.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + EPS)
    return (x - mean) * rstd * gamma.float() + beta.float(), mean, rstd


def _act(g, act):
    """The activation and its derivative."""
    if act == "silu":
        sg = 1.0 / (1.0 + torch.exp(-g))
        return g * sg, sg * (1.0 + g * (1.0 - sg))
    phi = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return g * phi, phi + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    kind = s["x"].dtype
    x = s["x"].float()
    if op == "int8_linear":
        q, scale = _quantise(x)
        y = (q @ s["w"].float().t()) * (scale * s["w_scale"])
        return (y if s["bias"] is None else y + s["bias"]).to(kind)
    if op == "norm":
        if not case["back"]:
            y, mean, rstd = _norm(x, s["gamma"], s["beta"])
            return y.to(kind), mean[:, 0], rstd[:, 0]
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        xh = (x - s["mean"][:, None]) * rstd
        p = dy * s["gamma"].float()
        dx = rstd * (p - p.mean(1, keepdim=True) - xh * (p * xh).mean(1, keepdim=True))
        return dx.to(kind), (dy * xh).sum(0).to(s["gamma"].dtype), dy.sum(0).to(s["gamma"].dtype)
    if op == "int8_gated":
        q, scale = _quantise(_norm(x, s["gamma"], s["beta"])[0])
        g = (q @ s["wg"].float().t()) * (scale * s["wg_scale"])
        u = (q @ s["wu"].float().t()) * (scale * s["wu_scale"])
        return (_act(g, case["act"])[0] * u).to(kind)
    wg, wu = s["wg"].float(), s["wu"].float()
    if not case["back"]:
        g, u = x @ wg.t(), x @ wu.t()
        return (_act(g, case["act"])[0] * u).to(kind), g.to(kind), u.to(kind)
    a, d = _act(s["g"].float(), case["act"])
    dh = s["dh"].float()
    dg, du = dh * s["u"].float() * d, dh * a
    return (dg @ wg + du @ wu).to(kind), (dg.t() @ x).to(kind), (du.t() @ x).to(kind)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------


def work(case):
    e = 4 if case["type"] == "fp32" else 2
    if case["op"] == "norm":
        n, c, pe = case["rows"], case["cols"], 4 if case["params"] == "fp32" else 2
        if case["back"]:
            return {"bytes": 3 * n * c * e + 8 * n + 3 * c * pe, "flops": 14 * n * c}
        return {"bytes": 2 * n * c * e + 8 * n + 2 * c * pe, "flops": 8 * n * c}
    m, k = case["tokens"], case["inner"]
    if case["op"] == "int8_linear":
        f = case["outer"]
        return {"bytes": m * k * e + f * k + 4 * f * (2 if case["bias"] else 1) + m * f * e, "flops": 2 * m * k * f}
    f = case["hidden"]
    if case["op"] == "int8_gated":
        return {"bytes": m * k * e + 8 * k + 2 * f * k + 8 * f + m * f * e, "flops": 4 * m * k * f}
    if case["back"]:
        return {"bytes": e * (2 * m * k + 4 * f * k + 3 * m * f), "flops": 8 * m * k * f}
    return {"bytes": e * (m * k + 2 * f * k + 3 * m * f), "flops": 4 * m * k * f}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------


def _exact_normed(x, gamma, beta):
    centred = x - x.sum(1, keepdim=True) / x.shape[1]
    spread = (centred * centred).sum(1, keepdim=True) / x.shape[1]
    return centred * (spread + EPS).pow(-0.5) * gamma.double() + beta.double(), x.sum(1) / x.shape[1], (spread[:, 0] + EPS).pow(-0.5)


def _exact_levels(x):
    step = x.abs().max(1, keepdim=True).values / 127.0
    return torch.round(x / step), step


def _exact_gate(g, act):
    return g * torch.sigmoid(g) if act == "silu" else 0.5 * g * torch.special.erfc(-g / math.sqrt(2.0))


def exact(case, seed):
    s = prepare(case, seed)
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    x = d["x"]
    if case["op"] == "int8_linear":
        q, step = _exact_levels(x)
        y = torch.matmul(q, d["w"].t()) * step * d["w_scale"][None, :]
        return y + d["bias"][None, :] if "bias" in d else y
    if case["op"] == "norm":
        if not case["back"]:
            return _exact_normed(x, s["gamma"], s["beta"])
        xh = (x - d["mean"][:, None]) * d["rstd"][:, None]
        p = d["dy"] * d["gamma"][None, :]
        n = x.shape[1]
        dx = (p - p.sum(1, keepdim=True) / n - xh * ((p * xh).sum(1, keepdim=True) / n)) * d["rstd"][:, None]
        return dx, (xh * d["dy"]).sum(0), d["dy"].sum(0)
    if case["op"] == "int8_gated":
        q, step = _exact_levels(_exact_normed(x, s["gamma"], s["beta"])[0])
        g = torch.matmul(q, d["wg"].t()) * step * d["wg_scale"][None, :]
        u = torch.matmul(q, d["wu"].t()) * step * d["wu_scale"][None, :]
        return _exact_gate(g, case["act"]) * u
    if not case["back"]:
        g, u = torch.matmul(x, d["wg"].t()), torch.matmul(x, d["wu"].t())
        return _exact_gate(g, case["act"]) * u, g, u
    g = d["g"]
    if case["act"] == "silu":
        slope = torch.sigmoid(g) + g * torch.sigmoid(g) * torch.sigmoid(-g)
    else:
        slope = 0.5 * torch.special.erfc(-g / math.sqrt(2.0)) + g * torch.exp(-g * g / 2.0) / math.sqrt(2.0 * math.pi)
    dg, du = d["dh"] * d["u"] * slope, d["dh"] * _exact_gate(g, case["act"])
    return torch.matmul(dg, d["wg"]) + torch.matmul(du, d["wu"]), torch.matmul(dg.t(), x), torch.matmul(du.t(), x)
