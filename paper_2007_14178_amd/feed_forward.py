"""A feed-forward layer as a network has it: trained in 16 bits, served in 8 or 4; and one of several experts.

    y = x + (act(n wg^T) * (n wu^T)) wd^T,   n = layer norm of x

``FeedForward`` holds the 16-bit parameters and trains by ``forward`` / ``backward``: the norm and the gated block and their gradients
are the library's, the plain product with wd is torch's.  ``serve`` makes an ``Int8FeedForward`` of it, whose products all run on
8-bit tokens and weights: the norm hands its output on quantised, the gated block is one kernel, and the last product
quantises the block's output on the way.  ``serve4`` makes an ``Int4FeedForward``: 4-bit weights with group scales, tokens in 16 bits.

``Experts`` is the same layer with a router and E such blocks, of which each token takes the k that its router scores highest:

    y = x + sum over the token's experts e of weight * ((act(n wg_e^T) * (n wu_e^T)) wd_e^T)

It trains an expert at a time by the 16-bit block, its router by the routing's gradient and its experts' balance by a bias that only the choice
sees; ``serve4`` makes an ``Int4Experts``, whose experts' products are one call on stacks of 4-bit weights.

    python -m paper_2007_14178_amd.feed_forward

trains small layers for some steps and compares what they serve with what they were trained to.
"""
from __future__ import annotations

import torch

from paper_2007_14178_amd import binding as xb


class FeedForward:
    def __init__(self, width: int, hidden: int, dtype: torch.dtype = torch.bfloat16, act: int = xb.ACT_SILU, eps: float = 1e-5,
                 device: str = "cuda", seed: int = 0):
        gen = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape: int, std: float) -> torch.Tensor:
            return (torch.randn(*shape, generator=gen, device=device) * std).to(dtype)
        self.act, self.eps = act, eps
        self.params = {"gamma": torch.ones(width, device=device), "beta": torch.zeros(width, device=device),
                       "wg": normal(hidden, width, std=width ** -0.5), "wu": normal(hidden, width, std=width ** -0.5),
                       "wd": normal(width, hidden, std=hidden ** -0.5)}

    def forward(self, x: torch.Tensor) -> tuple[torch.Tensor, tuple]:
        """y for tokens x [M][width], and what ``backward`` takes of the pass."""
        p = self.params
        n, mean, rstd = xb.xnor_layer_norm_fwd(x, p["gamma"], p["beta"], self.eps)
        h, g, u = xb.xnor_gated_fwd(n, p["wg"], p["wu"], self.act, want_pre=True)
        return x + h @ p["wd"].t(), (x, n, mean, rstd, h, g, u)

    def backward(self, dy: torch.Tensor, kept: tuple) -> tuple[torch.Tensor, dict]:
        """dx and the parameters' gradients from dy."""
        p = self.params
        x, n, mean, rstd, h, g, u = kept
        dn, dwg, dwu = xb.xnor_gated_bwd(dy @ p["wd"], n, p["wg"], p["wu"], g, u, self.act)
        dx, dgamma, dbeta = xb.xnor_layer_norm_bwd(dn, x, p["gamma"], mean, rstd)
        return dx + dy, {"gamma": dgamma, "beta": dbeta, "wg": dwg, "wu": dwu, "wd": dy.t() @ h}

    def serve(self) -> "Int8FeedForward":
        return Int8FeedForward(self)

    def serve4(self, group: int = 128, zeros: bool = False) -> "Int4FeedForward":
        return Int4FeedForward(self, group, zeros)


class Int8FeedForward:
    """The layer on 8-bit weights with a scale per output channel, for tokens in the type that it was trained in."""

    def __init__(self, layer: FeedForward):
        p = layer.params
        self.act, self.eps = layer.act, layer.eps
        self.gamma, self.beta = p["gamma"].clone(), p["beta"].clone()
        (self.wg, self.wg_scale), (self.wu, self.wu_scale), (self.wd, self.wd_scale) = (xb.xnor_int8_quantize(p[k]) for k in ("wg", "wu", "wd"))

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        q, scale = xb.xnor_layer_norm_fwd_int8(x, self.gamma, self.beta, self.eps)
        h = xb.xnor_int8_gated(q, scale, self.wg, self.wg_scale, self.wu, self.wu_scale, self.act, out_dtype=x.dtype)
        return x + xb.xnor_int8_linear(h, self.wd, self.wd_scale)


class Int4FeedForward:
    """The layer on 4-bit weights with a scale (``zeros``: and a zero point) for each output channel and group of inputs."""

    def __init__(self, layer: FeedForward, group: int = 128, zeros: bool = False):
        p = layer.params
        self.act, self.eps = layer.act, layer.eps
        self.gamma, self.beta = p["gamma"].clone(), p["beta"].clone()
        self.wg, self.wu, self.wd = (xb.xnor_int4_quantize(p[k], group, zeros) for k in ("wg", "wu", "wd"))

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        n, _, _ = xb.xnor_layer_norm_fwd(x, self.gamma, self.beta, self.eps, want_stats=False)
        return x + xb.xnor_int4_linear(xb.xnor_int4_gated(n, self.wg, self.wu, self.act), self.wd)


class Experts:
    def __init__(self, width: int, hidden: int, experts: int, chosen: int, dtype: torch.dtype = torch.bfloat16, act: int = xb.ACT_SILU,
                 score: int = xb.SCORE_SIGMOID, eps: float = 1e-5, device: str = "cuda", seed: int = 0):
        gen = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape: int, std: float) -> torch.Tensor:
            return (torch.randn(*shape, generator=gen, device=device) * std).to(dtype)
        self.act, self.eps, self.chosen, self.score = act, eps, chosen, score
        self.bias = torch.zeros(experts, device=device)         # of the choice; moved by balance(), not by gradients
        self.params = {"gamma": torch.ones(width, device=device), "beta": torch.zeros(width, device=device),
                       "router": normal(experts, width, std=width ** -0.5),
                       "wg": normal(experts, hidden, width, std=width ** -0.5), "wu": normal(experts, hidden, width, std=width ** -0.5),
                       "wd": normal(experts, width, hidden, std=hidden ** -0.5)}

    def route(self, n: torch.Tensor) -> tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
        logits = n @ self.params["router"].t()
        return logits, *xb.xnor_route_fwd(logits, self.chosen, self.bias, self.score)

    def forward(self, x: torch.Tensor) -> tuple[torch.Tensor, tuple]:
        """y for tokens x [T][width], and what ``backward`` takes of the pass."""
        p, k = self.params, self.chosen
        n, mean, rstd = xb.xnor_layer_norm_fwd(x, p["gamma"], p["beta"], self.eps)
        logits, experts, weights = self.route(n)
        offsets, order = xb.xnor_route_lists(experts, p["router"].shape[0])
        pairs = torch.zeros(x.shape[0] * k, x.shape[1], dtype=x.dtype, device=x.device)
        ends, blocks = offsets.tolist(), []
        for e, (begin, end) in enumerate(zip(ends, ends[1:])):
            mine = order[begin:end].long()
            m = n[mine // k]
            h, g, u = xb.xnor_gated_fwd(m, p["wg"][e], p["wu"][e], self.act, want_pre=True)
            pairs[mine] = h @ p["wd"][e].t()
            blocks.append((mine, m, h, g, u))
        y = x + (pairs.view(-1, k, x.shape[1]).float() * weights[:, :, None]).sum(1).to(x.dtype)
        return y, (x, n, mean, rstd, logits, experts, weights, offsets, pairs, blocks)

    def backward(self, dy: torch.Tensor, kept: tuple) -> tuple[torch.Tensor, dict]:
        """dx and the parameters' gradients from dy."""
        p, k = self.params, self.chosen
        x, n, mean, rstd, logits, experts, weights, _, pairs, blocks = kept
        dweights = (pairs.view(-1, k, x.shape[1]).float() * dy.float()[:, None]).sum(2)
        dpairs = (dy.float()[:, None] * weights[:, :, None]).to(x.dtype).view(pairs.shape)
        grads = {name: torch.zeros_like(p[name]) for name in ("wg", "wu", "wd")}
        dn_pairs = torch.zeros_like(pairs)
        for e, (mine, m, h, g, u) in enumerate(blocks):
            d = dpairs[mine]
            dm, _, _ = xb.xnor_gated_bwd(d @ p["wd"][e], m, p["wg"][e], p["wu"][e], g, u, self.act, dwg=grads["wg"][e], dwu=grads["wu"][e])
            grads["wd"][e] = d.t() @ h
            dn_pairs[mine] = dm
        dlogits = xb.xnor_route_bwd(dweights, logits, experts, score=self.score)
        grads["router"] = dlogits.t() @ n
        dn = (dn_pairs.view(-1, k, x.shape[1]).float().sum(1) + (dlogits @ p["router"]).float()).to(x.dtype)
        dx, grads["gamma"], grads["beta"] = xb.xnor_layer_norm_bwd(dn, x, p["gamma"], mean, rstd)
        return dx + dy, grads

    def balance(self, kept: tuple, step: float = 1e-3) -> None:
        """Experts that the pass chose less often than the mean are favoured by ``step`` from now on, the others put back by as much."""
        counts = kept[7].diff().float()
        self.bias += step * torch.sign(counts.mean() - counts)

    def serve4(self, group: int = 128, zeros: bool = False) -> "Int4Experts":
        return Int4Experts(self, group, zeros)


class Int4Experts:
    """The layer on stacks of 4-bit weights; the router stays in 16 bits."""

    def __init__(self, layer: Experts, group: int = 128, zeros: bool = False):
        p = layer.params
        self.act, self.eps, self.chosen, self.score = layer.act, layer.eps, layer.chosen, layer.score
        self.gamma, self.beta, self.router, self.bias = p["gamma"].clone(), p["beta"].clone(), p["router"].clone(), layer.bias.clone()
        self.wg, self.wu, self.wd = (xb.xnor_int4_quantize(p[k], group, zeros) for k in ("wg", "wu", "wd"))

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        n, _, _ = xb.xnor_layer_norm_fwd(x, self.gamma, self.beta, self.eps, want_stats=False)
        experts, weights = xb.xnor_route_fwd(n @ self.router.t(), self.chosen, self.bias, self.score)
        return x + xb.xnor_int4_experts(n, experts, weights, self.wg, self.wu, self.wd, self.act)


def _train(layer, target, tokens: int, width: int, steps: int) -> torch.Tensor:
    master = {k: v.float() for k, v in layer.params.items()}
    for step in range(steps):
        x = torch.randn(tokens, width, device="cuda").to(torch.bfloat16)
        want, _ = target.forward(x)
        y, kept = layer.forward(x)
        error = y.float() - want.float()
        _, grads = layer.backward((error * (2.0 / tokens)).to(torch.bfloat16), kept)
        if isinstance(layer, Experts):
            layer.balance(kept)
        for k, v in master.items():
            v -= 0.2 * grads[k].float()
            layer.params[k] = v.to(layer.params[k].dtype)
        if step % 20 == 0:
            print(f"step {step}: mean square error {error.square().mean().item():.4f}", flush=True)
    return x


def main() -> None:
    torch.manual_seed(0)
    width, hidden, tokens = 256, 512, 1024
    layer = FeedForward(width, hidden, seed=1)
    x = _train(layer, FeedForward(width, hidden, seed=2), tokens, width, 61)
    trained, _ = layer.forward(x)
    branch = (trained - x).float()
    for bits, served in ((8, layer.serve()), (4, layer.serve4())):
        off = (served(x) - trained).float().norm() / branch.norm()
        print(f"served in {bits} bits: {off.item():.2%} of the layer's own output away", flush=True)
    mixture = Experts(width, hidden // 2, 8, 2, seed=3)
    x = _train(mixture, FeedForward(width, hidden, seed=2), tokens, width, 41)
    trained, _ = mixture.forward(x)
    off = (mixture.serve4(group=64)(x) - trained).float().norm() / (trained - x).float().norm()
    print(f"experts served in 4 bits: {off.item():.2%} of the layer's own output away", flush=True)


if __name__ == "__main__":
    main()
