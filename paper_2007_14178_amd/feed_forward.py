"""A feed-forward layer as a network has it: trained in 16 bits, served in 8.

    y = x + (act(n wg^T) * (n wu^T)) wd^T,   n = layer norm of x

``FeedForward`` holds the 16-bit parameters and trains by ``forward`` / ``backward``: the norm and the gated block and their gradients
are the library's, the plain product with wd is torch's.  ``serve`` makes an ``Int8FeedForward`` of it, whose products all run on
8-bit tokens and weights: the norm hands its output on quantised, the gated block is one kernel, and the last product
quantises the block's output on the way.

    python -m paper_2007_14178_amd.feed_forward

trains a small layer for some steps and compares what it serves with what it was trained to.
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


def main() -> None:
    torch.manual_seed(0)
    width, hidden, tokens = 256, 512, 1024
    layer, target = FeedForward(width, hidden, seed=1), FeedForward(width, hidden, seed=2)
    master = {k: v.float() for k, v in layer.params.items()}
    for step in range(61):
        x = torch.randn(tokens, width, device="cuda").to(torch.bfloat16)
        want, _ = target.forward(x)
        y, kept = layer.forward(x)
        error = y.float() - want.float()
        _, grads = layer.backward((error * (2.0 / tokens)).to(torch.bfloat16), kept)
        for k, v in master.items():
            v -= 0.2 * grads[k].float()
            layer.params[k] = v.to(layer.params[k].dtype)
        if step % 20 == 0:
            print(f"step {step}: mean square error {error.square().mean().item():.4f}", flush=True)
    served, (trained, _) = layer.serve()(x), layer.forward(x)
    branch = (trained - x).float()
    print(f"served in 8 bits: {((served - trained).float().norm() / branch.norm()).item():.2%} of the layer's own output away", flush=True)


if __name__ == "__main__":
    main()
