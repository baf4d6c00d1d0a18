"""The feed-forward layer of several experts: gradients against autograd in 64 bits, and the 4-bit layers that are served."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import experts_reference as xref  # noqa: E402

pytestmark = pytest.mark.gpu

UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def normed(x, p, eps):
    centred = x - x.mean(1, keepdim=True)
    return centred / torch.sqrt(centred.square().mean(1, keepdim=True) + eps) * p["gamma"] + p["beta"]


def plain(x, p, chosen, score, eps):
    """The layer in 64 bits with the experts that were chosen, by torch's elementary operations."""
    n = normed(x, p, eps)
    weights = xref.weights_of(n @ p["router"].t(), chosen, score, True, 1.0)
    y = x
    for e in range(p["router"].shape[0]):
        g, u = n @ p["wg"][e].t(), n @ p["wu"][e].t()
        share = torch.where(chosen == e, weights, torch.zeros((), dtype=torch.float64, device=x.device)).sum(1, keepdim=True)
        y = y + share * ((g * torch.sigmoid(g) * u) @ p["wd"][e].t())
    return y


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=str)
@pytest.mark.parametrize("score", [xref.SOFTMAX, xref.SIGMOID])
@pytest.mark.parametrize("tokens,width,hidden,experts,chosen", [(1, 64, 96, 4, 2), (60, 100, 130, 6, 2), (300, 128, 64, 8, 3)])
def test_gradients(dtype, score, tokens, width, hidden, experts, chosen):
    from paper_2007_14178_amd.feed_forward import Experts
    layer = Experts(width, hidden, experts, chosen, dtype, score=score)
    layer.bias[0] = 0.2
    gen = torch.Generator(device="cuda").manual_seed(5)
    x, dy = (torch.randn(tokens, width, generator=gen, device="cuda").to(dtype) for _ in range(2))
    y, kept = layer.forward(x)
    dx, grads = layer.backward(dy, kept)
    assert set(grads) == set(layer.params)
    p = {k: v.double().requires_grad_() for k, v in layer.params.items()}
    xd = x.double().requires_grad_()
    want = plain(xd, p, kept[5], score, layer.eps)
    want.backward(dy.double())
    # a chain of at most twelve roundings to the type (n; logits; g, u; h; the pair; its gradient; dh; dg, du; dm; dlogits; dn; the result), each
    # within its unit
    unit = 12 * UNIT[dtype]
    assert off(y, want.detach()) <= unit and off(dx, xd.grad) <= unit
    for k, v in p.items():
        assert off(grads[k], v.grad) <= unit, k
    before = layer.bias.clone()
    layer.balance(kept, 0.5)
    counts = torch.bincount(kept[5].reshape(-1).long(), minlength=experts).float()
    assert torch.equal(layer.bias - before, 0.5 * torch.sign(counts.mean() - counts))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=str)
@pytest.mark.parametrize("tokens,width,hidden,group,zeros", [(1, 256, 512, 128, False), (2, 130, 300, 32, True), (40, 256, 512, 64, False), (700, 200, 333, 32, True)])
def test_served(dtype, tokens, width, hidden, group, zeros):
    """Against the layers on the values that their 4-bit weights stand for, so that what is compared are the served products' own roundings."""
    from paper_2007_14178_amd import binding as xb
    from paper_2007_14178_amd.feed_forward import Experts, FeedForward
    x = torch.randn(tokens, width, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(dtype)
    unit = 8 * UNIT[dtype]
    layer = FeedForward(width, hidden, dtype)
    served = layer.serve4(group, zeros)
    got = served(x)
    assert got.dtype is dtype
    p = {k: v.double() for k, v in layer.params.items()}
    for name in ("wg", "wu", "wd"):
        p[name] = xb.xnor_int4_dequantize(getattr(served, name)).double()
    n = normed(x.double(), p, layer.eps)
    g, u = n @ p["wg"].t(), n @ p["wu"].t()
    want = (g * torch.sigmoid(g) * u) @ p["wd"].t()
    # the norm's, the weights' (of many tokens), the block's, its output's and the sum's roundings; the last relative to x + branch
    assert float((got.double() - x.double() - want).norm()) <= unit * float(want.norm()) + UNIT[dtype] * float((x.double() + want).norm())

    mixture = Experts(width, hidden, 5, 2, dtype)
    served = mixture.serve4(group, zeros)
    got = served(x)
    p = {k: v.double() for k, v in mixture.params.items()}
    for name in ("wg", "wu", "wd"):
        stack = getattr(served, name)
        assert stack.q.shape[0] == 5
        p[name] = torch.stack([xb.xnor_int4_dequantize(xref.one(stack, e)).double() for e in range(5)])
    n, _, _ = xb.xnor_layer_norm_fwd(x, served.gamma, served.beta, served.eps)
    chosen, _ = xb.xnor_route_fwd(n @ served.router.t(), 2, served.bias, served.score)
    want = plain(x.double(), p, chosen, served.score, served.eps) - x.double()
    assert float((got.double() - x.double() - want).norm()) <= unit * float(want.norm()) + UNIT[dtype] * float((x.double() + want).norm())


def test_runs():
    """The example's training steps run, for the layer of several experts too."""
    from paper_2007_14178_amd import feed_forward as ff
    x = ff._train(ff.Experts(64, 64, 4, 2, seed=1), ff.FeedForward(64, 128, seed=2), 128, 64, 2)
    assert x.shape == (128, 64)
