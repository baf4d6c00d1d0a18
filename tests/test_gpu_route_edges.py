"""Routing where a limit lies: numbers of experts about which the lists' shared memory passes a workgroup's default, scores that leave 64 bits."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import dense_reference as ref  # noqa: E402
import experts_reference as xref  # noqa: E402

pytestmark = pytest.mark.gpu

SOFTMAX, SIGMOID = xref.SOFTMAX, xref.SIGMOID


@pytest.fixture(scope="module")
def xb():
    from paper_2007_14178_amd import binding
    return binding


@pytest.mark.parametrize("E", [480, 481, 482, 511, 1023])
@pytest.mark.parametrize("T,k", [(100, 3), (3000, 2)])
def test_lists_at_the_default_limit(xb, T, k, E):
    """16 words of 8 bytes and two of 4 for each expert, and 128 bytes beside them: 64 KB are passed from 481 experts on."""
    experts = torch.randint(-1, E + 1, (T, k), generator=torch.Generator().manual_seed(E), dtype=torch.int32)
    offsets, order = xb.xnor_route_lists(experts.cuda(), E)
    want = xref.lists(experts, E)
    assert torch.equal(offsets.cpu(), want[0]) and torch.equal(order.cpu(), want[1])


def shares(logits, chosen):
    """A softmax's weights divided by their sum: the softmax of the chosen logits alone."""
    return torch.softmax(logits.gather(1, chosen.long()), 1)


@pytest.mark.parametrize("E", [20, 64, 300, 700])
@pytest.mark.parametrize("below", [100.0, 740.0, 800.0, 3000.0])
def test_shares_far_below_the_largest(xb, E, below):
    """Experts that a bias puts before the one with the largest logit, whose softmax 64 bits do not hold: their weights are the shares that they have of one
    another, and the gradient is that of these weights."""
    k, T = 3, 6
    logits = torch.randn(T, E, generator=torch.Generator().manual_seed(E)).cuda()
    logits[:, 5:9] -= below
    bias = torch.zeros(E, device="cuda")
    bias[5:9] = 2.0
    experts, weights = xb.xnor_route_fwd(logits, k, bias, SOFTMAX)
    assert ((experts >= 5) & (experts < 9)).all()
    l = logits.cpu().double().requires_grad_(True)
    want = shares(l, experts.cpu())
    # (64 bits, rounded once)
    assert ((weights.cpu().double() - want).abs() <= ref.rounding(want.detach(), torch.float32) + 1e-13).all()
    dw = torch.randn(T, k, generator=torch.Generator().manual_seed(1)).cuda()
    (grad,) = torch.autograd.grad(want, l, dw.cpu().double())
    got = xb.xnor_route_bwd(dw, logits, experts, score=SOFTMAX).cpu().double()
    # shares by fp32 exponentials of differences (of at most 16, rounded by 2^-24 of the logits), sums and products of k: 64 + 4 max |logit| units, as elsewhere
    reach = torch.zeros_like(grad).scatter_(1, experts.cpu().long(), want.detach() * (dw.cpu().abs().double() + (dw.cpu().abs().double() * want.detach()).sum(1, keepdim=True)))
    assert ((got - grad).abs() <= (64.0 + 4.0 * 16.0) * ref.U * reach).all()
    assert (got.abs().amax(1) > 0).all()


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("E", [20, 300])
def test_sigmoids_that_64_bits_do_not_hold(xb, E, renorm):
    """Where all of a token's scores are 0 its weights are constant 0, and so is their gradient; where one is not, the others' share is 0; above -709 shares are
    what they are."""
    k = 4
    logits = torch.randn(7, E, generator=torch.Generator().manual_seed(E)).cuda()
    logits[0] = -800.0
    logits[1] = -710.0 - torch.arange(E, device="cuda")
    logits[2] = -1e30
    logits[3] = -900.0
    logits[3, 7] = -5.0
    logits[4] = -700.0 - torch.arange(E, device="cuda") / 64
    logits[5] = -709.5
    experts, weights = xb.xnor_route_fwd(logits, k, None, SIGMOID, renorm=renorm)
    want, w = xref.route(logits, k, None, SIGMOID, renorm=renorm)
    assert torch.equal(experts.cpu(), want)
    assert ((weights.cpu().double() - w).abs() <= ref.rounding(w, torch.float32) + 1e-13).all()
    dw = torch.randn(7, k, generator=torch.Generator().manual_seed(2)).cuda()
    got = xb.xnor_route_bwd(dw, logits, experts, score=SIGMOID, renorm=renorm)
    assert torch.isfinite(got).all()
    assert (weights[:3] == 0).all() and (got[:3] == 0).all()
    if renorm:
        assert (weights[4:6] > 0).all() and (got[4:6].abs().amax(1) > 0).all()
        l = logits.cpu().double().requires_grad_(True)
        # (the shares of sigmoids this small are those of exponentials: 1 - p is 1)
        (grad,) = torch.autograd.grad(shares(l[4:6], experts[4:6].cpu()), l, dw[4:6].cpu().double())
        reach = dw[4:6].abs().sum(1, keepdim=True).cpu().double()
        assert ((got[4:6].cpu().double() - grad[4:6]).abs() <= (64.0 + 4.0 * 16.0) * ref.U * reach).all()
