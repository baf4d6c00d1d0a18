"""Routing to experts against its definition in 64 bits: whole numbers equal, weights and gradients within the bounds that experts_reference derives."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import dense_reference as ref  # noqa: E402
import experts_reference as xref  # noqa: E402

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
SOFTMAX, SIGMOID = xref.SOFTMAX, xref.SIGMOID


@pytest.fixture(scope="module")
def xb():
    from paper_2007_14178_amd import binding
    return binding


def rand(seed, *shape, dtype=F32, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(dtype).cuda()


def check(xb, logits, k, **how):
    names = {"kept": "groups_kept", "top": "group_top"}
    experts, weights = xb.xnor_route_fwd(logits, k, **{names.get(n, n): v for n, v in how.items()})
    want, w = xref.route(logits, k, **how)
    assert torch.equal(experts.cpu(), want)
    got = weights.cpu().double()
    assert torch.equal(got.isnan(), w.isnan())
    off = (got - w).abs().nan_to_num(0.0) - ref.rounding(w, F32).nan_to_num(0.0) - 1e-14 * w.abs().nan_to_num(0.0)
    assert not (off > 0).any()
    return experts, weights


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 8), (5, 2, 2), (17, 3, 1), (9, 60, 5), (8, 64, 32), (33, 65, 4), (16, 100, 6), (7, 128, 8), (5, 129, 3),
                                   (20, 256, 8), (3, 257, 7), (4, 500, 9), (2, 513, 8), (3, 1000, 32), (4, 1024, 8)], ids=str)
@pytest.mark.parametrize("score,renorm,with_bias,dtype", [(SOFTMAX, True, False, BF16), (SIGMOID, True, True, F32), (SOFTMAX, False, True, F16),
                                                          (SIGMOID, False, False, F32)], ids=str)
def test_choice(xb, T, E, k, score, renorm, with_bias, dtype):
    logits = rand(T + E, T, E, dtype=dtype, std=2.0)
    check(xb, logits, k, score=score, renorm=renorm, bias=rand(3, E, std=0.1) if with_bias else None, factor=2.5)


@pytest.mark.parametrize("E,groups,kept,top,k", [(256, 8, 4, 2, 8), (256, 8, 1, 1, 8), (60, 4, 2, 2, 6), (60, 60, 5, 1, 5), (64, 2, 1, 2, 32), (15, 5, 3, 2, 4),
                                                 (1024, 16, 3, 2, 12), (512, 512, 7, 2, 7), (120, 8, 8, 2, 8), (6, 3, 2, 2, 1), (320, 10, 3, 2, 8)], ids=str)
@pytest.mark.parametrize("score,with_bias,dtype", [(SIGMOID, True, F32), (SOFTMAX, False, BF16)], ids=str)
def test_groups(xb, E, groups, kept, top, k, score, with_bias, dtype):
    logits = rand(E + groups, 21, E, dtype=dtype, std=1.5)
    check(xb, logits, k, score=score, bias=rand(3, E, std=0.2) if with_bias else None, groups=groups, kept=kept, top=top)


@pytest.mark.parametrize("E", [7, 64, 200, 700])
def test_ties_and_what_is_never_chosen(xb, E):
    """Equal scores go by the lower index; -inf logits, biases of -inf or NaN; rows with nothing to choose, with NaN, with +inf."""
    logits = torch.randint(0, 3, (12, E), generator=torch.Generator().manual_seed(E)).float().cuda()
    for score in (SOFTMAX, SIGMOID):
        check(xb, logits, 5, score=score)
        rows = logits.clone()
        rows[0] = -math.inf
        rows[1, :-2] = -math.inf
        rows[2, 3] = math.nan
        rows[3, E - 1] = math.inf
        rows[4, ::2] = -math.inf
        rows[5] = torch.finfo(F32).min
        rows[6, 0] = torch.finfo(F32).max
        rows[7] = -800.0
        rows[8, 1:] = -800.0
        bias = torch.zeros(E, device="cuda")
        bias[1], bias[2], bias[4] = -math.inf, math.nan, 1e30
        for renorm in (True, False):
            check(xb, rows, 6, score=score, renorm=renorm)
            check(xb, rows, 4, score=score, renorm=renorm, bias=bias)
        if E % 4 == 0:
            check(xb, rows, 3, score=score, groups=4, kept=2, top=2)
            check(xb, rows, 3, score=score, groups=E // 2, kept=2, top=2, bias=bias)


def test_near_ties(xb):
    """Scores that fp32 does not tell apart, nor a probability in fp32: the choice is formed in 64 bits."""
    E = 64
    logits = torch.full((8, E), 12.0, device="cuda")
    for t in range(8):
        logits[t, 5 + t] = torch.nextafter(torch.tensor(12.0), torch.tensor(20.0))      # sigmoid(12) and its neighbour are one number in fp32
        logits[t, 50 - t] = torch.nextafter(logits[t, 5 + t].cpu(), torch.tensor(20.0))
    for score in (SOFTMAX, SIGMOID):
        experts, _ = check(xb, logits, 4, score=score)
        assert all(experts[t, 0] == 50 - t and experts[t, 1] == 5 + t for t in range(8))


def test_strides_and_no_tokens(xb):
    logits = rand(1, 9, 90)
    for view in (logits[:, 7:71], logits[:1, :64].expand(9, 64), logits[:0, :64]):
        experts = torch.full((view.shape[0] + 1, 3), -9, dtype=torch.int32, device="cuda")
        e, w = xb.xnor_route_fwd(view, 3, experts=experts[:view.shape[0]])
        want, _ = xref.route(view, 3)
        assert torch.equal(e.cpu(), want) and (experts[-1] == -9).all()
        dw = rand(2, view.shape[0], 3)
        held = torch.full((view.shape[0] + 1, 70), 4.0, device="cuda")
        for score, renorm in ((SOFTMAX, False), (SIGMOID, True)):
            dl, bound = xref.route_back(dw, view, e, score, renorm, 1.0, F32)
            ref.assert_within(xb.xnor_route_bwd(dw, view, e, score=score, renorm=renorm, dlogits=held[:view.shape[0], 3:67]), dl, bound, "dlogits")
        assert (held[-1] == 4.0).all() and (held[:, :3] == 4.0).all() and (held[:, 67:] == 4.0).all()


@pytest.mark.parametrize("T,k,E", [(0, 4, 8), (1, 1, 1), (1, 8, 64), (3, 32, 1024), (128, 8, 256), (129, 8, 256), (1025, 1, 7), (2000, 3, 60), (5000, 8, 100),
                                   (40000, 8, 64), (16384, 2, 1024), (200000, 5, 3)], ids=str)
def test_lists(xb, T, k, E):
    """Experts that none chose, one that most did, numbers that stand for none, the same expert twice in a token."""
    g = torch.Generator().manual_seed(T + E)
    experts = (torch.rand(T, k, generator=g).square() * (E + 1)).int() - (torch.rand(T, k, generator=g) < 0.05).int() * (E + 2)
    offsets = torch.full((E + 2,), -5, dtype=torch.int32, device="cuda")
    order = torch.full((T * k + 1,), -5, dtype=torch.int32, device="cuda")
    xb.xnor_route_lists(experts.cuda(), E, offsets=offsets[:E + 1], order=order[:T * k])
    if T * k <= 50000:
        want = xref.lists(experts, E)
    else:
        flat = experts.reshape(-1).long()
        fit = (flat >= 0) & (flat < E)
        at = torch.argsort(torch.where(fit, flat, E), stable=True)
        n = int(fit.sum())
        want = (torch.searchsorted(flat[at[:n]], torch.arange(E + 1)).int(), torch.cat((at[:n], torch.full((T * k - n,), -1))).int())
    assert torch.equal(offsets[:-1].cpu(), want[0]) and torch.equal(order[:-1].cpu(), want[1])
    assert offsets[-1] == -5 and order[-1] == -5


HOW = [(SOFTMAX, True), (SOFTMAX, False), (SIGMOID, True), (SIGMOID, False)]


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 8), (19, 60, 5), (8, 64, 32), (5, 100, 3), (33, 256, 8), (2, 257, 20), (3, 700, 8), (4, 1024, 32)], ids=str)
@pytest.mark.parametrize("score,renorm", HOW, ids=str)
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
def test_gradient(xb, T, E, k, score, renorm, dtype):
    logits, dw = rand(T + E, T, E, dtype=dtype, std=2.0), rand(4, T, k)
    experts, _ = xb.xnor_route_fwd(logits, k, score=score, renorm=renorm, factor=1.5)
    want, bound = xref.route_back(dw, logits, experts, score, renorm, 1.5, dtype)
    got = xb.xnor_route_bwd(dw, logits, experts, score=score, renorm=renorm, factor=1.5)
    assert got.dtype is dtype
    ref.assert_within(got, want, bound, "dlogits")
    assert torch.equal(got, xb.xnor_route_bwd(dw, logits, experts, score=score, renorm=renorm, factor=1.5))


@pytest.mark.parametrize("score,renorm", HOW, ids=str)
def test_gradient_against_autograd_and_differences(xb, score, renorm):
    T, E, k = 6, 20, 4
    logits, dw = rand(1, T, E), rand(2, T, k)
    experts, weights = xb.xnor_route_fwd(logits, k, score=score, renorm=renorm, factor=0.7)
    got = xb.xnor_route_bwd(dw, logits, experts, score=score, renorm=renorm, factor=0.7).cpu().double()
    l = logits.cpu().double().requires_grad_(True)
    (auto,) = torch.autograd.grad(xref.weights_of(l, experts.cpu(), score, renorm, 0.7), l, dw.cpu().double())
    _, bound = xref.route_back(dw, logits, experts, score, renorm, 0.7, F32)
    assert ((got - auto).abs() <= bound + 1e-12).all()
    # differences of the library's own weights: their rounding, 2^-24 of each, over the step, and the third derivative's share, its square (derivatives of a
    # score in its logit are below 1)
    step = 2.0 ** -6
    for e in range(0, E, 3):
        up, down = logits.clone(), logits.clone()
        up[:, e] += step
        down[:, e] -= step
        values = []
        for moved in (up, down):
            there, w = xb.xnor_route_fwd(moved, k, score=score, renorm=renorm, factor=0.7)
            values.append((there, (w * dw).double().sum(1)))
        same = ((values[0][0] == experts).all(1) & (values[1][0] == experts).all(1)).cpu()
        difference = ((values[0][1] - values[1][1]) / (2 * step)).cpu()
        reach = dw.abs().sum(1).double().cpu()
        assert ((difference - got[:, e]).abs() <= reach * (step * step + 2 * 2.0 ** -24 / step) + 1e-6)[same].all()
        assert same.any()


@pytest.mark.parametrize("score,renorm", HOW, ids=str)
def test_gradient_edges(xb, score, renorm):
    """Slots without an expert, an expert in several slots, tokens without any, logits of -inf, scores that fp32 does not hold."""
    T, E, k = 8, 30, 5
    logits, dw = rand(1, T, E, std=3.0), rand(2, T, k)
    logits[:, 4] = -math.inf
    logits[5] = -200.0 - torch.arange(E, device="cuda")
    logits[6] = 90.0 + torch.arange(E, device="cuda") / 4
    experts, _ = xb.xnor_route_fwd(logits, k, score=score, renorm=renorm)
    experts[0] = -1
    experts[1, 2], experts[1, 4] = -1, E
    experts[2, 3] = experts[2, 0]
    want, bound = xref.route_back(dw, logits, experts, score, renorm, 1.0, F32)
    got = xb.xnor_route_bwd(dw, logits, experts, score=score, renorm=renorm)
    ref.assert_within(got, want, bound, "dlogits")
    assert (got[0] == 0).all() and (got[logits == -math.inf] == 0).all()


def test_gradient_replayed_beside_an_eager_one(xb):
    T, E, k = 40, 64, 6
    logits, dw = rand(1, T, E, dtype=BF16), rand(2, T, k)
    out = torch.empty_like(logits)
    experts, _ = xb.xnor_route_fwd(logits, k)
    xb.xnor_route_bwd(dw, logits, experts)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chosen, _ = xb.xnor_route_fwd(logits, k, experts=experts)
        xb.xnor_route_bwd(dw, logits, chosen, dlogits=out)
    for seed in range(3, 7):
        logits.copy_(rand(seed, T, E, dtype=BF16))
        chosen, _ = xb.xnor_route_fwd(logits, k)
        eager = xb.xnor_route_bwd(dw, logits, chosen)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager, out) and torch.equal(chosen, experts)
