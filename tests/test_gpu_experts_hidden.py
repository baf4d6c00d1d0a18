"""What the experts' blocks hold between their two products: tokens, levels and scales are whole numbers or powers of two, so that every sum is exact in
fp32 and outputs are compared by equality, whatever order the sums are formed in."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import dense_reference as ref  # noqa: E402
import experts_reference as xref  # noqa: E402

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def xb():
    from paper_2007_14178_amd import binding
    return binding


def whole(gen, most, *shape, dtype=BF16):
    return torch.randint(-most, most + 1, shape, generator=gen).to(dtype).cuda()


def stack(xb, gen, E, rows, cols, group, zeros, scale_dtype):
    """All levels, scales of 1, levels behind the last column too."""
    words, groups = (cols + 7) // 8, (cols + group - 1) // group
    q = torch.randint(0, 256, (E, rows, words * 4), generator=gen, dtype=torch.uint8).cuda()
    zero = torch.randint(0, 16, (E, groups, rows), generator=gen, dtype=torch.uint8).cuda() if zeros else None
    return xb.Int4(q, torch.ones(E, groups, rows, dtype=scale_dtype, device="cuda"), zero, cols, group)


def definition(x, chosen, share, wg, wu, wd):
    """(outputs, the largest hidden value, the largest sum of terms' magnitudes, the bound's sums) in 64 bits, relu."""
    x, share = x.cpu().double(), share.double()
    y = torch.zeros(x.shape[0], wd.rows).double()
    reach, largest = torch.zeros_like(y), 0.0
    for e in range(wg.q.shape[0]):
        g, u, d = (xref.values(xref.one(w, e))[0] for w in (wg, wu, wd))
        for s in range(chosen.shape[1]):
            rows = (chosen[:, s] == e).nonzero()[:, 0]
            h = (x[rows] @ g.t()).clamp(min=0.0) * (x[rows] @ u.t())
            largest = max(largest, float(h.abs().amax()) if h.numel() else 0.0)
            y[rows] += share[rows, s, None] * (h @ d.t())
            # (32 more for each level: what any form of a product with it may pass through a sum)
            reach[rows] += share[rows, s, None] * (h.abs() @ (d.abs() + 32.0).t())
    return y, largest, reach


def case(xb, T, k, E, K, F, N, group, zeros, dtype, scale_dtype, most):
    gen = torch.Generator().manual_seed(T + K)
    x = whole(gen, most, T, K, dtype=dtype)
    chosen = torch.rand(T, E, generator=gen).argsort(1)[:, :k].int()
    share = 2.0 ** torch.randint(-1, 1, (T, k), generator=gen).float()
    w = (stack(xb, gen, E, F, K, group, zeros, scale_dtype), stack(xb, gen, E, F, K, group, zeros, scale_dtype),
         stack(xb, gen, E, N, F, group, zeros, scale_dtype))
    return x, chosen, share, w


# pairs by themselves; lists of 16, 32, 64 and 128 pairs of an expert at a time
SIZES = [(1, 4, 64, 44, 33, 50), (5, 2, 16, 44, 40, 33), (30, 2, 4, 44, 33, 50), (60, 2, 4, 40, 36, 130), (110, 2, 4, 44, 33, 40), (300, 2, 3, 44, 33, 129)]


@pytest.mark.parametrize("T,k,E,K,F,N", SIZES, ids=str)
@pytest.mark.parametrize("dtype,scale_dtype,group,zeros,out_dtype", [
    (BF16, BF16, 128, False, BF16), (BF16, F32, 32, True, F32), (F16, F16, 32, True, F16), (F16, BF16, 64, False, BF16), (F16, F16, 128, False, F32)], ids=str)
def test_hidden_values_of_sixteen_bits(xb, T, k, E, K, F, N, dtype, scale_dtype, group, zeros, out_dtype):
    """Hidden values up to 2^16, which neither of the tokens' types holds, come through the second product as they are."""
    x, chosen, share, w = case(xb, T, k, E, K, F, N, group, zeros, dtype, scale_dtype, 1 if zeros else 2)
    want, largest, reach = definition(x, chosen, share, *w)
    assert 2.0 ** 11 < largest < 2.0 ** 16 and float(reach.max()) < 2.0 ** 23
    got = xb.xnor_int4_experts(x, chosen.cuda(), share.cuda(), *w, act=ref.RELU, out_dtype=out_dtype)
    assert torch.equal(got.cpu(), want.float().to(out_dtype))


@pytest.mark.parametrize("T,k,E,K,F,N", [(5, 2, 16, 16, 4, 20), (30, 2, 4, 16, 4, 20), (110, 2, 4, 16, 4, 20), (300, 2, 3, 16, 4, 20)], ids=str)
def test_hidden_values_past_f16(xb, T, k, E, K, F, N):
    """Blocks' outputs above f16's largest value: exact for fp32 outputs, within two terms' rounding for bf16 ones, whose 16 bits hold 2^-16 of a value."""
    x, chosen, share, w = case(xb, T, k, E, K, F, N, 32, False, F16, F16, 15)
    want, largest, reach = definition(x, chosen, share, *w)
    assert 2.0 ** 16 < largest < 2.0 ** 24 and float(reach.max()) < 2.0 ** 24 * 4
    got = xb.xnor_int4_experts(x, chosen.cuda(), share.cuda(), *w, act=ref.RELU, out_dtype=F32)
    # (sums up to 2^24 in steps of a half may be rounded; each of the sum's 4 hidden values, 2 slots and 3 terms once at most, where magnitudes reach that far)
    ref.assert_within(got, want, torch.where(reach < 2.0 ** 23, 0.0, 32 * ref.U * reach), "y")
    got = xb.xnor_int4_experts(x, chosen.cuda(), share.cuda(), *w, act=ref.RELU, out_dtype=BF16)
    ref.assert_within(got, want, 2.0 ** -16 * reach + 32 * ref.U * reach + ref.rounding(want, BF16) * 1.01, "y")


@pytest.mark.parametrize("T,k,E", [(1, 8, 32), (40, 2, 6), (300, 2, 3)], ids=str)
def test_as_far_from_the_definition_as_one_rounding(xb, T, k, E):
    """Outputs in bf16 are no further from 64 bits, in the root of the squares' sum, than those of values rounded once.  With d the error
    before the rounding, |round(y + d) - y| <= |round(y) - y| + 2 |d|, as a rounding goes to the nearest."""
    K, F, N, dtype = 256, 64, 300, BF16
    gen = torch.Generator().manual_seed(T)
    x = torch.randn(T, K, generator=gen).to(dtype).cuda()
    chosen = torch.rand(T, E, generator=gen).argsort(1)[:, :k].int()
    share = torch.rand(T, k, generator=gen)
    w = [m._replace(scale=m.scale * (torch.rand(m.scale.shape, generator=gen) + 0.5).to(m.scale.dtype).cuda() * 0.2 / m.cols ** 0.5)
         for m in (stack(xb, gen, E, F, K, 64, True, BF16), stack(xb, gen, E, F, K, 64, True, BF16), stack(xb, gen, E, N, F, 64, True, BF16))]
    want, off = torch.zeros(T, N).double(), torch.zeros(T, N).double()
    for e in range(E):
        g, u, d = (xref.one(m, e) for m in w)
        for s in range(k):
            rows = (chosen[:, s] == e).nonzero()[:, 0]
            if rows.numel() == 0:
                continue
            a, b = (x[rows.cuda()].cpu().double() @ xref.values(m)[0].t() for m in (g, u))
            h, v = a * torch.sigmoid(a) * b, share[rows, s, None].double()
            want[rows] += v * (h @ xref.values(d)[0].t())
            # 2^-16 of a hidden value is two terms' rounding; the activation's, 2^-18 of it, and the sums', of a few 2^-24 of their terms, are less
            off[rows] += v * (h.abs() @ xref.values(d)[0].abs().t()) * (2.0 ** -16 + 2.0 ** -18)
    got = xb.xnor_int4_experts(x, chosen.cuda(), share.cuda(), *w).cpu().double()
    once = (want.to(dtype).double() - want).norm()
    assert float(once + 2.0 * off.norm()) < 1.25 * float(once)
    assert float((got - want).norm()) <= float(once + 2.0 * off.norm())


@pytest.mark.parametrize("T", [2, 60, 300])
def test_hidden_values_that_are_not_finite(xb, T):
    """An infinite or NaN hidden value reaches the outputs that it would in products of the values, as infinity or NaN, and no other token's."""
    K, F, N = 8, 40, 30
    gen = torch.Generator().manual_seed(1)
    x, chosen, share, w = case(xb, T, 1, 1, K, F, N, 32, False, BF16, F32, 1)
    x[0] = float("inf")
    got = xb.xnor_int4_experts(x, chosen.cuda(), share.cuda(), *w, act=ref.RELU, out_dtype=F32).cpu().double()
    g, u, d = (xref.values(xref.one(m, 0))[0] for m in w)
    h = (x.cpu().double() @ g.t()).clamp(min=0.0) * (x.cpu().double() @ u.t())
    want = share.double() * (h[:, None, :] * d[None]).sum(2)
    assert not torch.isfinite(want[0]).any() and torch.isfinite(want[1:]).all()
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got[1:], want[1:])
    # one column alone infinite, with a sign: inf where its level is above the zero point, -inf below, NaN at it
    x[0] = 0.0
    w[0].scale[:, :, 3], w[1].scale[:, :, 3] = 2.0 ** 100, 2.0 ** 100
    x[0, :] = 1.0
    h = (x.cpu().double() @ xref.values(xref.one(w[0], 0))[0].t()).clamp(min=0.0) * (x.cpu().double() @ xref.values(xref.one(w[1], 0))[0].t())
    h = h.float().double()          # (past fp32: infinite)
    want = share.double() * (h[:, None, :] * d[None]).sum(2)
    got = xb.xnor_int4_experts(x, chosen.cuda(), share.cuda(), *w, act=ref.RELU, out_dtype=F32).cpu().double()
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.isinf(), want.isinf())
    assert torch.equal(got[got.isinf()] > 0, want[want.isinf()] > 0)
