"""Products with 4-bit weights of whole numbers: tokens are integers (or powers of two), scales powers of two, so that every sum is exact in fp32 and outputs are
compared by equality, whatever order the sums are formed in."""
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


def matrix(xb, gen, N, K, group, zeros, dtype, scale=1.0):
    """All levels, those behind the last column too."""
    groups = (K + group - 1) // group
    q = torch.randint(0, 256, (N, (K + 7) // 8 * 4), generator=gen, dtype=torch.uint8).cuda()
    zero = torch.randint(0, 16, (groups, N), generator=gen, dtype=torch.uint8).cuda() if zeros else None
    return xb.Int4(q, torch.full((groups, N), scale, dtype=dtype, device="cuda"), zero, K, group)


@pytest.mark.parametrize("M,N,K", [(2, 40, 128), (40, 50, 300), (100, 1100, 4224), (140, 300, 4160)], ids=str)
@pytest.mark.parametrize("group", [32, 128])
def test_tokens_near_the_largest_value(xb, M, N, K, group):
    """Levels 15 above their zero point, tokens of 2^127: with scales of 2^-30 the outputs are far from infinite, and so is every sum on their way."""
    w = matrix(xb, torch.Generator().manual_seed(1), N, K, group, True, F32, 2.0 ** -30)
    w.q.fill_(255), w.zero.fill_(0)
    x = torch.full((M, K), 2.0 ** 127, dtype=BF16, device="cuda")
    x[1] = -x[1]
    want = torch.full((M, N), 2.0 ** 97 * 15 * K)
    want[1] = -want[1]
    assert torch.equal(xb.xnor_int4_linear(x, w, out_dtype=F32).cpu(), want)


@pytest.mark.parametrize("M", [1, 5, 20, 40, 64, 300])
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True)], ids=str)
@pytest.mark.parametrize("dtype", [F16, BF16], ids=str)
def test_a_token_that_meets_zero_points_costs_nothing(xb, M, group, zeros, dtype):
    """Tokens far larger than the others at columns where every level is its zero point: their products are 0, and the others' sums keep all their bits."""
    N, K = 130, 300
    gen = torch.Generator().manual_seed(M)
    x = torch.randint(-2, 3, (M, K), generator=gen).to(dtype)
    levels = torch.randint(0, 16, (N, K), generator=gen, dtype=torch.uint8)
    groups = (K + group - 1) // group
    zero = torch.randint(0, 16, (groups, N), generator=gen, dtype=torch.uint8)
    for c in (7, 100, 299):
        x[:, c] = 2.0 ** (15 if dtype is F16 else 40)
        levels[:, c] = zero[c // group] if zeros else 8
    x = x.cuda()
    w = xb.Int4(xb.xnor_int4_pack(levels.cuda()), torch.ones(groups, N, dtype=dtype, device="cuda"), zero.cuda() if zeros else None, K, group)
    want = x.cpu().double() @ xref.values(w)[0].t()
    assert 0 < float(want.abs().max()) < 2.0 ** 15
    assert torch.equal(xb.xnor_int4_linear(x, w, out_dtype=F32).cpu().double(), want)
    got = xb.xnor_int4_gated(x, w, w, ref.RELU, out_dtype=F32).cpu().double()
    assert torch.equal(got, (want.clamp(min=0.0) * want).float().double())
