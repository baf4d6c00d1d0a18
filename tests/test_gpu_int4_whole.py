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


# few tokens by every kernel; tiles; tiles in shares of the contraction; contractions that end inside a step, behind very long ones too
SIZES = [(1, 50, 1), (13, 50, 33), (20, 50, 129), (33, 40, 41), (40, 2050, 65), (64, 9000, 39), (64, 300, 1031), (128, 50, 393), (65, 300, 30000), (129, 1100, 2600),
         (200, 1024, 4095), (1000, 520, 1100), (8200, 1030, 70), (90, 1, 5000000), (40, 1030, 8200), (33, 2050, 8195), (300, 1024, 4096), (40000, 300, 60), (3000, 70, 520)]


def marked(K, gen):
    """Columns of a contraction that hold tokens: all of a short one; of a long one its ends, both sides of every place where a share of it may begin, and
    others as they fall."""
    if K <= 40000:
        return torch.arange(K)
    at = [torch.arange(200), torch.arange(K - 200, K), torch.randint(0, K, (20000,), generator=gen)]
    whole = K // 64
    for parts in range(2, 17):
        for i in range(1, parts):
            at.append(torch.arange(-70, 70) + whole * i // parts * 64)
    return torch.unique(torch.cat(at))


@pytest.mark.parametrize("M,N,K", SIZES, ids=str)
@pytest.mark.parametrize("dtype,scale_dtype,group,zeros,gated", [(BF16, BF16, 128, False, False), (BF16, F32, 32, True, False), (F16, F16, 64, True, False),
                                                                (F16, F32, 32, False, True), (BF16, F16, 64, True, True), (F16, BF16, 128, True, False)], ids=str)
def test_equal(xb, M, N, K, dtype, scale_dtype, group, zeros, gated):
    """With the workspace and without.  What is compared would differ were one step of the contraction left out, the last one or a share's first among them."""
    gated = gated and K < 100000
    gen = torch.Generator().manual_seed(M + K)
    at = marked(K, gen)
    x = torch.zeros(M, K, dtype=dtype, device="cuda")
    # (-1, 0 and 1 in contractions whose sums would pass 2^24 otherwise)
    most = 2 if K <= 2600 else 1
    x[:, at.cuda()] = torch.randint(-most, most + 1, (M, len(at)), generator=gen).to(dtype).cuda()
    ws = [matrix(xb, gen, N, K, group, zeros, scale_dtype) for _ in range(2 if gated else 1)]
    xd = x[:, at.cuda()].cpu().double()
    values = [xref.levels_of(w.q, K)[:, at].double() - (8.0 if w.zero is None else w.zero.cpu().double()[at // group].t()) for w in ws]
    assert 15.0 * most * len(at) < 2.0 ** 24
    # (all outputs of the definition, or those of some tokens where that takes long)
    rows = torch.arange(M) if M * N * len(at) < 1 << 31 else torch.randint(0, M, (200,), generator=gen)
    sums = [xd[rows] @ v.t() for v in values]
    want = (sums[0].clamp(min=0.0) * sums[1]).float() if gated else sums[0].float()
    # each step that holds tokens changes some output
    steps = at // 64
    for step in {int(steps[0]), int(steps[-1]), int(steps[len(at) // 2]), int(steps[len(at) // 3])}:
        mine = steps == step
        assert (xd[rows][:, mine] @ values[0][:, mine].t()).any()
    call = (lambda space: xb.xnor_int4_gated(x, *ws, ref.RELU, out_dtype=F32, workspace=space)) if gated else (
        lambda space: xb.xnor_int4_linear(x, ws[0], out_dtype=F32, workspace=space))
    for space in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
        got = call(space)
        assert torch.equal(got[rows.cuda()].cpu(), want)
