"""The dense operators at the edges of what they take: no rows, more rows than a launch's workgroups hold at a time, operands off 16 bytes and
outputs in wider buffers, widths at which another kernel takes over, equal rows in different places.  Tolerances are the bounds that
dense_reference derives."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import dense_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
EPS = 1e-5


@pytest.fixture(scope="module")
def xb():
    from paper_2007_14178_amd import binding
    return binding


def rand(seed, *shape, dtype=F32, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(dtype).cuda()


@pytest.mark.parametrize("dtype,cols", [(F32, 33), (F32, 9000), (F16, 16384), (F16, 16392), (BF16, 20000), (BF16, 70001)], ids=str)
def test_norm_backward_without_rows(xb, dtype, cols):
    """No rows, short ones or long: gradients of the parameters are zeros, whatever their memory held."""
    x, none = torch.empty(0, cols, dtype=dtype, device="cuda"), torch.empty(0, device="cuda")
    gamma = rand(1, cols)
    dgamma, dbeta = torch.full((cols,), 5.0, device="cuda"), torch.full((cols,), float("nan"), device="cuda")
    dx, dg, db = xb.xnor_layer_norm_bwd(x, x, gamma, none, none, dgamma=dgamma, dbeta=dbeta)
    assert dx.shape == (0, cols) and dg is dgamma and db is dbeta
    assert (dgamma == 0).all() and (dbeta == 0).all()


def test_norm_backward_of_millions_of_long_rows(xb):
    """More long rows than a launch of 1024 threads each has room for (2^22 such workgroups are 2^32 threads): one row for all, so that
    all of dx's rows are alike."""
    rows, cols = (1 << 22) + 3, 16392
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < rows * cols * 2 + (8 << 30):
        pytest.skip("needs 145 GB of device memory")
    x, dy, gamma = rand(1, 1, cols, dtype=BF16), rand(2, 1, cols, dtype=BF16), rand(3, cols)
    _, mean, rstd = xb.xnor_layer_norm_fwd(x, None, None, EPS)
    want, bound = ref.norm_back(dy, x, gamma, mean, rstd, BF16, F32)
    dx, _, _ = xb.xnor_layer_norm_bwd(dy.expand(rows, cols), x.expand(rows, cols), gamma, mean.repeat(rows), rstd.repeat(rows), want_params=False)
    ref.assert_within(dx[:1], want[0], bound[0], "dx")
    for part in dx.split(1 << 18):
        assert torch.equal(part, dx[:1].expand_as(part))
    del dx, part
    torch.cuda.empty_cache()


def test_one_row_in_wider_buffers(xb):
    """One token's g and u, and one hidden unit's weight gradients, each in a buffer of its own width."""
    K, F = 72, 40
    x, wg, wu = rand(1, 1, K, dtype=BF16), rand(2, F, K, dtype=BF16, std=0.1), rand(3, F, K, dtype=BF16, std=0.1)
    held = [torch.full((1, F + spare), 5.0, dtype=BF16, device="cuda") for spare in (8, 3, 60)]
    got = xb.xnor_gated_fwd(x, wg, wu, h=held[0][:, :F], g=held[1][:, :F], u=held[2][:, :F], want_pre=True)
    want, bound = ref.gated(x, wg, wu, ref.SILU, BF16)
    for t, w, e, name in zip(got, want, bound, "hgu"):
        ref.assert_within(t, w, e, name)
    assert all((t[:, F:] == 5.0).all() for t in held)
    x, wg, wu = rand(4, 9, K, dtype=BF16), rand(5, 1, K, dtype=BF16), rand(6, 1, K, dtype=BF16)
    dh, g, u = (rand(7 + i, 9, 1, dtype=BF16) for i in range(3))
    held = [torch.full((1, K + spare), 5.0, dtype=BF16, device="cuda") for spare in (8, 33)]
    got = xb.xnor_gated_bwd(dh, x, wg, wu, g, u, dwg=held[0][:, :K], dwu=held[1][:, :K])
    want, bound = ref.gated_back(dh, x, wg, wu, g, u, ref.SILU, BF16)
    for t, w, e, name in zip(got, want, bound, ("dx", "dwg", "dwu")):
        ref.assert_within(t, w, e, name)
    assert all((t[:, K:] == 5.0).all() for t in held)


@pytest.mark.parametrize("shifted", ["x", "wg", "wu", "all"])
def test_gated_forward_off_16_bytes(xb, shifted):
    """Strides of whole chunks, but operands that start a value behind one: copied, where a workspace allows it, as odd strides are."""
    M, F, K = 300, 400, 3008
    need = xb.xnor_gated_fwd_workspace_bytes(M, F, K, K + 1, K)
    assert need > 0

    def operand(seed, rows, name, **kw):
        off = 1 if shifted in (name, "all") else 0
        return rand(seed, rows, K + 8, dtype=F16, **kw)[:, off:off + K]
    x, wg, wu = operand(1, M, "x"), operand(2, F, "wg", std=0.02), operand(3, F, "wu", std=0.02)
    want, bound = ref.gated(x, wg, wu, ref.GELU, F16)
    workspace = torch.full((need,), 77, dtype=torch.uint8, device="cuda")
    for ws in (None, workspace):
        got = xb.xnor_gated_fwd(x, wg, wu, ref.GELU, want_pre=True, workspace=ws)
        for t, w, e, name in zip(got, want, bound, "hgu"):
            ref.assert_within(t, w, e, name)
    rows = workspace[:2 * M * K].view(torch.float16).view(M, K)         # x's copy
    assert torch.equal(rows, x)


@pytest.mark.parametrize("M,K", [(1, 300), (2, 1037), (3, 2000), (8, 256), (9, 1280), (16, 77)])
def test_int8_linear_wide(xb, M, K):
    """A few tokens on wide layers: with the workspace they are quantised once, without one by every part of the product, and on both
    sides of the width where that changes the values are the same."""
    x, bias = rand(M, M, K, dtype=BF16), rand(9, 20000)
    w, sw = xb.xnor_int8_quantize(rand(2, 20000, K))
    q, s = ref.quantize(x)
    for N in (4096, 4097, 8192, 8193, 16385, 20000):
        out = xb.xnor_int8_linear(x, w[:N], sw[:N].contiguous(), bias[:N].contiguous())
        want, bound = ref.int8_matmul(q, s, w[:N], sw[:N], bias[:N], BF16)
        ref.assert_within(out, want, bound, f"N {N}")
        need = xb.xnor_int8_linear_layer_workspace_bytes(M, N, K)
        for nbytes in (16, max(16, need)):
            workspace = torch.full((nbytes,), 99, dtype=torch.uint8, device="cuda")
            again = xb.xnor_int8_linear(x, w[:N], sw[:N].contiguous(), bias[:N].contiguous(), workspace=workspace)
            assert torch.equal(out, again)
            if nbytes == need:
                assert torch.equal(workspace[:need - 4 * M].view(torch.int8).view(M, -1)[:, :K].cpu(), q)
            else:
                assert (workspace == 99).all()
    x[0, K // 2] = float("nan")
    assert xb.xnor_int8_linear(x, w, sw)[0].isnan().all() and not xb.xnor_int8_linear(x, w, sw)[1:].isnan().any()


def repeated(seed, rows, cols, dtype, std=1.0, period=61):
    """`period` rows over and over (61 shares no factor with a tile, a grid or a workgroup's rows)."""
    return rand(seed, period, cols, dtype=dtype, std=std).repeat((rows + period - 1) // period, 1)[:rows]


def assert_repeats(outputs, what, period=61):
    for i, t in enumerate(outputs):
        assert torch.equal(t[:-period], t[period:]), f"{what}: output {i} differs in {int((t[:-period] != t[period:]).sum())} of {t.numel()} values"


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("rows,cols", [(40003, 512), (35001, 264), (35001, 263), (12501, 2048), (9001, 4096), (9002, 8192), (3001, 16384), (3001, 1111), (1001, 40000)])
def test_rows_do_not_depend_on_their_place(xb, dtype, rows, cols):
    """The same row gives the same bits wherever it stands among the others."""
    x, dy = repeated(1, rows, cols, dtype), repeated(2, rows, cols, dtype)
    assert_repeats(xb.xnor_int8_quantize(x), "quantise")
    for p_dtype in {F32, dtype}:
        gamma, beta = (1.0 + rand(5, cols, std=0.2)).to(p_dtype), rand(6, cols, dtype=p_dtype)
        assert_repeats(xb.xnor_layer_norm_fwd_int8(x, gamma, beta, EPS), "quantised norm")
        y, mean, rstd = xb.xnor_layer_norm_fwd(x, gamma, beta, EPS)
        assert_repeats((y, mean, rstd), "norm")
        assert_repeats(xb.xnor_layer_norm_bwd(dy, x, gamma, mean, rstd)[:1], "norm backward")


@pytest.mark.parametrize("dtype", [F16, BF16], ids=str)
@pytest.mark.parametrize("M,F,K", [(64, 200, 256), (500, 333, 328), (500, 333, 331), (1300, 900, 1000), (4100, 4096, 1104), (128, 640, 4096)])
def test_tokens_do_not_depend_on_their_place(xb, dtype, M, F, K):
    """The same token gives the same bits wherever it stands, in a product's tile or in another one."""
    period = 61 if M > 64 else 13
    a, sa = xb.xnor_int8_quantize(repeated(1, M, K, F32, period=period))
    (wg, sg), (wu, su) = xb.xnor_int8_quantize(rand(2, F, K, std=K ** -0.5)), xb.xnor_int8_quantize(rand(3, F, K, std=K ** -0.5))
    bias = rand(4, F)
    for out_dtype in (F32, dtype):
        assert_repeats([xb.xnor_int8_matmul(a, sa, wg, sg, bias, out_dtype=out_dtype)], "8-bit product", period)
        for kind in (ref.SILU, ref.GELU, ref.RELU):
            assert_repeats([xb.xnor_int8_gated(a, sa, wg, sg, wu, su, kind, out_dtype=out_dtype)], "8-bit gated", period)
    x = repeated(5, M, K, dtype, period=period)
    w = [rand(6 + i, F, K, dtype=dtype, std=K ** -0.5) for i in range(2)]
    dh, g, u = (repeated(8 + i, M, F, dtype, period=period) for i in range(3))
    for kind in (ref.SILU, ref.GELU, ref.RELU):
        assert_repeats(xb.xnor_gated_fwd(x, *w, kind, want_pre=True), "gated", period)
        assert_repeats(xb.xnor_gated_bwd(dh, x, *w, g, u, kind)[:1], "gated backward, dx", period)


def sampled(rows):
    """Rows of the first turns of a grid of 1024, 4096 and 16384 rows, and of each turn after, on both sides of where it begins."""
    at = {0, 1, 2, rows // 2, rows - 3, rows - 2, rows - 1}
    for grid in (1024, 4096, 16384):
        for turn in range(1, 10):
            at |= {turn * grid - 1, turn * grid, turn * grid + 1, turn * grid + 3}
    return torch.tensor(sorted(r for r in at if 0 <= r < rows))


@pytest.mark.parametrize("dtype", [F16, BF16], ids=str)
@pytest.mark.parametrize("rows,cols", [(40003, 512), (35001, 264), (12501, 2048), (9001, 4096), (9002, 8192), (2501, 8192), (2501, 16384)])
def test_rows_in_turns(xb, dtype, rows, cols):
    """More rows of whole 16-byte chunks than a launch holds at a time: each workgroup takes several, with two on their way, up to an odd
    number of turns and a last one that some workgroups have no row for.  Rows differ in size by powers of two, so that one row's
    sums or maximum in another's place show."""
    x = rand(cols, 61, cols, dtype=dtype).repeat((rows + 60) // 61, 1)[:rows]          # (61 shares no factor with a grid)
    x = x * torch.exp2((torch.arange(rows, device="cuda") % 7 - 3).float())[:, None].to(dtype) + (torch.arange(rows, device="cuda") % 5)[:, None].to(dtype)
    gamma, beta = 1.0 + rand(5, cols, std=0.2), rand(6, cols)
    r = sampled(rows)
    some = x[r.cuda()]
    q, s = xb.xnor_int8_quantize(x)
    q0, s0 = ref.quantize(some)
    assert torch.equal(q[r.cuda()].cpu(), q0) and torch.equal(s[r.cuda()].cpu(), s0)
    got = xb.xnor_layer_norm_fwd(x, gamma, beta, EPS)
    want, bound = ref.norm(some, gamma, beta, EPS, dtype)
    for t, w, e, name in zip(got, want, bound, ("y", "mean", "rstd")):
        ref.assert_within(t[r.cuda()], w, e, name)
    q, s = xb.xnor_layer_norm_fwd_int8(x, gamma, beta, EPS)
    (y, _, _), (e, _, _) = ref.norm(some, gamma, beta, EPS, None)
    top, e_top = y.abs().amax(1), e.amax(1)
    ref.assert_within(s[r.cuda()], top / 127, e_top / 127 + 2 * ref.U * top / 127, "scale")
    level = s[r.cuda()].cpu().double()[:, None]
    ref.assert_within(q[r.cuda()].cpu().double() * level, y, 0.5 * level + e + 127 * 4 * ref.U * level, "levels")


@pytest.mark.parametrize("kind", [ref.SILU, ref.GELU])
@pytest.mark.parametrize("M,F,K", [(4090, 4081, 1104), (4096, 4096, 2000), (8150, 2040, 1168)])
def test_large_int8_gated_ends_inside_a_step(xb, kind, M, F, K):
    """Tiles of 256 x 256 on rows at multiples of 16 bytes, with a contraction that is no multiple of 128."""
    a, wg, wu = (torch.randint(-128, 128, (n, K + 16), generator=torch.Generator().manual_seed(K + i), dtype=torch.int32).to(torch.int8).cuda()[:, :K]
                 for i, n in enumerate((M, F, F)))
    sa, sg, su = rand(1, M).abs() * 0.01 + 1e-3, rand(2, F).abs() * 1e-3 + 1e-4, rand(3, F).abs() * 1e-3 + 1e-4

    def some(n):
        return torch.tensor(sorted({0, 1, 127, 128, 255, 256, 257, n // 2, n // 256 * 256 - 1, n - 2, n - 1}))
    for dtype in (F32, BF16):
        held = torch.full((M, F + 3), 5.0, dtype=dtype, device="cuda")
        h = xb.xnor_int8_gated(a, sa, wg, sg, wu, su, kind, h=held[:, :F])
        for r, c in ((some(M), torch.arange(F)), (torch.arange(M), some(F))):
            want, bound = ref.int8_gated(a[r], sa[r], wg[c], sg[c], wu[c], su[c], kind, dtype)
            ref.assert_within(h[r.cuda()][:, c.cuda()], want, bound, str(dtype))
        assert (held[:, F:] == 5.0).all()
