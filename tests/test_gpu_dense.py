"""The dense operators against their definitions in 64 bits: sizes around the tiles' edges, types, strides, rows that hold nothing
or what is not finite, long offsets, other streams, graphs.  Tolerances are the bounds that dense_reference derives."""
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


def ints(seed, rows, cols, spare=0):
    """int8 rows, the extremes -128 and 127 among them; `spare` values between rows that are none of theirs."""
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(-128, 128, (rows, cols + spare), generator=g, dtype=torch.int32).to(torch.int8)
    return t.cuda()[:, :cols]


def scales(seed, n):
    return rand(seed, n).abs() * 0.01 + 1e-3


def spaced(rows, cols, dtype, spare, fill):
    """An output whose rows have `spare` values behind them, all `fill`."""
    t = torch.full((rows, cols + spare), fill, dtype=dtype, device="cuda")
    return t, t[:, :cols]


# ---- quantisation ------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 64), (9, 513), (4, 1030), (2, 4096), (3, 9001), (2, 40000)])
def test_quantize(xb, dtype, rows, cols):
    x = rand(rows * cols, rows, cols, dtype=dtype)
    q, s = xb.xnor_int8_quantize(x)
    q0, s0 = ref.quantize(x)
    assert torch.equal(q.cpu(), q0) and torch.equal(s.cpu(), s0)
    # within half a level of the real value: two roundings of up to 127
    d = x.cpu().double() * (127.0 / x.cpu().double().abs().amax(1, keepdim=True))
    assert ((q.cpu().double() - d).abs() <= 0.5 + 127 * 2.1 * ref.U).all()


def test_quantize_special_rows(xb):
    for dtype in (F32, F16, BF16):
        x = rand(3, 9, 300, dtype=dtype)
        x[1] = 0.0
        x[2, 299] = float("nan")
        x[3, 0] = float("inf")
        x[4, 5] = float("-inf")
        x[5] = torch.finfo(dtype).max
        x[6] = torch.finfo(dtype).min
        x[7] *= 1e-7 if dtype is F16 else 2.0 ** -105
        q, s = xb.xnor_int8_quantize(x)
        q0, s0 = ref.quantize(x)
        assert torch.equal(q.cpu(), q0)
        assert torch.equal(s.cpu(), s0) or torch.equal(s.cpu()[~s0.isnan()], s0[~s0.isnan()]) and torch.equal(s.cpu().isnan(), s0.isnan())


# ---- 8-bit products ----------------------------------------------------------------------------------------------------

SIZES = [(1, 1, 1), (1, 17, 33), (1, 256, 128), (2, 3, 15), (3, 130, 1037), (15, 64, 16), (16, 65, 17), (17, 16, 127), (33, 48, 2048), (63, 257, 129),
         (64, 128, 640), (65, 130, 300), (128, 128, 128), (129, 300, 256), (257, 100, 1000), (300, 513, 384), (520, 260, 200)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_int8_matmul(xb, dtype, M, N, K):
    # rows of any alignment, and on a stride of 16 bytes
    for spare in (0, 5, (-K) % 16, (-K) % 16 + 16):
        a, b = ints(M + K, M, K, spare), ints(N * 7 + K, N, K, spare)
        sa, sb = scales(1, M), scales(2, N)
        bias = rand(4, N) if (M + N) % 2 else None
        held, out = spaced(M, N, dtype, 3, -7.0)
        xb.xnor_int8_matmul(a, sa, b, sb, bias, out=out)
        want, bound = ref.int8_matmul(a, sa, b, sb, bias, dtype)
        ref.assert_within(out, want, bound, f"spare {spare}")
        assert (held[:, N:] == -7.0).all()


def test_int8_matmul_largest_sum(xb):
    """K at its limit, all products 2^14: the sum is a multiple of 2^14 just below 2^31."""
    K = (1 << 17) - 1
    a = torch.full((2, K), -128, dtype=torch.int8, device="cuda")
    b = torch.full((3, K), -128, dtype=torch.int8, device="cuda")
    b[1] = 127
    one = torch.ones(3, device="cuda")
    out = xb.xnor_int8_matmul(a, one[:2].contiguous(), b, one)
    assert out[:, 0].tolist() == [float(K << 14)] * 2 and out[:, 1].tolist() == [float(torch.tensor(-128 * 127 * K, dtype=F32))] * 2


def test_int8_matmul_one_row_for_all_tokens(xb):
    a, b = ints(5, 1, 320).expand(70, 320), ints(6, 90, 320)
    sa, sb = scales(1, 70), scales(2, 90)
    want, bound = ref.int8_matmul(a, sa, b, sb, None, F32)
    ref.assert_within(xb.xnor_int8_matmul(a, sa, b, sb), want, bound, "stride 0")


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("M,N,K", [(1, 40, 1), (1, 512, 4096), (1, 90, 9000), (2, 1000, 300), (2, 70, 8192), (3, 50, 1), (7, 33, 1037), (8, 40, 2048), (9, 64, 2049), (16, 129, 512), (16, 48, 2000), (12, 70, 1000), (40, 96, 2000), (200, 130, 513)])
def test_int8_linear(xb, dtype, M, N, K):
    x, (w, sw) = rand(M, M, K + 3, dtype=dtype)[:, 1:K + 1], xb.xnor_int8_quantize(rand(N, N, K))
    bias = rand(9, N)
    q, s = ref.quantize(x)
    for out_dtype in (dtype, F32):
        want, bound = ref.int8_matmul(q, s, w, sw, bias, out_dtype)
        ref.assert_within(xb.xnor_int8_linear(x, w, sw, bias, out_dtype=out_dtype), want, bound, str(out_dtype))


def test_int8_linear_token_that_is_not_finite(xb):
    """It spoils its own outputs and no others."""
    for M in (2, 3, 13, 40, 100):
        x, (w, sw) = rand(1, M, 200), xb.xnor_int8_quantize(rand(2, 70, 200))
        clean = xb.xnor_int8_linear(x, w, sw)
        x[1, 7] = float("inf")
        out = xb.xnor_int8_linear(x, w, sw)
        assert out[1].isnan().all()
        keep = torch.arange(M, device="cuda") != 1
        assert torch.equal(out[keep], clean[keep])


# ---- layer norm --------------------------------------------------------------------------------------------------------

PAIRS = [(F32, F32), (F16, F32), (F16, F16), (BF16, F32), (BF16, BF16)]
NORM_SIZES = [(1, 1), (1, 2), (5, 3), (3, 64), (7, 255), (6, 513), (5, 1111), (3, 2048), (2, 4097), (3, 8200), (2, 20000), (2, 70001)]


def norm_inputs(rows, cols, dtype, p_dtype, spare=0):
    x = (rand(rows + cols, rows, cols + spare) * 2.0 + rand(cols, rows, 1) * 3.0).to(dtype)[:, :cols]
    return x, (1.0 + rand(5, cols, std=0.2)).to(p_dtype), rand(6, cols, dtype=p_dtype)


@pytest.mark.parametrize("dtype,p_dtype", PAIRS, ids=str)
@pytest.mark.parametrize("rows,cols", NORM_SIZES)
def test_norm_forward(xb, dtype, p_dtype, rows, cols):
    for spare in (0, 3):
        x, gamma, beta = norm_inputs(rows, cols, dtype, p_dtype, spare)
        for g, b in ((gamma, beta), (None, None), (gamma, None)):
            held, y = spaced(rows, cols, dtype, 5, 7.0)
            got = xb.xnor_layer_norm_fwd(x, g, b, EPS, y=y)
            want, bound = ref.norm(x, g, b, EPS, dtype)
            for t, w, e, name in zip(got, want, bound, ("y", "mean", "rstd")):
                ref.assert_within(t, w, e, name)
            assert (held[:, cols:] == 7.0).all()


@pytest.mark.parametrize("dtype,p_dtype", PAIRS, ids=str)
@pytest.mark.parametrize("rows,cols", NORM_SIZES)
def test_norm_int8(xb, dtype, p_dtype, rows, cols):
    x, gamma, beta = norm_inputs(rows, cols, dtype, p_dtype)
    q, s = xb.xnor_layer_norm_fwd_int8(x, gamma, beta, EPS)
    (y, _, _), (e, _, _) = ref.norm(x, gamma, beta, EPS, None)
    top, e_top = y.abs().amax(1), e.amax(1)
    ref.assert_within(s, top / 127, e_top / 127 + 2 * ref.U * top / 127, "scale")
    # half a level, the value's own error, and two roundings of up to 127 levels
    level = s.cpu().double()[:, None]
    ref.assert_within(q.cpu().double() * level, y, 0.5 * level + e + 127 * 4 * ref.U * level, "levels")


def test_norm_constant_rows(xb):
    """No variance: the output is beta, whatever the value."""
    x = torch.tensor([[3.0], [-1e4], [0.0]], device="cuda").expand(3, 640).contiguous()
    gamma, beta = rand(1, 640), rand(2, 640)
    y, mean, rstd = xb.xnor_layer_norm_fwd(x, gamma, beta, EPS)
    assert torch.equal(y, beta.expand(3, 640)) and mean.tolist() == [3.0, -1e4, 0.0]
    y, _, rstd = xb.xnor_layer_norm_fwd(x[:, :1], None, None, EPS)
    assert (y == 0).all()


@pytest.mark.parametrize("dtype,p_dtype", PAIRS, ids=str)
@pytest.mark.parametrize("rows,cols", NORM_SIZES + [(0, 33), (40, 70), (515, 130), (700, 1030), (300, 2500), (1030, 20)])
def test_norm_backward(xb, dtype, p_dtype, rows, cols):
    if rows * cols > 400000:
        rows = 2
    x, gamma, _ = norm_inputs(rows, cols, dtype, p_dtype, 1)
    dy = rand(rows + 77, rows, cols, dtype=dtype)
    (_, mean, rstd), _ = ref.norm(x, gamma, None, EPS, None)
    mean, rstd = mean.float().cuda(), rstd.float().cuda()
    for g in (gamma, None):
        p = p_dtype if g is not None else F32
        held, dx = spaced(rows, cols, dtype, 3, 7.0)
        got = xb.xnor_layer_norm_bwd(dy, x, g, mean, rstd, dx=dx)
        want, bound = ref.norm_back(dy, x, g, mean, rstd, dtype, p)
        for t, w, e, name in zip(got, want, bound, ("dx", "dgamma", "dbeta")):
            ref.assert_within(t, w, e, name)
        assert (held[:, cols:] == 7.0).all()
        again = xb.xnor_layer_norm_bwd(dy, x, g, mean, rstd)
        assert all(torch.equal(a, b) for a, b in zip(got, again))
        alone = xb.xnor_layer_norm_bwd(dy, x, g, mean, rstd, want_params=False)
        assert alone[1] is None and torch.equal(alone[0], got[0])


@pytest.mark.parametrize("dtype,p_dtype", PAIRS, ids=str)
@pytest.mark.parametrize("rows,cols", [(1, 8), (2, 64), (9, 520), (4100, 1024), (5, 2056), (2600, 4096), (3, 8192), (2, 16384)])
def test_norm_whole_chunks(xb, dtype, p_dtype, rows, cols):
    """Rows of whole 16-byte chunks at multiples of 16 bytes, with others behind them, up to more than a workgroup takes two of."""
    x, gamma, beta = norm_inputs(rows, cols, dtype, p_dtype, 16)
    dy = rand(rows + 78, rows, cols + 8, dtype=dtype)[:, :cols]
    got = xb.xnor_layer_norm_fwd(x, gamma, beta, EPS)
    want, bound = ref.norm(x, gamma, beta, EPS, dtype)
    for t, w, e, name in zip(got, want, bound, ("y", "mean", "rstd")):
        ref.assert_within(t, w, e, name)
    _, mean, rstd = got
    got = xb.xnor_layer_norm_bwd(dy, x, gamma, mean, rstd)
    want, bound = ref.norm_back(dy, x, gamma, mean, rstd, dtype, p_dtype)
    for t, w, e, name in zip(got, want, bound, ("dx", "dgamma", "dbeta")):
        ref.assert_within(t, w, e, name)
    q, s = xb.xnor_int8_quantize(x)
    want_q, want_s = xb.xnor_int8_quantize(x[-1:])
    assert torch.equal(q[-1:], want_q) and torch.equal(s[-1:], want_s)
    q, s = xb.xnor_layer_norm_fwd_int8(x, gamma, beta, EPS)
    want_q, want_s = xb.xnor_layer_norm_fwd_int8(x[rows // 2:], gamma, beta, EPS)
    assert torch.equal(q[rows // 2:], want_q) and torch.equal(s[rows // 2:], want_s)


def test_norm_gradient_against_differences(xb):
    rows, cols, h = 4, 37, 1e-4
    x, gamma, beta = norm_inputs(rows, cols, F32, F32)
    dy, v = rand(8, rows, cols), rand(9, rows, cols).double().cpu()
    y, mean, rstd = xb.xnor_layer_norm_fwd(x, gamma, beta, EPS)
    dx, dgamma, dbeta = xb.xnor_layer_norm_bwd(dy, x, gamma, mean, rstd)

    def loss(x, g, b):
        return float((ref.norm(x, g, b, EPS, None)[0][0] * dy.cpu().double()).sum())
    X, G, B = (t.cpu().double() for t in (x, gamma, beta))
    vg = rand(10, cols).double().cpu()
    # the differences are off by h^2 times third derivatives (about 1e-7 here); the kernel by a few 1e-6 of sums of order 10
    for slope, got in (((loss(X + h * v, G, B) - loss(X - h * v, G, B)) / (2 * h), dx.cpu().double().mul(v).sum()),
                       ((loss(X, G + h * vg, B) - loss(X, G - h * vg, B)) / (2 * h), dgamma.cpu().double().mul(vg).sum()),
                       ((loss(X, G, B + h * vg) - loss(X, G, B - h * vg)) / (2 * h), dbeta.cpu().double().mul(vg).sum())):
        assert abs(slope - float(got)) <= 1e-4 * max(1.0, abs(slope))


# ---- the gated block ---------------------------------------------------------------------------------------------------

GATED_SIZES = [(1, 1, 1), (1, 100, 64), (2, 17, 33), (5, 64, 8), (16, 65, 200), (33, 48, 1001), (64, 128, 64), (65, 130, 96), (130, 257, 72), (257, 129, 130),
               (300, 192, 320)]


@pytest.mark.parametrize("kind", [ref.SILU, ref.GELU, ref.RELU])
@pytest.mark.parametrize("dtype", [F16, BF16], ids=str)
@pytest.mark.parametrize("M,F,K", GATED_SIZES)
def test_gated_forward(xb, dtype, M, F, K, kind):
    for spare in (0, 1, (-K) % 8 + 8):
        x = rand(M, M, K + spare, dtype=dtype)[:, :K]
        wg, wu = (rand(F + i, F, K + spare, dtype=dtype, std=2.0 / K ** 0.5)[:, :K] for i in (0, 1))
        held, h = spaced(M, F, dtype, 1, 5.0)
        got = xb.xnor_gated_fwd(x, wg, wu, kind, h=h, want_pre=True)
        want, bound = ref.gated(x, wg, wu, kind, dtype)
        for t, w, e, name in zip(got, want, bound, "hgu"):
            ref.assert_within(t, w, e, f"{name}, spare {spare}")
        assert (held[:, F:] == 5.0).all()
        assert torch.equal(xb.xnor_gated_fwd(x, wg, wu, kind), got[0])


@pytest.mark.parametrize("kind", [ref.SILU, ref.GELU, ref.RELU])
@pytest.mark.parametrize("dtype", [F16, BF16], ids=str)
@pytest.mark.parametrize("M,F,K", [(0, 20, 30)] + GATED_SIZES)
def test_gated_backward(xb, dtype, M, F, K, kind):
    for spare in (0, 3, (-K) % 8 + 8):
        x = rand(M, M, K + spare, dtype=dtype)[:, :K]
        wg, wu = (rand(F + i, F, K + spare, dtype=dtype, std=K ** -0.5)[:, :K] for i in (0, 1))
        dh, g, u = (rand(M * 5 + i, M, F + spare, dtype=dtype)[:, :F] for i in range(3))
        held, dx = spaced(M, K, dtype, 2, 5.0)
        kept = [spaced(F, K, dtype, 2, 5.0) for _ in range(2)]
        got = xb.xnor_gated_bwd(dh, x, wg, wu, g, u, kind, dx=dx, dwg=kept[0][1], dwu=kept[1][1])
        want, bound = ref.gated_back(dh, x, wg, wu, g, u, kind, dtype)
        for t, w, e, name in zip(got, want, bound, ("dx", "dwg", "dwu")):
            ref.assert_within(t, w, e, f"{name}, spare {spare}")
        for t in (held, kept[0][0], kept[1][0]):
            assert (t[:, K:] == 5.0).all()


@pytest.mark.parametrize("kind", [ref.SILU, ref.GELU, ref.RELU])
def test_gated_gradient_against_differences(xb, kind):
    """With values that are exact in f16, along one direction of each operand, for a block of f16."""
    M, F, K, h = 6, 10, 24, 1e-4
    x, wg, wu, dh = rand(1, M, K, dtype=F16), rand(2, F, K, dtype=F16, std=0.3), rand(3, F, K, dtype=F16, std=0.3), rand(4, M, F, dtype=F16)
    _, g, u = xb.xnor_gated_fwd(x, wg, wu, kind, want_pre=True)
    got = xb.xnor_gated_bwd(dh, x, wg, wu, g, u, kind)
    at = [t.cpu().double() for t in (x, wg, wu)]

    def loss(x, wg, wu):
        return float((ref.act(x @ wg.t(), kind) * (x @ wu.t()) * dh.cpu().double()).sum())
    for i in range(3):
        v = rand(20 + i, *at[i].shape).cpu().double()
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + h * v, at[i] - h * v
        want = (loss(*up) - loss(*down)) / (2 * h)
        # g, u, dg, du and the outputs are rounded to 11 bits: five roundings of each of the gradient's terms
        terms = (got[i].cpu().double() * v).abs().sum()
        assert abs(want - float((got[i].cpu().double() * v).sum())) <= 5 * 2.0 ** -11 * 4 * float(terms)


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("kind", [ref.SILU, ref.GELU, ref.RELU])
@pytest.mark.parametrize("M,F,K", [(1, 1, 1), (1, 300, 1037), (2, 64, 256), (9, 33, 100), (16, 130, 512), (17, 66, 129), (64, 128, 256), (129, 257, 384), (300, 70, 2000)])
def test_int8_gated(xb, dtype, kind, M, F, K):
    for spare in (0, (-K) % 16):
        a, wg, wu = ints(M, M, K, spare), ints(F + 1, F, K, spare), ints(F + 2, F, K, spare)
        sa, sg, su = scales(1, M), scales(2, F) * 0.1, scales(3, F) * 0.1
        held, h = spaced(M, F, dtype, 3, 5.0)
        xb.xnor_int8_gated(a, sa, wg, sg, wu, su, kind, h=h)
        want, bound = ref.int8_gated(a, sa, wg, sg, wu, su, kind, dtype)
        fits = want.abs() < torch.finfo(dtype).max          # (beyond f16's range: an infinity)
        ref.assert_within(torch.where(fits.cuda(), h, 0), torch.where(fits, want, 0), bound, f"spare {spare}")
        assert (held[:, F:] == 5.0).all()


# ---- sizes that fill the chip: some rows and columns of the results ---------------------------------------------------------

LARGE = [(4100, 4200, 128), (4096, 4096, 64), (2100, 8200, 700), (9000, 1100, 1337), (4500, 2049, 2304), (2000, 8100, 1000)]


def some(n, block=256):
    """The first, the last and those around the edges of blocks."""
    at = {0, 1, 15, 16, n // 2, n - 2, n - 1}
    for e in range(block // 2, n, max(block // 2, n // 12 // (block // 2) * (block // 2))):
        at |= {e - 1, e}
    return torch.tensor(sorted(i for i in at if 0 <= i < n))


@pytest.mark.parametrize("M,N,K", LARGE)
def test_large_int8_matmul(xb, M, N, K):
    for spare in (0, (-K) % 16):
        a, b, sa, sb, bias = ints(1, M, K, spare), ints(2, N, K, spare), scales(3, M), scales(4, N), rand(5, N)
        rows, cols = some(M), some(N)
        for dtype in (F32, BF16):
            held, out = spaced(M, N, dtype, 3, -7.0)
            xb.xnor_int8_matmul(a, sa, b, sb, bias, out=out)
            for r, c in ((rows, torch.arange(N)), (torch.arange(M), cols)):
                want, bound = ref.int8_matmul(a[r], sa[r], b[c], sb[c], bias[c], dtype)
                ref.assert_within(out[r.cuda()][:, c.cuda()], want, bound, f"spare {spare} {dtype}")
            assert (held[:, N:] == -7.0).all()


@pytest.mark.parametrize("M,F,K", LARGE)
def test_large_gated(xb, M, F, K):
    x, wg, wu = rand(1, M, K, dtype=BF16), rand(2, F, K, dtype=BF16, std=K ** -0.5), rand(3, F, K, dtype=BF16, std=K ** -0.5)
    for spare in (0, 8):
        held, h = spaced(M, F, BF16, spare, 5.0)
        got = xb.xnor_gated_fwd(x, wg, wu, ref.GELU, h=h, want_pre=True)
        for r, c in ((some(M), torch.arange(F)), (torch.arange(M), some(F))):
            want, bound = ref.gated(x[r], wg[c], wu[c], ref.GELU, BF16)
            for t, w, e, name in zip(got, want, bound, "hgu"):
                ref.assert_within(t[r.cuda()][:, c.cuda()], w, e, name)
        assert (held[:, F:] == 5.0).all()
    a, sa, w8, u8, sg, su = ints(1, M, K), scales(2, M), ints(3, F, K), ints(4, F, K), scales(5, F) * 0.1, scales(6, F) * 0.1
    h8 = xb.xnor_int8_gated(a, sa, w8, sg, u8, su, ref.SILU)
    for r, c in ((some(M), torch.arange(F)), (torch.arange(M), some(F))):
        want, bound = ref.int8_gated(a[r], sa[r], w8[c], sg[c], u8[c], su[c], ref.SILU, F32)
        ref.assert_within(h8[r.cuda()][:, c.cuda()], want, bound, "8 bits")


@pytest.mark.parametrize("dtype", [F16, BF16], ids=str)
@pytest.mark.parametrize("M,F,K", [(4104, 2100, 2104), (2100, 4104, 4100), (9001, 1001, 1000), (1500, 300, 2048), (5, 3000, 1200)])
def test_large_gated_backward(xb, dtype, M, F, K):
    x = rand(1, M, K, dtype=dtype)
    wg, wu = rand(2, F, K, dtype=dtype, std=K ** -0.5), rand(3, F, K, dtype=dtype, std=K ** -0.5)
    dh, g, u = (rand(4 + i, M, F, dtype=dtype) for i in range(3))
    dx, dwg, dwu = xb.xnor_gated_bwd(dh, x, wg, wu, g, u, ref.SILU)
    r, c = some(M), some(F)
    want, bound = ref.gated_back(dh[r], x[r], wg, wu, g[r], u[r], ref.SILU, dtype)
    ref.assert_within(dx[r.cuda()], want[0], bound[0], "dx")
    want, bound = ref.gated_back(dh[:, c], x, wg[c], wu[c], g[:, c], u[:, c], ref.SILU, dtype)
    ref.assert_within(dwg[c.cuda()], want[1], bound[1], "dwg")
    ref.assert_within(dwu[c.cuda()], want[2], bound[2], "dwu")
    again = xb.xnor_gated_bwd(dh, x, wg, wu, g, u, ref.SILU)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dwg) and torch.equal(again[2], dwu)


def test_gated_backward_keeps_to_its_rows(xb):
    """What lies behind the operands' rows and columns, here infinities, reaches no result: contraction ends inside a step of 64."""
    M, F, K = 70, 100, 72
    def inside(rows, cols, seed, **kw):
        t = torch.full((rows + 3, cols + 8), float("inf"), dtype=BF16, device="cuda")
        t[:rows, :cols] = rand(seed, rows, cols, dtype=BF16, **kw)
        return t[:rows, :cols]
    x, wg, wu, dh, g, u = (inside(r, c, i) for i, (r, c) in enumerate(((M, K), (F, K), (F, K), (M, F), (M, F), (M, F))))
    got = xb.xnor_gated_bwd(dh, x, wg, wu, g, u)
    want, bound = ref.gated_back(dh, x, wg, wu, g, u, ref.SILU, BF16)
    for t, w, e, name in zip(got, want, bound, ("dx", "dwg", "dwu")):
        ref.assert_within(t, w, e, name)
    h = xb.xnor_gated_fwd(x, wg, wu)
    want, bound = ref.gated(x, wg, wu, ref.SILU, BF16)
    ref.assert_within(h, want[0], bound[0], "h")


def test_gated_forward_workspace(xb):
    """Rows of odd stride, with the copies that a workspace allows and without: the same values."""
    M, F, K = 300, 400, 3001
    x, wg, wu = rand(1, M, K, dtype=F16), rand(2, F, K, dtype=F16, std=0.02), rand(3, F, K, dtype=F16, std=0.02)
    need = xb.xnor_gated_fwd_workspace_bytes(M, F, K, K, K)
    assert need > 0 and xb.xnor_gated_fwd_workspace_bytes(M, F, K, 3008, 3008) == 0 and xb.xnor_gated_fwd_workspace_bytes(8, F, K, K, K) == 0
    want, bound = ref.gated(x, wg, wu, ref.GELU, F16)
    for workspace in (None, torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty(16, dtype=torch.uint8, device="cuda")):
        got = xb.xnor_gated_fwd(x, wg, wu, ref.GELU, want_pre=True, workspace=workspace)
        for t, w, e, name in zip(got, want, bound, "hgu"):
            ref.assert_within(t, w, e, name)
    # rows of one value apart and all of one row: strides that no fetch of whole chunks takes
    one = rand(4, 1, K, dtype=F16).expand(M, K)
    want, bound = ref.gated(one, wg, wu, ref.SILU, F16)
    ref.assert_within(xb.xnor_gated_fwd(one, wg, wu), want[0], bound[0], "stride 0")


# ---- no tokens, long offsets, streams, graphs --------------------------------------------------------------------------


def test_no_tokens(xb):
    x = torch.empty(0, 64, dtype=BF16, device="cuda")
    w, sw = xb.xnor_int8_quantize(rand(1, 32, 64))
    assert xb.xnor_int8_quantize(x)[0].shape == (0, 64)
    assert xb.xnor_int8_linear(x, w, sw).shape == (0, 32)
    q, s = xb.xnor_layer_norm_fwd_int8(x, None, None)
    assert xb.xnor_int8_matmul(q, s, w, sw).shape == (0, 32) and xb.xnor_int8_gated(q, s, w, sw, w, sw).shape == (0, 32)
    assert xb.xnor_layer_norm_fwd(x, None, None)[0].shape == (0, 64)
    wg = rand(2, 32, 64, dtype=BF16)
    assert xb.xnor_gated_fwd(x, wg, wg, want_pre=True)[1].shape == (0, 32)


def test_offsets_past_32_bits(xb):
    """Rows more than 2^31 values apart, and an operand whose last row starts behind 4 GiB."""
    stride = (1 << 31) + 24
    big = torch.empty(2 * stride + 1024, dtype=torch.int8, device="cuda")
    a = big.as_strided((3, 300), (stride, 1))
    a.copy_(ints(1, 3, 300))
    b, sa, sb = ints(2, 70, 300), scales(3, 3), scales(4, 70)
    want, bound = ref.int8_matmul(a, sa, b, sb, None, F32)
    ref.assert_within(xb.xnor_int8_matmul(a, sa, b, sb), want, bound, "tokens")
    b3, s3 = a, sa
    a3, sa3 = ints(5, 40, 300), scales(6, 40)
    want, bound = ref.int8_matmul(a3, sa3, b3, s3, None, F32)
    ref.assert_within(xb.xnor_int8_matmul(a3, sa3, b3, s3), want, bound, "weights")
    x = big.view(torch.bfloat16).as_strided((3, 300), (stride // 2, 1))
    x.copy_(rand(7, 3, 300, dtype=BF16))
    want, bound = ref.norm(x, None, None, EPS, BF16)
    ref.assert_within(xb.xnor_layer_norm_fwd(x, None, None, EPS)[0], want[0], bound[0], "norm")
    wg, wu = rand(8, 40, 300, dtype=BF16, std=0.05), rand(9, 40, 300, dtype=BF16, std=0.05)
    want, bound = ref.gated(x, wg, wu, ref.SILU, BF16)
    ref.assert_within(xb.xnor_gated_fwd(x, wg, wu), want[0], bound[0], "gated")


def test_many_rows(xb):
    """More rows than a launch has workgroups."""
    rows = (1 << 24) + 77
    x = torch.arange(rows, device="cuda", dtype=torch.int32).remainder(251).float()[:, None].expand(rows, 2) * torch.tensor([1.0, -2.0], device="cuda")
    x = x.contiguous()
    q, s = xb.xnor_int8_quantize(x)
    some = torch.tensor([0, 1, 1 << 22, (1 << 24) - 1, 1 << 24, rows - 2, rows - 1], device="cuda")
    q0, s0 = ref.quantize(x[some])
    assert torch.equal(q[some].cpu(), q0) and torch.equal(s[some].cpu(), s0)
    top = x.abs().amax(1)
    assert torch.equal(s, torch.where(top > 0, top / torch.full_like(top, 127.0), torch.zeros_like(top)))


def everything(xb, x, w8, w16, gamma, beta, dh):
    q, s = xb.xnor_layer_norm_fwd_int8(x, gamma, beta)
    h8 = xb.xnor_int8_gated(q, s, *w8, *w8, out_dtype=BF16)
    y, mean, rstd = xb.xnor_layer_norm_fwd(x, gamma, beta)
    h, g, u = xb.xnor_gated_fwd(y, *w16, want_pre=True)
    dy, dwg, dwu = xb.xnor_gated_bwd(dh, y, *w16, g, u)
    return [h8, xb.xnor_int8_linear(x, *w8), h, dwg, dwu, *xb.xnor_layer_norm_bwd(dy, x, gamma, mean, rstd)]


@pytest.mark.parametrize("M", [1, 200])
def test_other_stream_and_graph(xb, M):
    K, F = 192, 320
    x, gamma, beta = norm_inputs(M, K, BF16, F32)
    w8 = xb.xnor_int8_quantize(rand(1, F, K))
    w16 = (rand(2, F, K, dtype=BF16, std=0.1), rand(3, F, K, dtype=BF16, std=0.1))
    dh = rand(4, M, F, dtype=BF16)
    eager = everything(xb, x, w8, w16, gamma, beta, dh)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = everything(xb, x, w8, w16, gamma, beta, dh)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, there))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        held = everything(xb, x, w8, w16, gamma, beta, dh)
    for turn in range(3):
        x.copy_(norm_inputs(M, K + turn, BF16, F32)[0][:, :K])
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(everything(xb, x, w8, w16, gamma, beta, dh), held):
            assert torch.equal(a, b), f"replay {turn}"
