"""Products with 4-bit weights against their definition in 64 bits: sizes at which kernels and tiles end, groups, zero points, types, strides, values that
are not finite.  Tolerances are the bounds that experts_reference derives."""
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


def rand(seed, *shape, dtype=F32, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(dtype).cuda()


def weights(xb, seed, rows, cols, group, zeros, scale_dtype, count=None):
    """A matrix or stack of all levels, whose words hold levels behind the last column too."""
    g = torch.Generator().manual_seed(seed)
    many = () if count is None else (count,)
    words = (cols + 7) // 8
    held = torch.randint(0, 256, (*many, rows, (words + 3) // 4 * 16), generator=g, dtype=torch.uint8)
    groups = (cols + group - 1) // group
    scale = (torch.rand(*many, groups, rows, generator=g) + 0.5) * 0.2 / cols ** 0.5
    zero = torch.randint(0, 16, (*many, groups, rows), generator=g, dtype=torch.uint8).cuda() if zeros else None
    return xb.Int4(held.cuda()[..., :words * 4], scale.to(scale_dtype).cuda(), zero, cols, group)


@pytest.mark.parametrize("dtype,scale_dtype,group,zeros,rows,cols", [
    (F32, F32, 32, False, 1, 1), (BF16, BF16, 128, False, 7, 300), (F16, F16, 64, True, 16, 129), (F32, BF16, 32, True, 5, 31), (F32, F16, 128, True, 33, 2050),
    (BF16, F32, 64, False, 3, 4096), (F16, BF16, 32, False, 2, 8193)], ids=str)
def test_quantize_pack_dequantize(xb, dtype, scale_dtype, group, zeros, rows, cols):
    w = rand(1, rows, cols, dtype=dtype)
    if rows > 2:
        w[1] = 0.0
        w[2, :1] = float("inf")
    got = xb.xnor_int4_quantize(w, group, zeros, scale_dtype)
    levels, scale, zero = xref.quantize(w, group, zeros, scale_dtype)
    assert torch.equal(xref.levels_of(got.q, cols), levels)
    assert torch.equal(got.scale.cpu().nan_to_num(-1.0), scale.nan_to_num(-1.0))
    assert (got.zero is None) == (zero is None) and (zero is None or torch.equal(got.zero.cpu(), zero))
    assert torch.equal(xb.xnor_int4_pack(levels.cuda()), got.q)
    for out in (F32, F16, BF16):
        v = xb.xnor_int4_dequantize(got, out_dtype=out).cpu().double()
        want = xref.values(got)[0]
        assert torch.equal(v.isnan(), want.isnan())
        want, v = want.nan_to_num(0.0), v.nan_to_num(0.0)
        assert ((v - want).abs() <= ref.U * want.abs() + ref.rounding(want, out)).all()
    # a level is half a step at most from its value (a step more where the scale's rounding, of the zero point's, made the range shorter)
    ok = torch.isfinite(w).all(1).cpu()
    w, s = w.cpu().double()[ok], xref.values(got)[1][ok]
    assert ((xref.values(got)[0][ok] - w).abs() <= (0.5 + 15 * ref.UT[scale_dtype] + (0.51 if zeros else 0.0)) * s + 1e-30).all()


SIZES = [(1, 1, 1), (1, 16, 128), (1, 17, 7), (1, 2050, 4100), (3, 33, 129), (5, 1, 1000), (15, 64, 1023), (16, 100, 2048), (17, 40, 1037), (33, 50, 300),
         (64, 130, 520), (65, 70, 513), (128, 128, 128), (129, 300, 1000), (257, 129, 2049), (1000, 255, 96)]


@pytest.mark.parametrize("M,N,K", SIZES, ids=str)
@pytest.mark.parametrize("dtype,scale_dtype,group,zeros,out_dtype", [
    (BF16, BF16, 128, False, BF16), (F16, F16, 32, True, F16), (BF16, F32, 64, True, F32), (F16, BF16, 64, False, BF16), (BF16, F16, 32, False, F16)], ids=str)
def test_linear(xb, M, N, K, dtype, scale_dtype, group, zeros, out_dtype):
    x, w = rand(M + N, M, K, dtype=dtype), weights(xb, K, N, K, group, zeros, scale_dtype)
    bias = rand(5, N) if zeros else None
    want, bound = xref.linear(x, w, bias, out_dtype)
    got = xb.xnor_int4_linear(x, w, bias, out_dtype=out_dtype)
    assert got.dtype is out_dtype
    ref.assert_within(got, want, bound, "y")
    assert torch.equal(got, xb.xnor_int4_linear(x, w, bias, out_dtype=out_dtype))


@pytest.mark.parametrize("M,F,K", SIZES, ids=str)
@pytest.mark.parametrize("dtype,scale_dtype,group,zeros,act,out_dtype", [
    (BF16, BF16, 64, True, ref.SILU, BF16), (F16, F16, 128, False, ref.GELU, F16), (F16, F32, 32, True, ref.RELU, F32),
    (BF16, BF16, 32, False, ref.GELU, F32)], ids=str)
def test_gated(xb, M, F, K, dtype, scale_dtype, group, zeros, act, out_dtype):
    x = rand(M + F, M, K, dtype=dtype)
    wg, wu = weights(xb, K, F, K, group, zeros, scale_dtype), weights(xb, K + 1, F, K, group, zeros, scale_dtype)
    want, bound = xref.gated(x, wg, wu, act, out_dtype)
    ref.assert_within(xb.xnor_int4_gated(x, wg, wu, act, out_dtype=out_dtype), want, bound, "h")


@pytest.mark.parametrize("M", [0, 1, 20, 200])
def test_strides_and_edges(xb, M):
    """Tokens one row for all or at odd strides, weights' rows 4 bytes on from one another's end, outputs in a wider buffer that keeps what it holds."""
    N, K = 37, 205
    w = weights(xb, 3, N, K, 32, True, F16)
    apart = torch.zeros(N * 108 + 4, dtype=torch.uint8, device="cuda")
    held = torch.as_strided(apart, (N, 104), (108, 1), 4)
    held.copy_(w.q)
    odd = w._replace(q=held)
    buffer = torch.full((M + 2, N + 5), 7.0, dtype=BF16, device="cuda")
    for x in (rand(1, M, K + 3, dtype=BF16)[:, 3:], rand(2, 1, K, dtype=BF16).expand(M, K)):
        want, bound = xref.linear(x, w, None, BF16)
        got = xb.xnor_int4_linear(x, odd, out=buffer[1:M + 1, 2:N + 2])
        ref.assert_within(got, want, bound, "y")
        assert torch.equal(got, xb.xnor_int4_linear(x.contiguous(), w))
        edge = buffer.clone()
        edge[1:M + 1, 2:N + 2] = 7.0
        assert (edge == 7.0).all()
        want, bound = xref.gated(x, w, w, ref.SILU, F32)
        ref.assert_within(xb.xnor_int4_gated(x, odd, odd, out_dtype=F32), want, bound, "h")


@pytest.mark.parametrize("M", [5, 40, 150])
@pytest.mark.parametrize("dtype", [F16, BF16], ids=str)
def test_values_that_are_not_finite(xb, M, dtype):
    """A token's infinity or NaN and a group's scale NaN reach the outputs that they belong to, as they would in products of the values, and no others."""
    N, K = 50, 300
    x, w = rand(1, M, K, dtype=dtype), weights(xb, 2, N, K, 64, False, BF16)
    w.scale[2, 7] = float("nan")
    x[1, 5], x[2, 6], x[3, 299] = float("inf"), float("nan"), float("-inf")
    got = xb.xnor_int4_linear(x, w, out_dtype=F32).cpu().double()
    clean = x.clone()
    clean[1, 5], clean[2, 6], clean[3, 299] = 0.0, 0.0, 0.0
    well = w._replace(scale=w.scale.nan_to_num(1.0))
    want, bound = xref.linear(clean, well, None, F32)
    v = xref.values(well)[0]
    want[1] += v[:, 5] * float("inf")
    want[3] += v[:, 299] * float("-inf")
    want[2], want[:, 7] = float("nan"), float("nan")
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.isinf(), want.isinf()) and torch.equal(got[got.isinf()] > 0, want[want.isinf()] > 0)
    fine = torch.isfinite(want)
    assert ((got - want).abs()[fine] <= bound[fine]).all()


@pytest.mark.parametrize("M", [2, 100])
def test_large_values(xb, M):
    """bf16 tokens near the type's largest value, whose products with levels are not finite though their sums with zero points taken off are."""
    N, K = 40, 128
    x, w = torch.full((M, K), 2.0 ** 124, dtype=BF16, device="cuda"), weights(xb, 2, N, K, 128, False, BF16)
    x[:, 64:] *= -1.0
    w.scale.fill_(2.0 ** -20)
    want, bound = xref.linear(x, w, None, F32)
    got = xb.xnor_int4_linear(x, w, out_dtype=F32)
    assert torch.isfinite(got).all()
    assert ((got.cpu().double() - want).abs() <= bound * 1.01).all()


@pytest.mark.parametrize("M", [1, 300])
def test_replayed_and_on_another_stream(xb, M):
    N, K = 256, 1024
    x, w, wu = rand(1, M, K, dtype=BF16), weights(xb, 2, N, K, 128, False, BF16), weights(xb, 3, N, K, 128, False, BF16)
    eager = [xb.xnor_int4_linear(x, w), xb.xnor_int4_gated(x, w, wu)]
    out = [torch.empty_like(t) for t in eager]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        xb.xnor_int4_linear(x, w, out=out[0])
        xb.xnor_int4_gated(x, w, wu, h=out[1])
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(eager, out))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        xb.xnor_int4_linear(x, w, out=out[0])
        xb.xnor_int4_gated(x, w, wu, h=out[1])
    for seed in (4, 5, 6):
        x.copy_(rand(seed, M, K, dtype=BF16))
        eager = [xb.xnor_int4_linear(x, w), xb.xnor_int4_gated(x, w, wu)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, out))


def stacks(xb, E, K, F, N, group, zeros, scale_dtype):
    return (weights(xb, 1, F, K, group, zeros, scale_dtype, E), weights(xb, 2, F, K, group, zeros, scale_dtype, E),
            weights(xb, 3, N, F, group, zeros, scale_dtype, E))


@pytest.mark.parametrize("T,k,E,K,F,N", [(1, 1, 1, 1, 1, 1), (1, 8, 64, 256, 128, 256), (1, 3, 5, 77, 33, 50), (7, 2, 4, 130, 70, 130), (24, 3, 30, 110, 77, 110),
                                         (40, 4, 6, 300, 130, 300), (65, 1, 2, 64, 100, 40), (300, 2, 3, 140, 129, 140), (200, 32, 40, 40, 40, 40),
                                         (1000, 2, 2, 70, 64, 33), (3, 2, 1000, 40, 24, 40)], ids=str)
@pytest.mark.parametrize("dtype,scale_dtype,group,zeros,act,out_dtype", [
    (BF16, BF16, 128, False, ref.SILU, BF16), (F16, F16, 32, True, ref.GELU, F16), (BF16, F32, 64, True, ref.RELU, F32)], ids=str)
def test_experts(xb, T, k, E, K, F, N, dtype, scale_dtype, group, zeros, act, out_dtype):
    """Experts that few or none chose, one that most did, slots without one, one expert in two slots of a token."""
    g = torch.Generator().manual_seed(T + E)
    chosen = torch.rand(T, E, generator=g).mul(torch.linspace(3, 1, E)).argsort(1, descending=True)[:, :min(k, E)]
    chosen = torch.nn.functional.pad(chosen, (0, k - chosen.shape[1])).int()
    if T > 4 and k > 1:
        chosen[1, 0], chosen[2], chosen[3, 1], chosen[4, 1] = -1, -1, E, chosen[4, 0]
    share = torch.rand(T, k, generator=g)
    wg, wu, wd = stacks(xb, E, K, F, N, group, zeros, scale_dtype)
    x = rand(9, T, K, dtype=dtype)
    want, bound = xref.experts(x, chosen, share, wg, wu, wd, act, out_dtype)
    got = xb.xnor_int4_experts(x, chosen.cuda(), share.cuda(), wg, wu, wd, act, out_dtype=out_dtype)
    assert got.dtype is out_dtype
    ref.assert_within(got, want, bound, "y")
    assert torch.equal(got, xb.xnor_int4_experts(x, chosen.cuda(), share.cuda(), wg, wu, wd, act, out_dtype=out_dtype))


@pytest.mark.parametrize("T", [6, 100])
def test_experts_of_tokens_that_were_not_routed(xb, T):
    """Weights NaN show, slots without an expert add nothing, and what lies behind the outputs stays."""
    E, K, F, N = 4, 64, 48, 52
    wg, wu, wd = stacks(xb, E, K, F, N, 32, False, BF16)
    x = rand(1, T, K, dtype=BF16)
    chosen = torch.zeros(T, 2, dtype=torch.int32, device="cuda")
    share = torch.full((T, 2), 0.5, device="cuda")
    chosen[0], share[0] = -1, float("nan")
    chosen[1], share[1] = -1, 0.0
    held = torch.full((T + 1, N + 4), 3.0, dtype=BF16, device="cuda")
    got = xb.xnor_int4_experts(x, chosen, share, wg, wu, wd, out=held[:T, :N])
    assert got[0].isnan().all() and (got[1] == 0).all() and torch.isfinite(got[1:]).all()
    assert (held[T] == 3.0).all() and (held[:, N:] == 3.0).all()
    none = xb.xnor_int4_experts(x, torch.full_like(chosen, -1), torch.zeros_like(share), wg, wu, wd)
    assert (none == 0).all()
    assert xb.xnor_int4_experts(x[:0], chosen[:0], share[:0], wg, wu, wd).shape == (0, N)


@pytest.mark.parametrize("T", [1, 30, 600])
def test_routed_experts_replayed(xb, T):
    """The served layer's calls as one graph, replayed with other tokens: logits, choice, experts' products; two graphs and eager calls in turn, each with
    workspaces of its own or one for both."""
    E, K, F, k = 16, 256, 128, 4
    wg, wu, wd = stacks(xb, E, K, F, K, 128, False, BF16)
    gate = rand(7, K, E, dtype=BF16, std=K ** -0.5)
    x = rand(1, T, K, dtype=BF16)
    space = torch.empty(xb.xnor_int4_experts_workspace_bytes(T, k, E, K, F, K), dtype=torch.uint8, device="cuda")

    def layer(workspace):
        experts, share = xb.xnor_route_fwd(x @ gate, k, score=xb.SCORE_SIGMOID)
        offsets, order = xb.xnor_route_lists(experts, E)
        return xb.xnor_int4_experts(x, experts, share, wg, wu, wd, workspace=workspace), experts, share, offsets, order
    layer(None)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    outs = []
    for graph in graphs:
        with torch.cuda.graph(graph):
            outs.append(layer(space))
    for seed in range(4):
        x.copy_(rand(20 + seed, T, K, dtype=BF16))
        eager = layer(None)
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for out in outs:
            assert all(torch.equal(a, b) for a, b in zip(eager, out))


MANY = [(65, 300, 30000), (129, 1100, 2600), (1000, 520, 1100), (8200, 1030, 70), (20000, 260, 130), (40000, 300, 60), (300, 1024, 4096), (90, 1, 5000000), (40, 1030, 8200),
        (33, 2050, 8195)]


@pytest.mark.parametrize("M,N,K", MANY, ids=str)
@pytest.mark.parametrize("dtype,scale_dtype,group,zeros,out_dtype", [(BF16, BF16, 128, False, BF16), (F16, F32, 32, True, F32)], ids=str)
def test_many_tokens(xb, M, N, K, dtype, scale_dtype, group, zeros, out_dtype):
    """Products that go to the tiles: whole and in shares of the contraction, of 128 and 256 tokens, of a contraction that ends inside the only step; with
    the workspace and without one."""
    x, w = rand(M + N, M, K, dtype=dtype), weights(xb, K, N, K, group, zeros, scale_dtype)
    bias = rand(5, N) if zeros else None
    want, bound = xref.linear(x, w, bias, out_dtype)
    got = xb.xnor_int4_linear(x, w, bias, out_dtype=out_dtype)
    ref.assert_within(got, want, bound, "y")
    assert torch.equal(got, xb.xnor_int4_linear(x, w, bias, out_dtype=out_dtype))
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    ref.assert_within(xb.xnor_int4_linear(x, w, bias, out_dtype=out_dtype, workspace=none), want, bound, "y without a workspace")


@pytest.mark.parametrize("M,F,K", [(70, 520, 9000), (129, 1100, 2600), (700, 555, 1500), (8200, 515, 131)], ids=str)
@pytest.mark.parametrize("dtype,scale_dtype,group,zeros,act,out_dtype", [(BF16, BF16, 64, True, ref.SILU, BF16), (F16, F16, 128, False, ref.GELU, F32)], ids=str)
def test_many_tokens_gated(xb, M, F, K, dtype, scale_dtype, group, zeros, act, out_dtype):
    x = rand(M + F, M, K, dtype=dtype)
    wg, wu = weights(xb, K, F, K, group, zeros, scale_dtype), weights(xb, K + 1, F, K, group, zeros, scale_dtype)
    want, bound = xref.gated(x, wg, wu, act, out_dtype)
    ref.assert_within(xb.xnor_int4_gated(x, wg, wu, act, out_dtype=out_dtype), want, bound, "h")
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    ref.assert_within(xb.xnor_int4_gated(x, wg, wu, act, out_dtype=out_dtype, workspace=none), want, bound, "h without a workspace")


def test_many_tokens_strides_and_what_is_not_finite(xb):
    """As test_strides_and_edges and test_values_that_are_not_finite, on the tiles, in shares of the contraction."""
    M, N, K = 150, 515, 5643
    assert xb.xnor_int4_linear_workspace_bytes(M, N, K) > 0
    w = weights(xb, 3, N, K, 32, True, F16)
    held = torch.as_strided(torch.zeros(N * 2828 + 4, dtype=torch.uint8, device="cuda"), (N, 2824), (2828, 1), 4)
    held.copy_(w.q)
    buffer = torch.full((M + 2, N + 5), 7.0, device="cuda")
    x = rand(1, M, K + 3, dtype=BF16)[:, 3:]
    x[1, 5], x[2, 6], x[3, K - 1] = float("inf"), float("nan"), float("-inf")
    got = xb.xnor_int4_linear(x, w._replace(q=held), out=buffer[1:M + 1, 2:N + 2]).cpu().double()
    clean = x.clone()
    clean[1, 5], clean[2, 6], clean[3, K - 1] = 0.0, 0.0, 0.0
    want, bound = xref.linear(clean, w, None, F32)
    v = xref.values(w)[0]
    want[1] += v[:, 5] * float("inf")
    want[3] += v[:, K - 1] * float("-inf")
    want[2] = float("nan")
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.isinf(), want.isinf())
    assert torch.equal(got[got.isinf()] > 0, want[want.isinf()] > 0)
    fine = torch.isfinite(want)
    assert ((got - want).abs()[fine] <= bound[fine]).all()
    buffer[1:M + 1, 2:N + 2] = 7.0
    assert (buffer == 7.0).all()


def test_many_tokens_replayed(xb):
    """Shares of the contraction in a captured graph, two graphs on one workspace and eager calls in turn."""
    M, N, K = 200, 1024, 4096
    x, w, wu = rand(1, M, K, dtype=BF16), weights(xb, 2, N, K, 128, False, BF16), weights(xb, 3, N, K, 128, False, BF16)
    space = torch.empty(max(xb.xnor_int4_linear_workspace_bytes(M, N, K), xb.xnor_int4_gated_workspace_bytes(M, N, K)), dtype=torch.uint8, device="cuda")
    assert xb.xnor_int4_linear_workspace_bytes(M, N, K) > 0 and xb.xnor_int4_gated_workspace_bytes(M, N, K) > 0
    out = [torch.empty(M, N, dtype=BF16, device="cuda") for _ in range(2)]
    xb.xnor_int4_linear(x, w, workspace=space), xb.xnor_int4_gated(x, w, wu, workspace=space)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.graph(graphs[0]):
        xb.xnor_int4_linear(x, w, out=out[0], workspace=space)
    with torch.cuda.graph(graphs[1]):
        xb.xnor_int4_gated(x, w, wu, h=out[1], workspace=space)
    for seed in range(4, 8):
        x.copy_(rand(seed, M, K, dtype=BF16))
        eager = [xb.xnor_int4_linear(x, w), xb.xnor_int4_gated(x, w, wu)]
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, out))


@pytest.mark.parametrize("T,k,E,K,F,N", [(400, 1, 2, 40, 50, 40), (700, 2, 3, 190, 130, 190), (64, 1, 1, 300, 200, 100), (2, 2, 16, 4000, 40, 600),
                                         (3, 5, 64, 130, 1000, 7)], ids=str)
def test_experts_by_tiles_and_pairs(xb, T, k, E, K, F, N):
    chosen = torch.rand(T, E, generator=torch.Generator().manual_seed(T)).argsort(1)[:, :k].int()
    share = torch.rand(T, k, generator=torch.Generator().manual_seed(1))
    chosen[0, 0] = -1
    wg, wu, wd = stacks(xb, E, K, F, N, 64, True, BF16)
    x = rand(9, T, K, dtype=BF16)
    x[T - 1, K // 2] = float("nan")
    want, bound = xref.experts(x[:T - 1], chosen[:T - 1], share[:T - 1], wg, wu, wd, ref.SILU, F32)
    got = xb.xnor_int4_experts(x, chosen.cuda(), share.cuda(), wg, wu, wd, out_dtype=F32)
    ref.assert_within(got[:T - 1], want, bound, "y")
    assert got[T - 1].isnan().all()


@pytest.mark.parametrize("M,gated", [(100, False), (128, True), (250, False), (130, True)])
def test_as_many_tiles_as_units(xb, M, gated):
    """Wide layers whose tiles of 128 tokens are as many as the units or half of those, in shares of the contraction all the same."""
    N, K = (16384 if gated else 32768) // (1 if M <= 128 else 2), 2560
    ask = xb.xnor_int4_gated_workspace_bytes if gated else xb.xnor_int4_linear_workspace_bytes
    assert ask(M, N, K) > 0
    x, w, wu = rand(1, M, K, dtype=BF16), weights(xb, 2, N, K, 128, False, BF16), weights(xb, 3, N, K, 128, False, BF16)
    out = torch.full((M, N), float("nan"), dtype=F32, device="cuda")
    got = xb.xnor_int4_gated(x, w, wu, h=out) if gated else xb.xnor_int4_linear(x, w, out=out)
    assert torch.isfinite(got).all()
    for part in (slice(0, 150), slice(N - 150, N)):
        of = [m._replace(q=m.q[part], scale=m.scale[:, part].contiguous()) for m in (w, wu)]
        want, bound = xref.gated(x, *of, ref.SILU, F32) if gated else xref.linear(x, of[0], None, F32)
        ref.assert_within(got[:, part], want, bound, "rows")
