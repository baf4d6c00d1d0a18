"""Experts' calls that are taken in runs: of more pairs than the workspace is for, and of tokens that lie further apart than a tile's 31-bit offsets reach.  Whole
numbers, compared by equality."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import dense_reference as ref  # noqa: E402
from test_gpu_experts_hidden import definition, stack  # noqa: E402

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def xb():
    from paper_2007_14178_amd import binding
    return binding


def case(xb, T, k, E, K, F, N):
    gen = torch.Generator().manual_seed(T)
    w = stack(xb, gen, E, F, K, 32, True, BF16), stack(xb, gen, E, F, K, 32, True, BF16), stack(xb, gen, E, N, F, 32, True, BF16)
    x = torch.randint(-1, 2, (T, K), generator=gen).to(BF16)
    chosen = torch.rand(T, E, generator=gen).argsort(1)[:, :k].int()
    chosen[5, 0] = -1
    return x, chosen, 2.0 ** torch.randint(-1, 1, (T, k), generator=gen).float(), w


def test_the_workspace_does_not_grow_with_runs(xb):
    sizes = (8, 64, 2048, 1024, 2048)
    most = xb.xnor_int4_experts_workspace_bytes(1 << 15, *sizes)
    assert xb.xnor_int4_experts_workspace_bytes((1 << 15) - 1, *sizes) < most
    for T in ((1 << 15) + 1, 1 << 20, 1 << 27):
        assert xb.xnor_int4_experts_workspace_bytes(T, *sizes) == most


@pytest.mark.parametrize("T,k,E", [(131073, 2, 5), (70000, 4, 6), (300000, 1, 3)], ids=str)
def test_more_pairs_than_a_run(xb, T, k, E):
    x, chosen, share, w = case(xb, T, k, E, 24, 20, 36)
    out = torch.full((T + 1, 40), 3.0, device="cuda")
    xb.xnor_int4_experts(x.cuda(), chosen.cuda(), share.cuda(), *w, act=ref.RELU, out=out[:T, :36])
    run = (1 << 18) // k
    rows = torch.unique(torch.cat((torch.arange(200), torch.arange(run - 100, min(run + 100, T)), torch.arange(T - 100, T), torch.randint(0, T, (2000,)))))
    want, _, reach = definition(x[rows], chosen[rows], share[rows], *w)
    assert float(reach.max()) < 2.0 ** 23
    assert torch.equal(out[rows.cuda(), :36].cpu().double(), want)
    assert (out[T] == 3.0).all() and (out[:, 36:] == 3.0).all()


@pytest.mark.parametrize("T,apart", [(600, 1 << 21), (3000, 1 << 19)], ids=str)
def test_tokens_far_apart(xb, T, apart):
    """Rows of a buffer of 2.5 to 3 GB: in runs, or where these would be short by the kernel for few tokens."""
    x, chosen, share, w = case(xb, T, 2, 3, 24, 20, 36)
    held = torch.empty((T - 1) * apart + 24, dtype=BF16, device="cuda")
    far = held.as_strided((T, 24), (apart, 1))
    far.copy_(x)
    assert (T - 1) * apart * 2 > 1 << 31
    want, _, _ = definition(x, chosen, share, *w)
    got = xb.xnor_int4_experts(far, chosen.cuda(), share.cuda(), *w, act=ref.RELU, out_dtype=F32)
    assert torch.equal(got.cpu().double(), want)


def test_runs_replayed(xb):
    """A call of two runs and one of a single run captured with one workspace, replayed in turn with other tokens beside eager calls."""
    T, k, E = 131073, 2, 5
    x, chosen, share, w = case(xb, T, k, E, 24, 20, 36)
    x, chosen, share = x.cuda(), chosen.cuda(), share.cuda()
    space = torch.empty(xb.xnor_int4_experts_workspace_bytes(T, k, E, 24, 20, 36), dtype=torch.uint8, device="cuda")
    outs = [torch.empty(n, 36, device="cuda") for n in (T, 700)]

    def call(n, out=None, workspace=None):
        return xb.xnor_int4_experts(x[:n], chosen[:n], share[:n], *w, act=ref.RELU, out=out, out_dtype=F32 if out is None else None, workspace=workspace)
    for out in outs:
        call(len(out), out, space)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for graph, out in zip(graphs, outs):
        with torch.cuda.graph(graph):
            call(len(out), out, space)
    for seed in range(3):
        x.copy_(torch.randint(-1, 2, x.shape, generator=torch.Generator().manual_seed(seed)))
        eager = [call(len(out)) for out in outs]
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, outs))
