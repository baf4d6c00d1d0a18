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
