"""Edges of the dense operators that show on the host: workspaces of empty inputs, sizes past 32 bits, rows whose stride means nothing."""
import os
import re

import pytest
import torch


@pytest.fixture(scope="module")
def xb():
    from paper_2007_14178_amd import binding
    return binding


@pytest.mark.parametrize("dtype,cols", [(torch.float32, 8), (torch.float32, 8196), (torch.float32, 9000), (torch.bfloat16, 600), (torch.bfloat16, 16392),
                                        (torch.float16, 20000)], ids=str)
def test_norm_back_workspace_without_rows(xb, dtype, cols):
    """Gradients of the parameters need a workspace, and a caller who asks for its size gets one, however many rows there are."""
    assert xb.xnor_layer_norm_bwd_workspace_bytes(dtype, 0, cols) >= 2 * 4 * cols


def test_asm_tells_the_compiler_of_m0():
    """Loads into LDS take their place from m0.  A compiler that is not told keeps or moves values of its own there: the register is an
    operand of the statement, and no statement's text writes it."""
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2007_14178_amd", "csrc")
    users = 0
    for name in sorted(os.listdir(csrc)):
        text = open(os.path.join(csrc, name)).read()
        for statement in re.findall(r"\basm\b[^;{}]*?\((?:\"(?:[^\"\\]|\\.)*\"|[^\";])*;", text):
            assert not re.search(r"\bs_\w+ m0\b", statement), f"{name}: {statement}"
            if re.search(r"\blds\b", statement):
                users += 1
                assert '"{m0}"' in statement, f"{name}: {statement}"
    assert users > 0
