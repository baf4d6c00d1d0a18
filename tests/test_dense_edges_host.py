"""Edges of the dense operators that show on the host: workspaces of empty inputs, sizes past 32 bits, rows whose stride means nothing."""
import ctypes
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


class FakeMatrix:
    """What the binding looks at of a tensor on the GPU, without its memory: sizes that this machine does not hold."""
    is_cuda, device = True, "cuda:0"

    def __init__(self, rows, cols, dtype):
        self.shape, self.dtype = (rows, cols), dtype

    def stride(self):
        return (self.shape[1], 1)

    def data_ptr(self):
        return 0x1000

    def is_contiguous(self):
        return True


class FakeVector(FakeMatrix):
    def __init__(self, n, dtype=torch.float32):
        self.shape, self.dtype = (n,), dtype


@pytest.mark.parametrize("past", [1 << 31, (1 << 32) + 8, (1 << 33) + 16])
def test_sizes_past_32_bits_are_refused(xb, monkeypatch, past):
    """A size beyond what the library counts in is refused as one, never taken modulo 2^32 for a smaller one.  (Nothing is launched: the
    library's calls are replaced.)"""
    class Calls:
        def __getattr__(self, name):
            return getattr(xb_lib, name) if name in ("xnor_strerror", "xnor_last_hip_error") else lambda *a: pytest.fail(f"{name}{a}")
    xb_lib = xb.lib
    monkeypatch.setattr(xb, "lib", Calls())
    monkeypatch.setattr(xb, "_stream", lambda: 0)
    f32, f16, i8 = torch.float32, torch.float16, torch.int8
    M = FakeMatrix

    def refused(call, *args, **kw):
        with pytest.raises(xb.XnorError) as e:
            call(*args, **kw)
        assert e.value.status == xb.E_SHAPE
    for rows, cols in ((1, past), (past, 1)):
        n, c = FakeVector(rows), FakeVector(cols)
        refused(xb.xnor_int8_quantize, M(rows, cols, f32), M(rows, cols, i8), n)
        refused(xb.xnor_layer_norm_fwd, M(rows, cols, f16), c, c, 1e-5, M(rows, cols, f16), n, n)
        refused(xb.xnor_layer_norm_fwd_int8, M(rows, cols, f16), c, c, 1e-5, M(rows, cols, i8), n)
        refused(xb.xnor_layer_norm_bwd, M(rows, cols, f32), M(rows, cols, f32), c, n, n, M(rows, cols, f32), c, c)
        # tokens, weights or the contraction of that size
        two = FakeVector(2)
        refused(xb.xnor_int8_matmul, M(rows, cols, i8), n, M(2, cols, i8), two, out=M(rows, 2, f32))
        refused(xb.xnor_int8_matmul, M(2, cols, i8), two, M(rows, cols, i8), n, out=M(2, rows, f32))
        refused(xb.xnor_int8_linear, M(2, cols, f16), M(rows, cols, i8), n, out=M(2, rows, f16))
        refused(xb.xnor_int8_gated, M(2, cols, i8), two, M(rows, cols, i8), n, M(rows, cols, i8), n, h=M(2, rows, f32))
        refused(xb.xnor_gated_fwd, M(2, cols, f16), M(rows, cols, f16), M(rows, cols, f16), h=M(2, rows, f16))
        refused(xb.xnor_gated_bwd, M(2, rows, f16), M(2, cols, f16), M(rows, cols, f16), M(rows, cols, f16), M(2, rows, f16), M(2, rows, f16),
                dx=M(2, cols, f16), dwg=M(rows, cols, f16), dwu=M(rows, cols, f16))
    with pytest.raises(xb.XnorError):
        xb.xnor_int8_linear_workspace_bytes(100, past)
    with pytest.raises(xb.XnorError):
        xb.xnor_layer_norm_bwd_workspace_bytes(f32, 100, past)
    for sizes in ((100, past, 64), (100, 64, past), (past, 64, 64)):
        with pytest.raises(xb.XnorError):
            xb.xnor_gated_bwd_workspace_bytes(*sizes)
        with pytest.raises(xb.XnorError):
            xb.xnor_gated_fwd_workspace_bytes(*sizes, 64, 64)


def test_one_row_has_no_stride(xb, monkeypatch):
    """The stride of a matrix of one row (or none) means nothing: outputs that share one agree whatever theirs are."""
    class Calls:
        def __getattr__(self, name):
            return getattr(xb_lib, name) if name.endswith("_bytes") else lambda *a: calls.append(a) or 0
    xb_lib, calls = xb.lib, []
    monkeypatch.setattr(xb, "lib", Calls())
    monkeypatch.setattr(xb, "_stream", lambda: 0)

    class Apart(FakeMatrix):
        def __init__(self, rows, cols, stride, dtype=torch.float16):
            super().__init__(rows, cols, dtype)
            self.apart = stride

        def stride(self):
            return (self.apart, 1)
    K, F = 64, 24
    w = FakeMatrix(F, K, torch.float16)
    for M in (0, 1):
        x = FakeMatrix(M, K, torch.float16)
        h, g, u = xb.xnor_gated_fwd(x, w, w, h=Apart(M, F, 100), g=Apart(M, F, 48), u=Apart(M, F, 7), want_pre=True)
        assert calls.pop()[14] >= F
        assert u.apart == 7 and g.apart == 48
    one = FakeMatrix(1, K, torch.float16)
    x, dh = FakeMatrix(5, K, torch.float16), FakeMatrix(5, 1, torch.float16)
    xb.xnor_gated_bwd(dh, x, one, one, dh, dh, dx=x, dwg=Apart(1, K, 200), dwu=Apart(1, K, 64), workspace=FakeBytes(1 << 20))
    assert calls.pop()[19] >= K
    # of two rows the strides count
    x = FakeMatrix(2, K, torch.float16)
    with pytest.raises(ValueError):
        xb.xnor_gated_fwd(x, w, w, h=Apart(2, F, 100), g=Apart(2, F, 48), u=Apart(2, F, 24), want_pre=True)


class FakeBytes(FakeVector):
    def __init__(self, n):
        super().__init__(n, torch.uint8)

    def numel(self):
        return self.shape[0]


def test_gated_workspace_for_operands_off_16_bytes(xb, monkeypatch):
    """The copies that a workspace allows are worth as much where an operand starts off 16 bytes, or its rows are too far apart for the
    fetches of whole chunks, as where a stride is odd; the binding asks for one then."""
    M, F, K = 300, 400, 3008
    need = xb.xnor_gated_fwd_workspace_bytes(M, F, K, K + 1, K)
    assert need > 0 and xb.xnor_gated_fwd_workspace_bytes(M, F, K, K, K) == 0
    assert xb.xnor_gated_fwd_workspace_bytes(M, F, K, 1 << 23, K) == need == xb.xnor_gated_fwd_workspace_bytes(M, F, K, K, 1 << 23)
    assert xb.xnor_gated_fwd_workspace_bytes(M, F, K, 1 << 60, K) == need

    class Calls:
        def __getattr__(self, name):
            return getattr(xb_lib, name) if name.endswith("_bytes") else lambda *a: 0
    xb_lib, asked = xb.lib, []
    monkeypatch.setattr(xb, "lib", Calls())
    monkeypatch.setattr(xb, "_stream", lambda: 0)
    monkeypatch.setattr(xb, "_workspace", lambda given, like, nbytes: asked.append(nbytes) or (None, None, 0))

    class At(FakeMatrix):
        def __init__(self, rows, cols, ptr):
            super().__init__(rows, cols, torch.float16)
            self.ptr = ptr

        def data_ptr(self):
            return self.ptr
    h = At(M, F, 0x1000)
    for off in ((0, 0, 0), (2, 0, 0), (0, 8, 0), (0, 0, 14), (0, 16, 32)):
        xb.xnor_gated_fwd(At(M, K, 0x1000 + off[0]), At(F, K, 0x2000 + off[1]), At(F, K, 0x3000 + off[2]), h=h)
        assert asked.pop() == (need if any(o % 16 for o in off) else 0), off


def test_linear_workspace_by_the_layers_width(xb):
    """A few tokens are quantised by the product's own launch in narrow layers only, and a workspace for a launch of theirs in wide ones."""
    ask, least = xb.xnor_int8_linear_layer_workspace_bytes, xb.xnor_int8_linear_workspace_bytes
    for M, K, narrow in ((1, 4096, 16384), (2, 8192, 8192), (3, 2048, 8192), (8, 256, 8192), (9, 1280, 4096), (16, 1, 4096)):
        assert least(M, K) == 0 and ask(M, narrow, K) == 0 and ask(M, 1, K) == 0
        assert ask(M, narrow + 1, K) == ask(M, 50000, K) == M * ((K + 127) // 128 * 128 + 4)
    # where the product's launch does not take them the width makes no difference
    for M, K in ((1, 8193), (3, 2049), (9, 1281), (17, 64), (1000, 4096)):
        assert ask(M, 1, K) == ask(M, 50000, K) == least(M, K) > 0
    assert ask(0, 64, 64) == ask(0, 50000, 64) == 0
    n = ctypes.c_size_t()
    assert xb.lib.xnor_int8_linear_layer_workspace_bytes(4, 64, 64, None) == xb.E_NULL
    for M, N, K in ((-1, 64, 64), (4, 0, 64), (4, 64, 0), (4, 64, 1 << 17), (4, (1 << 26) + 1, 64)):
        assert xb.lib.xnor_int8_linear_layer_workspace_bytes(M, N, K, ctypes.byref(n)) == xb.E_SHAPE


def test_gated_copies_where_they_pay(xb):
    """Sizes at which copying the rows first measured much faster, and much slower, than reading them where they lie."""
    ask = xb.xnor_gated_fwd_workspace_bytes
    for M, F, K in ((1000, 4096, 4095), (8192, 300, 3001), (900, 4000, 2501), (500, 5500, 2501), (4096, 4096, 4095), (300, 1000, 3001), (65, 2501, 2001)):
        assert ask(M, F, K, K, K) > 0, (M, F, K)
    for M, F, K in ((128, 8192, 8191), (4398, 177, 183), (1288, 118, 65), (100, 8192, 1001), (64, 4096, 4095), (1, 4096, 4095)):
        assert ask(M, F, K, K, K) == 0, (M, F, K)


def test_fit_of_erfc():
    """The coefficients in the source against erfc in 64 bits: the fit itself, and what fp32 leaves of it with an exact exponential."""
    np, special = pytest.importorskip("numpy"), pytest.importorskip("scipy.special")
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2007_14178_amd", "csrc")
    body = open(os.path.join(csrc, "dense_common.hpp")).read().split("float erfc_short(float z)")[1].split("\n}")[0]
    p = [float(body.split("float p = ")[1].split("f;")[0])] + [float(sign + c) for sign, c in re.findall(r"p = p \* t ([+-]) ([0-9.]+)f;", body)]
    assert len(p) == 8
    z = np.linspace(0.0, 14.0, 100001)
    t = 1.0 / (1.0 + 0.5 * z)
    assert np.abs(np.polyval(p, t) - np.log(special.erfcx(z) / t)).max() < 7e-7
    z = np.linspace(0.0, 9.0, 300001).astype(np.float32)
    t = np.float32(1.0) / (np.float32(1.0) + np.float32(0.5) * z)
    v = np.full_like(t, np.float32(p[0]))
    for c in p[1:]:
        v = v * t + np.float32(c)
    v = (v - z * z) * np.float32(1.44269504)
    off = np.abs(t.astype(np.float64) * np.exp2(v.astype(np.float64)) / special.erfc(z.astype(np.float64)) - 1.0)
    assert off[z <= 2].max() < 1.2e-6 and off[z <= 5].max() < 3.6e-6 and off.max() < 1.25e-5
