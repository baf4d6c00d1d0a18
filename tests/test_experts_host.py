"""What routing and the products with 4-bit weights refuse, before anything reaches a GPU."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def xb():
    from paper_2007_14178_amd import binding
    return binding


OK, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1001)


def with_bad(good, call, cases):
    """`call` on `good` with one argument replaced, and the status that is expected."""
    for at, value, status in cases:
        args = list(good)
        args[at] = value
        assert call(*args) == status, f"argument {at} = {value}"


def matrix(xb, **changed):
    m = dict(q=0x1000, q_stride=32, scale=0x2000, zero=0x3000, rows=8, cols=64, group=32, scale_type=2)
    m.update(changed)
    return xb.CInt4(*(m[k] for k in ("q", "q_stride", "scale", "zero", "rows", "cols", "group", "scale_type")))


BAD_MATRICES = [(dict(q=None), "E_NULL"), (dict(scale=None), "E_NULL"), (dict(scale_type=3), "E_UNSUPPORTED"), (dict(group=48), "E_UNSUPPORTED"),
                (dict(group=0), "E_UNSUPPORTED"), (dict(rows=0), "E_SHAPE"), (dict(cols=0), "E_SHAPE"), (dict(cols=-5), "E_SHAPE"),
                (dict(rows=(1 << 26) + 1), "E_SHAPE"), (dict(q_stride=28), "E_SHAPE"), (dict(q_stride=-32), "E_SHAPE"), (dict(q_stride=34), "E_ALIGN"),
                (dict(q=0x1002), "E_ALIGN"), (dict(scale=0x2001), "E_ALIGN"), (dict(q_stride=1 << 60), "E_SHAPE")]


def bad_matrices(xb, at):
    return [(at, ctypes.byref(matrix(xb, **changed)), getattr(xb, status)) for changed, status in BAD_MATRICES] + [(at, None, xb.E_NULL)]


def test_quantize_refuses(xb):
    # (w, type, rows, cols, w_stride, group, q, q_stride, scale, scale_type, zero, stream)
    with_bad([OK, 0, 4, 64, 64, 32, OK, 32, OK, 2, None, None], xb.lib.xnor_int4_quantize, [
        (0, None, xb.E_NULL), (6, None, xb.E_NULL), (8, None, xb.E_NULL), (1, 3, xb.E_UNSUPPORTED), (9, -1, xb.E_UNSUPPORTED), (5, 16, xb.E_UNSUPPORTED),
        (2, -1, xb.E_SHAPE), (3, 0, xb.E_SHAPE), (4, -1, xb.E_SHAPE), (7, 28, xb.E_SHAPE), (7, 33, xb.E_ALIGN), (0, ODD, xb.E_ALIGN), (6, ODD, xb.E_ALIGN),
        (8, ODD, xb.E_ALIGN)])
    # (levels, rows, cols, stride, q, q_stride, stream)
    with_bad([OK, 4, 64, 64, OK, 32, None], xb.lib.xnor_int4_pack, [
        (0, None, xb.E_NULL), (4, None, xb.E_NULL), (1, -1, xb.E_SHAPE), (2, 0, xb.E_SHAPE), (5, 28, xb.E_SHAPE), (5, 34, xb.E_ALIGN), (4, ODD, xb.E_ALIGN)])
    with_bad([ctypes.byref(matrix(xb)), OK, 0, 64, None], xb.lib.xnor_int4_dequantize, [
        (1, None, xb.E_NULL), (2, 5, xb.E_UNSUPPORTED), (3, 63, xb.E_SHAPE), (1, ODD, xb.E_ALIGN), *bad_matrices(xb, 0)])


def test_linear_refuses(xb):
    # (x, type, x_stride, w, bias, M, out, out_type, out_stride, workspace, bytes, stream)
    with_bad([OK, 2, 64, ctypes.byref(matrix(xb)), None, 4, OK, 2, 8, None, 0, None], xb.lib.xnor_int4_linear, [
        (0, None, xb.E_NULL), (6, None, xb.E_NULL), (1, 0, xb.E_UNSUPPORTED), (7, 3, xb.E_UNSUPPORTED), (5, -1, xb.E_SHAPE), (2, -1, xb.E_SHAPE),
        (8, 7, xb.E_SHAPE), (0, ODD, xb.E_ALIGN), (4, ODD, xb.E_ALIGN), (6, ODD, xb.E_ALIGN), (9, ctypes.c_void_p(0x1008), xb.E_ALIGN), *bad_matrices(xb, 3)])
    n = ctypes.c_size_t()
    assert xb.lib.xnor_int4_linear_workspace_bytes(4, 8, 64, None) == xb.E_NULL
    for sizes in ((-1, 8, 64), (4, 0, 64), (4, 8, 0)):
        assert xb.lib.xnor_int4_linear_workspace_bytes(*sizes, ctypes.byref(n)) == xb.E_SHAPE


def test_gated_refuses(xb):
    other = [(dict(rows=7), xb.E_SHAPE), (dict(cols=63), xb.E_SHAPE), (dict(group=64), xb.E_SHAPE), (dict(q_stride=36), xb.E_SHAPE),
             (dict(scale_type=1), xb.E_UNSUPPORTED), (dict(zero=None), xb.E_UNSUPPORTED)]
    # (x, type, x_stride, wg, wu, act, M, h, h_type, h_stride, workspace, bytes, stream)
    with_bad([OK, 1, 64, ctypes.byref(matrix(xb)), ctypes.byref(matrix(xb)), 0, 4, OK, 1, 8, None, 0, None], xb.lib.xnor_int4_gated, [
        (0, None, xb.E_NULL), (7, None, xb.E_NULL), (1, 0, xb.E_UNSUPPORTED), (5, 3, xb.E_UNSUPPORTED), (8, 3, xb.E_UNSUPPORTED), (6, -1, xb.E_SHAPE),
        (9, 7, xb.E_SHAPE), (0, ODD, xb.E_ALIGN), (7, ODD, xb.E_ALIGN), *bad_matrices(xb, 3), *bad_matrices(xb, 4),
        *((4, ctypes.byref(matrix(xb, **changed)), status) for changed, status in other)])


def test_route_refuses(xb):
    # (logits, type, T, E, stride, bias, score, groups, kept, top, k, renorm, factor, experts, weights, stream)
    with_bad([OK, 0, 4, 64, 64, OK, 1, 8, 2, 2, 8, 1, 1.0, OK, OK, None], xb.lib.xnor_route_fwd, [
        (0, None, xb.E_NULL), (13, None, xb.E_NULL), (14, None, xb.E_NULL), (1, 3, xb.E_UNSUPPORTED), (6, 2, xb.E_UNSUPPORTED), (2, -1, xb.E_SHAPE),
        (3, 0, xb.E_SHAPE), (3, 1025, xb.E_SHAPE), (4, -1, xb.E_SHAPE), (7, 0, xb.E_SHAPE), (7, 7, xb.E_SHAPE), (8, 0, xb.E_SHAPE), (8, 9, xb.E_SHAPE),
        (9, 0, xb.E_SHAPE), (9, 3, xb.E_SHAPE), (10, 0, xb.E_SHAPE), (10, 17, xb.E_SHAPE), (10, 33, xb.E_SHAPE), (2, 1 << 28, xb.E_SHAPE),
        (0, ODD, xb.E_ALIGN), (5, ODD, xb.E_ALIGN), (13, ODD, xb.E_ALIGN), (14, ODD, xb.E_ALIGN)])
    # (dweights, logits, type, T, E, stride, experts, k, score, renorm, factor, dlogits, dstride, stream)
    with_bad([OK, OK, 1, 4, 64, 64, OK, 8, 0, 1, 1.0, OK, 64, None], xb.lib.xnor_route_bwd, [
        (0, None, xb.E_NULL), (1, None, xb.E_NULL), (6, None, xb.E_NULL), (11, None, xb.E_NULL), (2, 3, xb.E_UNSUPPORTED), (8, 2, xb.E_UNSUPPORTED),
        (3, -1, xb.E_SHAPE), (4, 1025, xb.E_SHAPE), (7, 0, xb.E_SHAPE), (7, 33, xb.E_SHAPE), (12, 63, xb.E_SHAPE), (0, ODD, xb.E_ALIGN),
        (1, ODD, xb.E_ALIGN), (6, ODD, xb.E_ALIGN), (11, ODD, xb.E_ALIGN)])


def test_lists_refuse(xb):
    need = xb.xnor_route_lists_workspace_bytes(1000, 8, 64)
    assert need > 0 and xb.xnor_route_lists_workspace_bytes(128, 8, 64) == 0
    # (experts, T, k, E, offsets, order, workspace, bytes, stream)
    with_bad([OK, 1000, 8, 64, OK, OK, OK, need, None], xb.lib.xnor_route_lists, [
        (0, None, xb.E_NULL), (4, None, xb.E_NULL), (5, None, xb.E_NULL), (6, None, xb.E_NULL), (1, -1, xb.E_SHAPE), (2, 0, xb.E_SHAPE), (2, 33, xb.E_SHAPE),
        (3, 0, xb.E_SHAPE), (3, 1025, xb.E_SHAPE), (1, 1 << 28, xb.E_SHAPE), (0, ODD, xb.E_ALIGN), (4, ODD, xb.E_ALIGN), (5, ODD, xb.E_ALIGN),
        (6, ctypes.c_void_p(0x1008), xb.E_ALIGN), (7, need - 1, xb.E_WORKSPACE)])
    assert xb.lib.xnor_route_lists_workspace_bytes(4, 8, 64, None) == xb.E_NULL


def test_experts_refuse(xb):
    w, d = matrix(xb, rows=16), matrix(xb, rows=64, cols=16, q_stride=8)
    need = xb.xnor_int4_experts_workspace_bytes(4, 2, 5, 64, 16, 64)
    # (x, type, x_stride, T, experts, weights, k, E, wg, wu, wd, act, out, out_type, out_stride, workspace, bytes, stream)
    good = [OK, 2, 64, 4, OK, OK, 2, 5, ctypes.byref(w), ctypes.byref(w), ctypes.byref(d), 0, OK, 2, 64, OK, need, None]
    with_bad(good, xb.lib.xnor_int4_experts, [
        (0, None, xb.E_NULL), (4, None, xb.E_NULL), (5, None, xb.E_NULL), (12, None, xb.E_NULL), (15, None, xb.E_NULL), (1, 0, xb.E_UNSUPPORTED),
        (11, 3, xb.E_UNSUPPORTED), (13, 3, xb.E_UNSUPPORTED), (3, -1, xb.E_SHAPE), (6, 0, xb.E_SHAPE), (6, 33, xb.E_SHAPE), (7, 0, xb.E_SHAPE),
        (7, 1025, xb.E_SHAPE), (3, 1 << 30, xb.E_SHAPE), (14, 63, xb.E_SHAPE), (10, ctypes.byref(matrix(xb, rows=64, cols=24, q_stride=12)), xb.E_SHAPE),
        (0, ODD, xb.E_ALIGN), (4, ODD, xb.E_ALIGN), (5, ODD, xb.E_ALIGN), (12, ODD, xb.E_ALIGN), (15, ctypes.c_void_p(0x1008), xb.E_ALIGN),
        (16, need - 1, xb.E_WORKSPACE), *bad_matrices(xb, 8), *bad_matrices(xb, 9), *bad_matrices(xb, 10)])
    assert xb.lib.xnor_int4_experts_workspace_bytes(4, 2, 5, 64, 16, 64, None) == xb.E_NULL
    assert xb.xnor_int4_experts_workspace_bytes(0, 2, 5, 64, 16, 64) == 0


def test_binding_refuses(xb):
    """Tensors that are not on a GPU, of another type or another shape."""
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    w = xb.Int4(torch.zeros(8, 32, dtype=torch.uint8), torch.ones(2, 8), None, 64, 32)
    with pytest.raises(TypeError):
        xb.xnor_int4_linear(x, w)
    with pytest.raises(TypeError):
        xb.xnor_int4_dequantize(w)
    with pytest.raises(ValueError):
        xb.xnor_int4_dequantize(w._replace(cols=72))
    with pytest.raises(xb.XnorError):
        xb.xnor_int4_dequantize(w._replace(group=16))
    with pytest.raises(xb.XnorError):
        xb.xnor_int4_quantize(x, group=100)
    for call in (lambda: xb.xnor_route_fwd(x, 2), lambda: xb.xnor_route_lists(torch.zeros(4, 2, dtype=torch.int32), 8),
                 lambda: xb.xnor_int4_pack(torch.zeros(4, 8, dtype=torch.uint8)), lambda: xb.xnor_int4_quantize(x)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        xb.xnor_route_lists(torch.zeros(4, dtype=torch.int32), 8)
    with pytest.raises(TypeError):
        xb.xnor_route_lists(torch.zeros(4, 2, dtype=torch.int64), 8)
