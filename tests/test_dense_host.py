"""What the dense operators refuse, before anything reaches a GPU."""
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


def test_quantize_refuses(xb):
    # (x, type, rows, cols, x_stride, q, q_stride, scale, stream)
    with_bad([OK, 0, 4, 8, 8, OK, 8, OK, None], xb.lib.xnor_int8_quantize, [
        (0, None, xb.E_NULL), (5, None, xb.E_NULL), (7, None, xb.E_NULL), (1, 3, xb.E_UNSUPPORTED), (1, -1, xb.E_UNSUPPORTED),
        (2, -1, xb.E_SHAPE), (2, 1 << 31, xb.E_SHAPE), (3, 0, xb.E_SHAPE), (3, (1 << 30) + 1, xb.E_SHAPE), (4, -1, xb.E_SHAPE),
        (4, 1 << 60, xb.E_SHAPE), (6, 7, xb.E_SHAPE), (0, ODD, xb.E_ALIGN), (7, ODD, xb.E_ALIGN)])


def test_int8_matmul_refuses(xb):
    # (a, a_stride, a_scale, b, b_stride, b_scale, bias, M, N, K, out, type, out_stride, stream)
    with_bad([OK, 64, OK, OK, 64, OK, None, 4, 8, 64, OK, 1, 8, None], xb.lib.xnor_int8_matmul, [
        (0, None, xb.E_NULL), (2, None, xb.E_NULL), (3, None, xb.E_NULL), (5, None, xb.E_NULL), (10, None, xb.E_NULL), (11, 9, xb.E_UNSUPPORTED),
        (7, -1, xb.E_SHAPE), (8, 0, xb.E_SHAPE), (9, 0, xb.E_SHAPE), (9, 1 << 17, xb.E_SHAPE), (1, -64, xb.E_SHAPE), (12, 7, xb.E_SHAPE),
        (2, ODD, xb.E_ALIGN), (5, ODD, xb.E_ALIGN), (6, ODD, xb.E_ALIGN), (10, ODD, xb.E_ALIGN)])


def test_int8_linear_refuses(xb):
    need = xb.xnor_int8_linear_workspace_bytes(40, 64)
    # (x, type, x_stride, w, w_stride, w_scale, bias, M, N, K, out, type, out_stride, workspace, bytes, stream)
    with_bad([OK, 2, 64, OK, 64, OK, None, 40, 8, 64, OK, 2, 8, OK, need, None], xb.lib.xnor_int8_linear, [
        (0, None, xb.E_NULL), (3, None, xb.E_NULL), (5, None, xb.E_NULL), (10, None, xb.E_NULL), (13, None, xb.E_NULL), (1, 7, xb.E_UNSUPPORTED),
        (11, 3, xb.E_UNSUPPORTED), (9, 1 << 17, xb.E_SHAPE), (8, -1, xb.E_SHAPE), (12, 7, xb.E_SHAPE), (0, ODD, xb.E_ALIGN),
        (13, ctypes.c_void_p(0x1008), xb.E_ALIGN), (14, need - 1, xb.E_WORKSPACE)])
    n = ctypes.c_size_t()
    assert xb.lib.xnor_int8_linear_workspace_bytes(4, 64, None) == xb.E_NULL
    for M, K in ((-1, 64), (4, 0), (4, 1 << 17)):
        assert xb.lib.xnor_int8_linear_workspace_bytes(M, K, ctypes.byref(n)) == xb.E_SHAPE
    assert xb.xnor_int8_linear_workspace_bytes(0, 64) == 0


def test_int8_gated_refuses(xb):
    # (a, a_stride, a_scale, wg, sg, wu, su, w_stride, act, M, F, K, h, type, h_stride, stream)
    with_bad([OK, 64, OK, OK, OK, OK, OK, 64, 0, 4, 8, 64, OK, 0, 8, None], xb.lib.xnor_int8_gated, [
        *((k, None, xb.E_NULL) for k in (0, 2, 3, 4, 5, 6, 12)), (8, 3, xb.E_UNSUPPORTED), (13, 3, xb.E_UNSUPPORTED), (9, -1, xb.E_SHAPE),
        (10, 0, xb.E_SHAPE), (11, 1 << 17, xb.E_SHAPE), (14, 7, xb.E_SHAPE), (2, ODD, xb.E_ALIGN), (4, ODD, xb.E_ALIGN), (12, ODD, xb.E_ALIGN)])


def test_norm_refuses(xb):
    # (x, type, rows, cols, x_stride, gamma, beta, p_type, eps, y, y_stride, mean, rstd, stream)
    bad = [(0, None, xb.E_NULL), (9, None, xb.E_NULL), (1, 5, xb.E_UNSUPPORTED), (7, 2, xb.E_UNSUPPORTED), (2, -1, xb.E_SHAPE), (3, 0, xb.E_SHAPE),
           (4, -8, xb.E_SHAPE), (10, 7, xb.E_SHAPE), (8, -1.0, xb.E_SHAPE), (8, float("nan"), xb.E_SHAPE), (0, ODD, xb.E_ALIGN), (5, ODD, xb.E_ALIGN)]
    with_bad([OK, 1, 4, 8, 8, OK, OK, 0, 1e-5, OK, 8, OK, OK, None], xb.lib.xnor_layer_norm_fwd, bad + [(9, ODD, xb.E_ALIGN), (12, ODD, xb.E_ALIGN)])
    # (..., q, q_stride, scale, mean, rstd, stream)
    with_bad([OK, 1, 4, 8, 8, OK, OK, 0, 1e-5, OK, 8, OK, None, None, None], xb.lib.xnor_layer_norm_fwd_int8, bad + [(11, None, xb.E_NULL)])


def test_norm_back_refuses(xb):
    need = xb.xnor_layer_norm_bwd_workspace_bytes(torch.float16, 4, 8)
    # (dy, dy_stride, x, type, rows, cols, x_stride, gamma, p_type, mean, rstd, dx, dx_stride, dgamma, dbeta, workspace, bytes, stream)
    with_bad([OK, 8, OK, 1, 4, 8, 8, OK, 0, OK, OK, OK, 8, OK, OK, OK, need, None], xb.lib.xnor_layer_norm_bwd, [
        *((k, None, xb.E_NULL) for k in (0, 2, 9, 10, 11, 13, 14, 15)), (3, 4, xb.E_UNSUPPORTED), (8, 2, xb.E_UNSUPPORTED), (4, -1, xb.E_SHAPE),
        (5, 0, xb.E_SHAPE), (12, 7, xb.E_SHAPE), (0, ODD, xb.E_ALIGN), (13, ODD, xb.E_ALIGN), (15, ctypes.c_void_p(0x1004), xb.E_ALIGN),
        (16, need - 1, xb.E_WORKSPACE)])
    n = ctypes.c_size_t()
    assert xb.lib.xnor_layer_norm_bwd_workspace_bytes(0, 4, 8, None) == xb.E_NULL
    assert xb.lib.xnor_layer_norm_bwd_workspace_bytes(9, 4, 8, ctypes.byref(n)) == xb.E_UNSUPPORTED
    assert xb.lib.xnor_layer_norm_bwd_workspace_bytes(0, -1, 8, ctypes.byref(n)) == xb.E_SHAPE


def test_gated_refuses(xb):
    # (x, type, x_stride, wg, wu, w_stride, act, M, F, K, h, h_stride, g, u, gu_stride, stream)
    with_bad([OK, 1, 64, OK, OK, 64, 0, 4, 8, 64, OK, 8, OK, OK, 8, None], xb.lib.xnor_gated_fwd, [
        *((k, None, xb.E_NULL) for k in (0, 3, 4, 10, 12, 13)), (1, 0, xb.E_UNSUPPORTED), (6, 3, xb.E_UNSUPPORTED), (7, -1, xb.E_SHAPE),
        (8, 0, xb.E_SHAPE), (9, 0, xb.E_SHAPE), (11, 7, xb.E_SHAPE), (14, 7, xb.E_SHAPE), (0, ODD, xb.E_ALIGN), (4, ODD, xb.E_ALIGN)])
    # (..., gu_stride, workspace, bytes, stream): a workspace is optional, but has to be aligned
    with_bad([OK, 1, 64, OK, OK, 64, 0, 4, 8, 64, OK, 8, OK, OK, 8, OK, 64, None], xb.lib.xnor_gated_fwd_ws, [
        *((k, None, xb.E_NULL) for k in (0, 3, 4, 10, 12, 13)), (1, 0, xb.E_UNSUPPORTED), (9, 0, xb.E_SHAPE), (15, ctypes.c_void_p(0x1008), xb.E_ALIGN)])
    n = ctypes.c_size_t()
    assert xb.lib.xnor_gated_fwd_workspace_bytes(4, 8, 64, 64, 64, None) == xb.E_NULL
    for M, F, K, stride in ((-1, 8, 64, 64), (4, 0, 64, 64), (4, 8, 0, 64), (4, 8, 64, -1)):
        assert xb.lib.xnor_gated_fwd_workspace_bytes(M, F, K, stride, 64, ctypes.byref(n)) == xb.E_SHAPE
    need = xb.xnor_gated_bwd_workspace_bytes(4, 8, 64)
    # (dh, dh_stride, x, type, x_stride, wg, wu, w_stride, g, u, gu_stride, act, M, F, K, dx, dx_stride, dwg, dwu, dw_stride, workspace, bytes, stream)
    with_bad([OK, 8, OK, 1, 64, OK, OK, 64, OK, OK, 8, 0, 4, 8, 64, OK, 64, OK, OK, 64, OK, need, None], xb.lib.xnor_gated_bwd, [
        *((k, None, xb.E_NULL) for k in (0, 2, 5, 6, 8, 9, 15, 17, 18, 20)), (3, 0, xb.E_UNSUPPORTED), (11, -1, xb.E_UNSUPPORTED), (12, -1, xb.E_SHAPE),
        (16, 63, xb.E_SHAPE), (19, 63, xb.E_SHAPE), (8, ODD, xb.E_ALIGN), (20, ctypes.c_void_p(0x1008), xb.E_ALIGN), (21, need - 1, xb.E_WORKSPACE)])
    n = ctypes.c_size_t()
    assert xb.lib.xnor_gated_bwd_workspace_bytes(4, 8, 64, None) == xb.E_NULL
    for M, F, K in ((-1, 8, 8), (4, 0, 8), (4, 1 << 30, 8), (4, 8, 0)):
        assert xb.lib.xnor_gated_bwd_workspace_bytes(M, F, K, ctypes.byref(n)) == xb.E_SHAPE


def test_binding_refuses(xb):
    """Tensors that are on the CPU, of another type or another shape."""
    x = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        xb.xnor_int8_quantize(x)
    with pytest.raises(TypeError):
        xb.xnor_int8_quantize(x.to(torch.float64))
    with pytest.raises(ValueError):
        xb.xnor_layer_norm_fwd(x[0], None, None)
    with pytest.raises(TypeError):
        xb.xnor_gated_fwd(x.half(), x.half(), x.half())
