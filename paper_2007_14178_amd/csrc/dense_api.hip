// Host side of the dense layers' part of the C ABI: argument validation, then the launchers.
#include <algorithm>

#include "dense_check.hpp"

namespace {

using namespace xnor;

constexpr int kMaxInt8Cols = (1 << 17) - 1;        // |sum of K products of two int8| <= K 2^14 < 2^31

int norm_types(int x_type, int p_type, int *xs, int *ps)
{
    *xs = value_size(x_type), *ps = value_size(p_type);
    return *xs && *ps && (p_type == XNOR_TYPE_FP32 || p_type == x_type) ? XNOR_OK : XNOR_E_UNSUPPORTED;
}

int norm_forward(const void *x, int x_type, long long rows, int cols, long long x_stride, const void *gamma, const void *beta, int p_type,
                 float eps, const Matrix &out, int8_t *q, float *scale, float *mean, float *rstd, void *stream)
{
    int xs, ps, rc = norm_types(x_type, p_type, &xs, &ps);
    if (rc) return rc;
    const Matrix all[] = {{x, rows, cols, x_stride, xs, false}, out, vec(scale, q ? rows : 0, 4)};
    if ((rc = check(all))) return rc;
    if (!(eps >= 0.f)) return XNOR_E_SHAPE;
    if (!aligned(gamma, ps) || !aligned(beta, ps) || !aligned(mean, 4) || !aligned(rstd, 4)) return XNOR_E_ALIGN;
    RowArgs a{};
    a.x = x, a.rows = rows, a.cols = cols, a.x_stride = x_stride;
    a.gamma = gamma, a.beta = beta, a.eps = eps;
    a.y = q ? nullptr : const_cast<void *>(out.p), a.q = q, a.y_stride = out.stride;
    a.scale = scale, a.mean = mean, a.rstd = rstd;
    return hip_status(launch_layer_norm(a, x_type, p_type, (hipStream_t)stream));
}

size_t q_stride_of(int K) { return ((size_t)K + 127) / 128 * 128; }       // whole cache lines
size_t linear_workspace(long long M, int K) { return (size_t)M * (q_stride_of(K) + sizeof(float)); }

}  // namespace

extern "C" {

int xnor_int8_quantize(const void *x, int x_type, long long rows, int cols, long long x_stride, int8_t *q, long long q_stride, float *scale,
                       void *stream)
{
    const int xs = value_size(x_type);
    if (!xs) return XNOR_E_UNSUPPORTED;
    const Matrix all[] = {{x, rows, cols, x_stride, xs, false}, {q, rows, cols, q_stride, 1, true}, vec(scale, rows, 4, true)};
    if (const int rc = check(all)) return rc;
    RowArgs a{};
    a.x = x, a.rows = rows, a.cols = cols, a.x_stride = x_stride, a.q = q, a.y_stride = q_stride, a.scale = scale;
    return hip_status(launch_quantize(a, x_type, (hipStream_t)stream));
}

int xnor_int8_matmul(const int8_t *a, long long a_stride, const float *a_scale, const int8_t *b, long long b_stride, const float *b_scale,
                     const float *bias, long long M, int N, int K, void *out, int out_type, long long out_stride, void *stream)
{
    const int os = value_size(out_type);
    if (!os) return XNOR_E_UNSUPPORTED;
    const Matrix all[] = {{a, M, K, a_stride, 1, false}, vec(a_scale, M, 4), {b, N, K, b_stride, 1, false}, vec(b_scale, N, 4),
                          {out, M, N, out_stride, os, true}};
    if (const int rc = check(all)) return rc;
    if (K > kMaxInt8Cols) return XNOR_E_SHAPE;
    if (!aligned(bias, 4)) return XNOR_E_ALIGN;
    DenseArgs d{};
    d.a = a, d.lda = a_stride, d.a_scale = a_scale, d.b = b, d.ldb = b_stride, d.b_scale = b_scale, d.bias = bias;
    d.M = M, d.N = N, d.K = K, d.out = out, d.ldo = out_stride;
    return hip_status(launch_dense_int8(d, out_type, (hipStream_t)stream));
}

int xnor_int8_linear_workspace_bytes(long long M, int K, size_t *bytes)
{
    if (!bytes) return XNOR_E_NULL;
    if (M < 0 || M > kMaxRows || K <= 0 || K > kMaxInt8Cols) return XNOR_E_SHAPE;
    *bytes = dense_few_real_supports(M, K) ? 0 : linear_workspace(M, K);
    return XNOR_OK;
}

int xnor_int8_linear_layer_workspace_bytes(long long M, int N, int K, size_t *bytes)
{
    if (const int rc = xnor_int8_linear_workspace_bytes(M, K, bytes)) return rc;
    if (N <= 0 || N > kMaxCols) return XNOR_E_SHAPE;
    if (!dense_few_real_pays(M, N)) *bytes = linear_workspace(M, K);
    return XNOR_OK;
}

int xnor_int8_linear(const void *x, int x_type, long long x_stride, const int8_t *w, long long w_stride, const float *w_scale, const float *bias,
                     long long M, int N, int K, void *out, int out_type, long long out_stride, void *workspace, size_t workspace_bytes,
                     void *stream)
{
    const int xs = value_size(x_type), os = value_size(out_type);
    if (!xs || !os) return XNOR_E_UNSUPPORTED;
    size_t need;
    if (const int rc = xnor_int8_linear_workspace_bytes(M, K, &need)) return rc;
    const Matrix all[] = {{x, M, K, x_stride, xs, false}, {w, N, K, w_stride, 1, false}, vec(w_scale, N, 4), {out, M, N, out_stride, os, true},
                          vec(workspace, need ? M : 0, 16)};
    if (const int rc = check(all)) return rc;
    if (!aligned(bias, 4)) return XNOR_E_ALIGN;
    if (workspace_bytes < need) return XNOR_E_WORKSPACE;
    const bool alone = need > 0 || (workspace && workspace_bytes >= linear_workspace(M, K) && !dense_few_real_pays(M, N));
    if (M > 0 && !alone) {
        DenseArgs d{};
        d.a = x, d.lda = x_stride * xs, d.b = w, d.ldb = w_stride, d.b_scale = w_scale, d.bias = bias;
        d.M = M, d.N = N, d.K = K, d.out = out, d.ldo = out_stride;
        return hip_status(launch_dense_few_real(d, x_type, out_type, (hipStream_t)stream));
    }
    int8_t *q = (int8_t *)workspace;
    const long long q_stride = (long long)q_stride_of(K);
    float *scale = (float *)(q + M * q_stride);
    if (const int rc = xnor_int8_quantize(x, x_type, M, K, x_stride, q, q_stride, scale, stream)) return rc;
    return xnor_int8_matmul(q, q_stride, scale, w, w_stride, w_scale, bias, M, N, K, out, out_type, out_stride, stream);
}

int xnor_layer_norm_fwd(const void *x, int x_type, long long rows, int cols, long long x_stride, const void *gamma, const void *beta, int p_type,
                        float eps, void *y, long long y_stride, float *mean, float *rstd, void *stream)
{
    return norm_forward(x, x_type, rows, cols, x_stride, gamma, beta, p_type, eps, {y, rows, cols, y_stride, std::max(1, value_size(x_type)), true},
                        nullptr, nullptr, mean, rstd, stream);
}

int xnor_layer_norm_fwd_int8(const void *x, int x_type, long long rows, int cols, long long x_stride, const void *gamma, const void *beta,
                             int p_type, float eps, int8_t *q, long long q_stride, float *scale, float *mean, float *rstd, void *stream)
{
    if (rows == 0 && !q) return xnor_layer_norm_fwd(x, x_type, rows, cols, x_stride, gamma, beta, p_type, eps, nullptr, q_stride, mean, rstd, stream);
    if (!q) return XNOR_E_NULL;
    return norm_forward(x, x_type, rows, cols, x_stride, gamma, beta, p_type, eps, {q, rows, cols, q_stride, 1, true}, q, scale, mean, rstd, stream);
}

int xnor_layer_norm_bwd_workspace_bytes(int x_type, long long rows, int cols, size_t *bytes)
{
    if (!bytes) return XNOR_E_NULL;
    if (!value_size(x_type)) return XNOR_E_UNSUPPORTED;
    if (rows < 0 || rows > kMaxRows || cols <= 0 || cols > kMaxCols) return XNOR_E_SHAPE;
    *bytes = layer_norm_bwd_workspace(x_type, rows, cols);
    return XNOR_OK;
}

int xnor_layer_norm_bwd(const void *dy, long long dy_stride, const void *x, int x_type, long long rows, int cols, long long x_stride,
                        const void *gamma, int p_type, const float *mean, const float *rstd, void *dx, long long dx_stride, void *dgamma,
                        void *dbeta, void *workspace, size_t workspace_bytes, void *stream)
{
    int xs, ps, rc = norm_types(x_type, p_type, &xs, &ps);
    if (rc) return rc;
    const Matrix all[] = {{dy, rows, cols, dy_stride, xs, false}, {x, rows, cols, x_stride, xs, false}, vec(mean, rows, 4), vec(rstd, rows, 4),
                          {dx, rows, cols, dx_stride, xs, true}};
    if ((rc = check(all))) return rc;
    if (!dgamma != !dbeta) return XNOR_E_NULL;
    if (!aligned(gamma, ps) || !aligned(dgamma, ps) || !aligned(dbeta, ps)) return XNOR_E_ALIGN;
    if (dgamma) {
        if (!workspace) return XNOR_E_NULL;
        if (!aligned(workspace, 16)) return XNOR_E_ALIGN;
        if (workspace_bytes < layer_norm_bwd_workspace(x_type, rows, cols)) return XNOR_E_WORKSPACE;
    }
    NormBackArgs a{};
    a.dy = dy, a.x = x, a.gamma = gamma, a.rows = rows, a.cols = cols;
    a.dy_stride = dy_stride, a.x_stride = x_stride, a.dx_stride = dx_stride;
    a.mean = mean, a.rstd = rstd, a.dx = dx, a.dgamma = dgamma, a.dbeta = dbeta, a.partial = dgamma ? (float *)workspace : nullptr;
    return hip_status(launch_layer_norm_bwd(a, x_type, p_type, (hipStream_t)stream));
}

int xnor_gated_fwd(const void *x, int type, long long x_stride, const void *wg, const void *wu, long long w_stride, int act, long long M, int F,
                   int K, void *h, long long h_stride, void *g, void *u, long long gu_stride, void *stream)
{
    return xnor_gated_fwd_ws(x, type, x_stride, wg, wu, w_stride, act, M, F, K, h, h_stride, g, u, gu_stride, nullptr, 0, stream);
}

int xnor_gated_fwd_workspace_bytes(long long M, int F, int K, long long x_stride, long long w_stride, size_t *bytes)
{
    if (!bytes) return XNOR_E_NULL;
    if (M < 0 || M > kMaxRows || F <= 0 || F > kMaxCols || K <= 0 || K > kMaxCols || x_stride < 0 || w_stride < 0) return XNOR_E_SHAPE;
    DenseArgs d{};
    d.lda = 2 * std::min(x_stride, kMaxStride), d.ldb = 2 * std::min(w_stride, kMaxStride), d.K = K;
    *bytes = !dense_direct_supports(d, XNOR_TYPE_F16) && gated_fwd_copy_pays(M, F, K) ? gated_fwd_workspace(M, F, K) : 0;
    return XNOR_OK;
}

int xnor_gated_fwd_ws(const void *x, int type, long long x_stride, const void *wg, const void *wu, long long w_stride, int act, long long M, int F,
                      int K, void *h, long long h_stride, void *g, void *u, long long gu_stride, void *workspace, size_t workspace_bytes, void *stream)
{
    if (value_size(type) != 2 || !known_act(act)) return XNOR_E_UNSUPPORTED;
    if (M > 0 && !g != !u) return XNOR_E_NULL;
    const long long kept = g ? M : 0;
    const Matrix all[] = {{x, M, K, x_stride, 2, false}, {wg, F, K, w_stride, 2, false}, {wu, F, K, w_stride, 2, false}, {h, M, F, h_stride, 2, true},
                          {g, kept, F, g ? gu_stride : F, 2, true}, {u, kept, F, g ? gu_stride : F, 2, true}};
    if (const int rc = check(all)) return rc;
    if (!aligned(workspace, 16)) return XNOR_E_ALIGN;
    DenseArgs d{};
    d.a = x, d.lda = 2 * x_stride, d.b = wg, d.b2 = wu, d.ldb = 2 * w_stride, d.act = act;
    d.M = M, d.N = F, d.K = K, d.out = h, d.ldo = h_stride, d.out2 = g, d.out3 = u, d.ldo2 = gu_stride;
    if (workspace && !dense_direct_supports(d, type) && gated_fwd_copy_pays(M, F, K) && workspace_bytes >= gated_fwd_workspace(M, F, K)) {
        const hipError_t e = gated_fwd_copy(&d, workspace, (hipStream_t)stream);
        if (e != hipSuccess) return hip_status(e);
    }
    return hip_status(launch_dense_gated(d, type, (hipStream_t)stream));
}

int xnor_gated_bwd_workspace_bytes(long long M, int F, int K, size_t *bytes)
{
    if (!bytes) return XNOR_E_NULL;
    if (M < 0 || M > kMaxRows || F <= 0 || F > kMaxGatedBack || K <= 0 || K > kMaxGatedBack) return XNOR_E_SHAPE;
    *bytes = gated_bwd_workspace(M, F, K);
    return XNOR_OK;
}

int xnor_gated_bwd(const void *dh, long long dh_stride, const void *x, int type, long long x_stride, const void *wg, const void *wu,
                   long long w_stride, const void *g, const void *u, long long gu_stride, int act, long long M, int F, int K, void *dx,
                   long long dx_stride, void *dwg, void *dwu, long long dw_stride, void *workspace, size_t workspace_bytes, void *stream)
{
    if (value_size(type) != 2 || !known_act(act)) return XNOR_E_UNSUPPORTED;
    const Matrix all[] = {{dh, M, F, dh_stride, 2, false}, {x, M, K, x_stride, 2, false}, {wg, F, K, w_stride, 2, false},
                          {wu, F, K, w_stride, 2, false}, {g, M, F, gu_stride, 2, false}, {u, M, F, gu_stride, 2, false},
                          {dx, M, K, dx_stride, 2, true}, {dwg, F, K, dw_stride, 2, true}, {dwu, F, K, dw_stride, 2, true}, vec(workspace, F, 16)};
    if (const int rc = check(all)) return rc;
    size_t need;
    if (const int rc = xnor_gated_bwd_workspace_bytes(M, F, K, &need)) return rc;
    if (workspace_bytes < need) return XNOR_E_WORKSPACE;
    GatedBackArgs a{};
    a.dh = dh, a.x = x, a.wg = wg, a.wu = wu, a.g = g, a.u = u;
    a.dh_stride = dh_stride, a.x_stride = x_stride, a.w_stride = w_stride, a.gu_stride = gu_stride;
    a.dx_stride = dx_stride, a.dw_stride = dw_stride, a.act = act, a.M = M, a.F = F, a.K = K;
    a.dx = dx, a.dwg = dwg, a.dwu = dwu, a.workspace = workspace;
    return hip_status(launch_gated_bwd(a, type, (hipStream_t)stream));
}

int xnor_int8_gated(const int8_t *a, long long a_stride, const float *a_scale, const int8_t *wg, const float *wg_scale, const int8_t *wu,
                    const float *wu_scale, long long w_stride, int act, long long M, int F, int K, void *h, int h_type, long long h_stride,
                    void *stream)
{
    const int hs = value_size(h_type);
    if (!hs || !known_act(act)) return XNOR_E_UNSUPPORTED;
    const Matrix all[] = {{a, M, K, a_stride, 1, false}, vec(a_scale, M, 4), {wg, F, K, w_stride, 1, false}, vec(wg_scale, F, 4),
                          {wu, F, K, w_stride, 1, false}, vec(wu_scale, F, 4), {h, M, F, h_stride, hs, true}};
    if (const int rc = check(all)) return rc;
    if (K > kMaxInt8Cols) return XNOR_E_SHAPE;
    DenseArgs d{};
    d.a = a, d.lda = a_stride, d.a_scale = a_scale, d.b = wg, d.b2 = wu, d.ldb = w_stride, d.b_scale = wg_scale, d.b2_scale = wu_scale, d.act = act;
    d.M = M, d.N = F, d.K = K, d.out = h, d.ldo = h_stride;
    return hip_status(launch_dense_int8_gated(d, h_type, (hipStream_t)stream));
}

}  // extern "C"
