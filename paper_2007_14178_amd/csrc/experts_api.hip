// Host side of routing and of the products with 4-bit weights in the C ABI: argument validation, then the launchers.
#include <algorithm>

#include "dense_check.hpp"
#include "experts_common.hpp"

namespace {

using namespace xnor;

bool known_group(int g) { return g == 32 || g == 64 || g == 128; }
int row_bytes(int cols) { return (int)(((long long)cols + 7) / 8 * 4); }

// Status of a matrix of 4-bit weights or of a stack of `count`.
int check_int4(const xnor_int4 *w, int count)
{
    if (!w) return XNOR_E_NULL;
    if (!value_size(w->scale_type) || !known_group(w->group)) return XNOR_E_UNSUPPORTED;
    if (w->rows <= 0 || w->rows > kMaxCols || w->cols <= 0 || w->cols > kMaxCols) return XNOR_E_SHAPE;
    if (!w->q || !w->scale) return XNOR_E_NULL;
    if (w->q_stride < row_bytes(w->cols) || !stride_fits((long long)w->rows * count, w->q_stride)) return XNOR_E_SHAPE;
    if (!aligned(w->q, 4) || w->q_stride % 4 || !aligned(w->scale, value_size(w->scale_type))) return XNOR_E_ALIGN;
    return XNOR_OK;
}

// The gated block's two matrices.
int check_pair(const xnor_int4 *wg, const xnor_int4 *wu, int count)
{
    int rc = check_int4(wg, count);
    if (rc || (rc = check_int4(wu, count))) return rc;
    if (wg->rows != wu->rows || wg->cols != wu->cols || wg->group != wu->group || wg->q_stride != wu->q_stride) return XNOR_E_SHAPE;
    return wg->scale_type != wu->scale_type || !wg->zero != !wu->zero ? XNOR_E_UNSUPPORTED : XNOR_OK;
}

Int4Args args_of(const void *x, long long ldx, const xnor_int4 *w, const xnor_int4 *w2, long long M, void *out, int out_type, long long ldo)
{
    Int4Args a{};
    a.x = x, a.ldx = ldx, a.w = {w->q, w->scale, w->zero}, a.ldq = w->q_stride, a.scale_type = w->scale_type, a.group = w->group;
    if (w2) a.w2 = {w2->q, w2->scale, w2->zero};
    a.parts = 1, a.M = M, a.N = w->rows, a.K = w->cols, a.out = out, a.out_type = out_type, a.ldo = ldo;
    return a;
}

int product_workspace(long long M, int N, int K, bool gated, size_t *bytes)
{
    if (M < 0 || M > kMaxRows || N <= 0 || N > kMaxCols || K <= 0 || K > kMaxCols) return XNOR_E_SHAPE;
    const int parts = int4_tile_parts(M, N, K, gated);
    *bytes = parts > 1 ? (size_t)parts * (gated ? 2 : 1) * M * N * sizeof(float) : 0;
    return XNOR_OK;
}
// Shares of the contraction, given the workspace for them.
void take_workspace(Int4Args *a, bool gated, void *workspace, size_t bytes)
{
    const int parts = int4_tile_parts(a->M, a->N, a->K, gated);
    if (parts > 1 && workspace && bytes >= (size_t)parts * (gated ? 2 : 1) * a->M * a->N * sizeof(float)) a->parts = parts, a->sums = (float *)workspace;
}

// Sizes of a call of xnor_int4_experts, and its workspace's parts, each at a multiple of 256 bytes.
int check_experts(long long T, int k, int E)
{
    if (T < 0 || T > kMaxRows || k <= 0 || k > kMaxChosen || E <= 0 || E > kMaxExperts || T * k > kMaxRows) return XNOR_E_SHAPE;
    return XNOR_OK;
}
// Tokens whose pairs the workspace is for: longer calls take one run after the other, so that it does not grow with them.  (A run of 2^18 pairs reads each of 256
// experts' weights for 1024 of them.)
long long most_tokens(int k) { return std::max(1LL, (1LL << 18) / k); }

struct ExpertParts {
    size_t offsets, order, lists, tiles, hidden, pairs, bytes;
    int tile;
};
ExpertParts expert_parts(long long T, int k, int E, int F, int N)
{
    const long long pairs = T * k;
    ExpertParts to{};
    size_t at = 0;
    auto part = [&](size_t bytes) {
        const size_t from = at;
        at += (bytes + 255) / 256 * 256;
        return from;
    };
    to.offsets = part((size_t)(E + 1) * 4);
    to.order = part((size_t)pairs * 4);
    to.lists = part(route_lists_workspace(pairs, E));
    to.tile = int4_expert_tile(pairs, E);
    to.tiles = part((size_t)(1 + most_tiles(pairs, E, std::min(to.tile, kInt4Few))) * sizeof(ExpertTile));
    to.hidden = part((size_t)pairs * hidden_stride(F) * kMostTerms * 2);
    to.pairs = part((size_t)pairs * N * 4);
    to.bytes = at;
    return to;
}

int check_route(long long T, int E, int k)
{
    if (T < 0 || T > kMaxRows || E <= 0 || E > kMaxExperts || k <= 0 || k > kMaxChosen || T * k > kMaxRows) return XNOR_E_SHAPE;
    return XNOR_OK;
}

}  // namespace

extern "C" {

int xnor_int4_quantize(const void *w, int w_type, long long rows, int cols, long long w_stride, int group, uint8_t *q, long long q_stride,
                       void *scale, int scale_type, uint8_t *zero, void *stream)
{
    const int ws = value_size(w_type), ss = value_size(scale_type);
    if (!ws || !ss || !known_group(group)) return XNOR_E_UNSUPPORTED;
    const Matrix all[] = {{w, rows, cols, w_stride, ws, false}, {q, rows, cols, std::max<long long>(q_stride, cols), 4, false}, vec(scale, rows, ss)};
    if (const int rc = check(all)) return rc;
    if (q_stride < row_bytes(cols) || !stride_fits(rows, q_stride)) return XNOR_E_SHAPE;
    if (q_stride % 4) return XNOR_E_ALIGN;
    Int4Make a{};
    a.from = w, a.rows = rows, a.cols = cols, a.stride = w_stride, a.group = group, a.q = q, a.q_stride = q_stride, a.scale = scale, a.zero = zero;
    a.scale_type = scale_type;
    return hip_status(launch_int4_quantize(a, w_type, (hipStream_t)stream));
}

int xnor_int4_pack(const uint8_t *levels, long long rows, int cols, long long levels_stride, uint8_t *q, long long q_stride, void *stream)
{
    const Matrix all[] = {{levels, rows, cols, levels_stride, 1, false}, {q, rows, cols, std::max<long long>(q_stride, cols), 4, false}};
    if (const int rc = check(all)) return rc;
    if (q_stride < row_bytes(cols) || !stride_fits(rows, q_stride)) return XNOR_E_SHAPE;
    if (q_stride % 4) return XNOR_E_ALIGN;
    Int4Make a{};
    a.from = levels, a.rows = rows, a.cols = cols, a.stride = levels_stride, a.q = q, a.q_stride = q_stride;
    return hip_status(launch_int4_pack(a, (hipStream_t)stream));
}

int xnor_int4_dequantize(const xnor_int4 *w, void *out, int out_type, long long out_stride, void *stream)
{
    if (const int rc = check_int4(w, 1)) return rc;
    const int os = value_size(out_type);
    if (!os) return XNOR_E_UNSUPPORTED;
    const Matrix all[] = {{out, w->rows, w->cols, out_stride, os, true}};
    if (const int rc = check(all)) return rc;
    Int4Make a{};
    a.rows = w->rows, a.cols = w->cols, a.group = w->group, a.q = const_cast<uint8_t *>(w->q), a.q_stride = w->q_stride;
    a.scale = const_cast<void *>(w->scale), a.zero = const_cast<uint8_t *>(w->zero), a.scale_type = w->scale_type;
    a.out = out, a.out_type = out_type, a.stride = out_stride;
    return hip_status(launch_int4_dequantize(a, (hipStream_t)stream));
}

int xnor_int4_linear_workspace_bytes(long long M, int N, int K, size_t *bytes)
{
    if (!bytes) return XNOR_E_NULL;
    return product_workspace(M, N, K, false, bytes);
}

int xnor_int4_linear(const void *x, int type, long long x_stride, const xnor_int4 *w, const float *bias, long long M, void *out, int out_type,
                     long long out_stride, void *workspace, size_t workspace_bytes, void *stream)
{
    const int os = value_size(out_type);
    if (value_size(type) != 2 || !os) return XNOR_E_UNSUPPORTED;
    if (const int rc = check_int4(w, 1)) return rc;
    const Matrix all[] = {{x, M, w->cols, x_stride, 2, false}, {out, M, w->rows, out_stride, os, true}};
    if (const int rc = check(all)) return rc;
    if (!aligned(bias, 4) || !aligned(workspace, 16)) return XNOR_E_ALIGN;
    Int4Args a = args_of(x, 2 * x_stride, w, nullptr, M, out, out_type, out_stride);
    a.bias = bias;
    take_workspace(&a, false, workspace, workspace_bytes);
    return hip_status(launch_int4(a, type, false, (hipStream_t)stream));
}

int xnor_int4_gated_workspace_bytes(long long M, int F, int K, size_t *bytes)
{
    if (!bytes) return XNOR_E_NULL;
    return product_workspace(M, F, K, true, bytes);
}

int xnor_int4_gated(const void *x, int type, long long x_stride, const xnor_int4 *wg, const xnor_int4 *wu, int act, long long M, void *h, int h_type,
                    long long h_stride, void *workspace, size_t workspace_bytes, void *stream)
{
    const int hs = value_size(h_type);
    if (value_size(type) != 2 || !hs || !known_act(act)) return XNOR_E_UNSUPPORTED;
    if (const int rc = check_pair(wg, wu, 1)) return rc;
    const Matrix all[] = {{x, M, wg->cols, x_stride, 2, false}, {h, M, wg->rows, h_stride, hs, true}};
    if (const int rc = check(all)) return rc;
    if (!aligned(workspace, 16)) return XNOR_E_ALIGN;
    Int4Args a = args_of(x, 2 * x_stride, wg, wu, M, h, h_type, h_stride);
    a.act = act;
    take_workspace(&a, true, workspace, workspace_bytes);
    return hip_status(launch_int4(a, type, true, (hipStream_t)stream));
}

int xnor_route_fwd(const void *logits, int type, long long T, int E, long long logits_stride, const float *bias, int score, int groups,
                   int groups_kept, int group_top, int k, int renorm, float factor, int32_t *experts, float *weights, void *stream)
{
    const int size = value_size(type);
    if (!size || (score != XNOR_SCORE_SOFTMAX && score != XNOR_SCORE_SIGMOID)) return XNOR_E_UNSUPPORTED;
    if (const int rc = check_route(T, E, k)) return rc;
    if (groups < 1 || groups > E || E % groups || groups_kept < 1 || groups_kept > groups || group_top < 1 || group_top > 2) return XNOR_E_SHAPE;
    if (k > E / groups * groups_kept) return XNOR_E_SHAPE;
    const Matrix all[] = {{logits, T, E, logits_stride, size, false}, {experts, T, k, k, 4, true}, {weights, T, k, k, 4, true}};
    if (const int rc = check(all)) return rc;
    if (!aligned(bias, 4)) return XNOR_E_ALIGN;
    RouteArgs a{};
    a.logits = logits, a.T = T, a.stride = logits_stride, a.E = E, a.bias = bias, a.score = score, a.groups = groups, a.kept = groups_kept;
    a.top = group_top, a.k = k, a.renorm = renorm != 0, a.factor = factor, a.experts = experts, a.weights = weights;
    return hip_status(launch_route(a, type, (hipStream_t)stream));
}

int xnor_route_lists_workspace_bytes(long long T, int k, int E, size_t *bytes)
{
    if (!bytes) return XNOR_E_NULL;
    if (const int rc = check_route(T, E, k)) return rc;
    *bytes = route_lists_workspace(T * k, E);
    return XNOR_OK;
}

int xnor_route_lists(const int32_t *experts, long long T, int k, int E, int32_t *offsets, int32_t *order, void *workspace, size_t workspace_bytes,
                     void *stream)
{
    if (const int rc = check_route(T, E, k)) return rc;
    const size_t need = route_lists_workspace(T * k, E);
    const Matrix all[] = {{experts, T, k, k, 4, false}, vec(offsets, E + 1, 4), {order, T, k, k, 4, true}, vec(workspace, need ? 1 : 0, 16)};
    if (const int rc = check(all)) return rc;
    if (workspace_bytes < need) return XNOR_E_WORKSPACE;
    ListArgs a{};
    a.experts = experts, a.pairs = T * k, a.E = E, a.offsets = offsets, a.order = order, a.counts = (int32_t *)workspace;
    return hip_status(launch_route_lists(a, (hipStream_t)stream));
}

int xnor_route_bwd(const float *dweights, const void *logits, int type, long long T, int E, long long logits_stride, const int32_t *experts, int k,
                   int score, int renorm, float factor, void *dlogits, long long dlogits_stride, void *stream)
{
    const int size = value_size(type);
    if (!size || (score != XNOR_SCORE_SOFTMAX && score != XNOR_SCORE_SIGMOID)) return XNOR_E_UNSUPPORTED;
    if (const int rc = check_route(T, E, k)) return rc;
    const Matrix all[] = {{dweights, T, k, k, 4, false}, {logits, T, E, logits_stride, size, false}, {experts, T, k, k, 4, false},
                          {dlogits, T, E, dlogits_stride, size, true}};
    if (const int rc = check(all)) return rc;
    RouteArgs a{};
    a.logits = logits, a.T = T, a.stride = logits_stride, a.E = E, a.score = score, a.k = k, a.renorm = renorm != 0, a.factor = factor;
    a.experts = const_cast<int32_t *>(experts), a.dweights = dweights, a.dlogits = dlogits, a.dstride = dlogits_stride;
    return T > 0 ? hip_status(launch_route_bwd(a, type, (hipStream_t)stream)) : XNOR_OK;
}

int xnor_int4_experts_workspace_bytes(long long T, int k, int E, int K, int F, int N, size_t *bytes)
{
    if (!bytes) return XNOR_E_NULL;
    if (const int rc = check_experts(T, k, E)) return rc;
    if (K <= 0 || K > kMaxCols || F <= 0 || F > kMaxCols || N <= 0 || N > kMaxCols) return XNOR_E_SHAPE;
    *bytes = T > 0 ? expert_parts(std::min(T, most_tokens(k)), k, E, F, N).bytes : 0;
    return XNOR_OK;
}

int xnor_int4_experts(const void *x, int type, long long x_stride, long long T, const int32_t *experts, const float *weights, int k, int E,
                      const xnor_int4 *wg, const xnor_int4 *wu, const xnor_int4 *wd, int act, void *out, int out_type, long long out_stride,
                      void *workspace, size_t workspace_bytes, void *stream)
{
    const int os = value_size(out_type);
    if (value_size(type) != 2 || !os || !known_act(act)) return XNOR_E_UNSUPPORTED;
    if (const int rc = check_experts(T, k, E)) return rc;
    int rc = check_pair(wg, wu, E);
    if (rc || (rc = check_int4(wd, E))) return rc;
    const int K = wg->cols, F = wg->rows, N = wd->rows;
    if (wd->cols != F) return XNOR_E_SHAPE;
    const Matrix all[] = {{x, T, K, x_stride, 2, false}, {experts, T, k, k, 4, false}, {weights, T, k, k, 4, false}, {out, T, N, out_stride, os, true},
                          vec(workspace, T > 0 ? 1 : 0, 16)};
    if ((rc = check(all))) return rc;
    if (T == 0) return XNOR_OK;
    ExpertParts at = expert_parts(std::min(T, most_tokens(k)), k, E, F, N);
    if (workspace_bytes < at.bytes) return XNOR_E_WORKSPACE;
    char *const held = (char *)workspace;
    const hipStream_t st = (hipStream_t)stream;
    // hidden rows: of bf16 terms
    const int terms = hidden_terms(out_type);
    const long long ldh = (long long)terms * hidden_stride(F);

    if (int4_pairs_pay(T * k, E)) {
        // hidden: rows by pair
        Int4Args a = args_of(x, 2 * x_stride, wg, wu, T * k, held + at.hidden, out_type, ldh);
        a.act = act, a.pairs = experts, a.E = E, a.chosen = k, a.out_terms = terms;
        const hipError_t e = launch_int4(a, type, true, st);
        if (e != hipSuccess) return hip_status(e);
        Int4Args b = args_of(held + at.hidden, 2 * ldh, wd, nullptr, T, out, out_type, out_stride);
        b.pairs = experts, b.E = E, b.chosen = k, b.terms = terms;
        return hip_status(launch_int4_down(b, weights, st));
    }
    // Tokens in runs: of what the workspace is for, and of what tiles reach with 31 bits from a run's first token.  (Tokens so far apart that a run would be short are
    // left to the kernel for few, which reaches all of them.)
    const long long ldx = 2 * x_stride, reach = ldx > 0 ? std::max(0LL, kTileReach - 2LL * K) / ldx : T;
    long long run = std::min(T, most_tokens(k));
    if (reach >= std::min<long long>(T, 1024)) run = std::min(run, reach);
    for (long long from = 0; from < T; from += run) {
        const long long n = std::min(run, T - from);
        ListArgs l{};
        l.experts = experts + from * k, l.pairs = n * k, l.E = E, l.offsets = (int32_t *)(held + at.offsets), l.order = (int32_t *)(held + at.order);
        l.counts = (int32_t *)(held + at.lists), l.tiles = (ExpertTile *)(held + at.tiles);
        // hidden: rows by sorted position; pairs: rows by token and slot
        Int4Args a = args_of((const char *)x + from * ldx, ldx, wg, wu, n * k, held + at.hidden, out_type, ldh);
        a.act = act, a.tiles = l.tiles, a.order_x = l.order, a.E = E, a.chosen = k, a.out_terms = terms;
        Int4Args b = args_of(held + at.hidden, 2 * ldh, wd, nullptr, n * k, held + at.pairs, XNOR_TYPE_FP32, N);
        b.tiles = l.tiles, b.order_out = l.order, b.E = E, b.chosen = k, b.terms = terms;
        if (!int4_tiles_support(a) || !int4_tiles_support(b)) at.tile = std::min(at.tile, kInt4Few);
        l.tile = a.tile = b.tile = at.tile;
        hipError_t e = launch_route_lists(l, st);
        if (e == hipSuccess) e = launch_int4(a, type, true, st);
        if (e == hipSuccess) e = launch_int4(b, XNOR_TYPE_BF16, false, st);
        if (e != hipSuccess) return hip_status(e);
        CombineArgs c{};
        c.pairs = (const float *)(held + at.pairs), c.experts = l.experts, c.weights = weights + from * k, c.T = n, c.ldo = out_stride, c.k = k, c.E = E, c.N = N;
        c.out = (char *)out + from * out_stride * os, c.out_type = out_type;
        e = launch_combine(c, st);
        if (e != hipSuccess) return hip_status(e);
    }
    return XNOR_OK;
}

}  // extern "C"
