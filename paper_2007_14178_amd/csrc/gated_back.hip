// Backward pass of the gated block h = act(g) u, g = x wg^T, u = x wu^T:
//   dg = dh u act'(g)   du = dh act(g)   dx = dg wg + du wu   dwg = dg^T x   dwu = du^T x
// The products run on the kernel that takes rows along the contraction, so this file lays the operands out so: [dg du] by token
// and transposed, x and [wg wu] transposed.  dg and du are rounded to the block's type, which the matrix instructions
// take; everything else is summed in fp32 and rounded once.
#include <algorithm>

#include "dense_common.hpp"

namespace xnor {
namespace {

constexpr int kTile = 64;

size_t pad(long long n) { return (size_t)((n + 7) / 8 * 8); }

// A 64 x 64 tile of 16-bit values, written by rows and read by columns.  (A row is 66 values: columns spread over the banks.)
template <class T>
struct Tile {
    T v[kTile][kTile + 2];
};

// dst[c][r] = tile[r][c] for the tile at (r0, c0) of a matrix of `rows` rows; c below `cols`.
template <class T>
__device__ inline void store_transposed(const Tile<T> &tile, T *dst, long long ld, long long r0, long long rows, int c0, int cols)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = (threadIdx.x >> 3) + 32 * i, r = (threadIdx.x & 7) * 8;
        if (c0 + c >= cols || r0 + r >= rows) continue;
        T out[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) out[k] = tile.v[r + k][c];
        T *to = dst + (c0 + c) * ld + r0 + r;
        const int n = (int)min(rows - (r0 + r), 8LL);
        store_values(to, 0, n, out);
    }
}

// dst[c][r] = src[r][c].  `dst_rows` >= cols: rows behind the matrix are zeros.
template <class T>
__global__ __launch_bounds__(256) void transpose_kernel(const T *src, long long ld_src, long long rows, int cols, T *dst, long long ld_dst, int tiles_c)
{
    __shared__ Tile<T> tile;
    const int c0 = (int)(blockIdx.x % (unsigned)tiles_c) * kTile;
    const long long r0 = (long long)(blockIdx.x / (unsigned)tiles_c) * kTile;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = (threadIdx.x >> 3) + 32 * i, c = (threadIdx.x & 7) * 8;
        Chunk<T> v{};
        if (r0 + r < rows && c0 + c < cols) v = load_chunk(src + (r0 + r) * ld_src + c0, c, cols - c0);
#pragma unroll
        for (int k = 0; k < 8; ++k) tile.v[r][c + k] = v.v[k];
    }
    __syncthreads();
    store_transposed(tile, dst, ld_dst, r0, rows, c0, cols);
}

// [dg du] by token (row stride 2 fp, zeros behind F in each half) and transposed (rows f and fp + f).
template <class T, int ACT>
__global__ __launch_bounds__(256) void gate_back_kernel(const GatedBackArgs p, T *dgu, T *dgu_t, int fp, long long mp, int tiles_f)
{
    __shared__ Tile<T> tg, tu;
    const int f0 = (int)(blockIdx.x % (unsigned)tiles_f) * kTile;
    const long long m0 = (long long)(blockIdx.x / (unsigned)tiles_f) * kTile;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = (threadIdx.x >> 3) + 32 * i, c = (threadIdx.x & 7) * 8;
        const long long m = m0 + r;
        T dg[8] = {}, du[8] = {};
        if (m < p.M && f0 + c < p.F) {
            const Chunk<T> dh = load_chunk((const T *)p.dh + m * p.dh_stride + f0, c, p.F - f0);
            const Chunk<T> g = load_chunk((const T *)p.g + m * p.gu_stride + f0, c, p.F - f0);
            const Chunk<T> u = load_chunk((const T *)p.u + m * p.gu_stride + f0, c, p.F - f0);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (f0 + c + k >= p.F) break;
                const float d = (float)dh.v[k], gv = (float)g.v[k];
                dg[k] = (T)(d * (float)u.v[k] * act_slope<ACT>(gv));
                du[k] = (T)(d * act_value<ACT>(gv));
            }
        }
        if (m < p.M && f0 + c < fp) {
            __builtin_memcpy(dgu + m * 2 * fp + f0 + c, dg, 16);
            __builtin_memcpy(dgu + m * 2 * fp + fp + f0 + c, du, 16);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            tg.v[r][c + k] = dg[k];
            tu.v[r][c + k] = du[k];
        }
    }
    __syncthreads();
    store_transposed(tg, dgu_t, mp, m0, p.M, f0, fp);
    store_transposed(tu, dgu_t + (long long)fp * mp, mp, m0, p.M, f0, fp);
}

// Zeros in columns F .. fp of both halves of w^T's K rows.
template <class T>
__global__ __launch_bounds__(256) void clear_pads_kernel(T *wt, int K, int F, int fp)
{
    const int i = blockIdx.x * 256 + threadIdx.x, n = fp - F;
    if (i >= K * 2 * n) return;
    const int k = i / (2 * n), j = i % (2 * n);
    wt[(long long)k * 2 * fp + (j / n) * fp + F + j % n] = T(0);
}

template <class T>
hipError_t transpose(const T *src, long long ld_src, long long rows, int cols, T *dst, long long ld_dst, hipStream_t st)
{
    const int tiles_c = ceil_div(cols, kTile);
    const long long most = std::max<long long>(1, kMaxBlocks / tiles_c) * kTile;
    for (long long r = 0; r < rows; r += most) {
        const long long n = std::min(most, rows - r);
        transpose_kernel<T><<<dim3((unsigned)(tiles_c * ((n + kTile - 1) / kTile))), dim3(256), 0, st>>>(src + r * ld_src, ld_src, n, cols, dst + r, ld_dst, tiles_c);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

struct Layout {
    size_t fp, mp, dgu, dgu_t, xt, wt, bytes;
};
Layout layout(long long M, int F, int K)
{
    Layout l;
    l.fp = pad(F), l.mp = pad(M);
    size_t at = 0;
    auto take = [&](size_t values) { const size_t here = at; at += (values * 2 + 255) / 256 * 256; return here; };
    l.dgu = take((size_t)M * 2 * l.fp);
    l.dgu_t = take(2 * l.fp * l.mp);
    l.xt = take((size_t)K * l.mp);
    l.wt = take((size_t)K * 2 * l.fp);
    l.bytes = at;
    return l;
}

template <class T>
hipError_t run(const GatedBackArgs &p, int type, hipStream_t st)
{
    const Layout l = layout(p.M, p.F, p.K);
    char *ws = (char *)p.workspace;
    T *dgu = (T *)(ws + l.dgu), *dgu_t = (T *)(ws + l.dgu_t), *xt = (T *)(ws + l.xt), *wt = (T *)(ws + l.wt);
    const int fp = (int)l.fp;
    hipError_t e;
    const int tiles_f = ceil_div(fp, kTile);
    const long long most = std::max<long long>(1, kMaxBlocks / tiles_f) * kTile;
    for (long long m = 0; m < p.M; m += most) {
        GatedBackArgs q = p;
        q.M = std::min(most, p.M - m);
        q.dh = (const T *)p.dh + m * p.dh_stride;
        q.g = (const T *)p.g + m * p.gu_stride;
        q.u = (const T *)p.u + m * p.gu_stride;
        const dim3 grid((unsigned)(tiles_f * ((q.M + kTile - 1) / kTile)));
        T *by_token = dgu + m * 2 * fp, *by_unit = dgu_t + m;
        if (p.act == XNOR_ACT_SILU) gate_back_kernel<T, XNOR_ACT_SILU><<<grid, dim3(256), 0, st>>>(q, by_token, by_unit, fp, (long long)l.mp, tiles_f);
        else if (p.act == XNOR_ACT_GELU) gate_back_kernel<T, XNOR_ACT_GELU><<<grid, dim3(256), 0, st>>>(q, by_token, by_unit, fp, (long long)l.mp, tiles_f);
        else gate_back_kernel<T, XNOR_ACT_RELU><<<grid, dim3(256), 0, st>>>(q, by_token, by_unit, fp, (long long)l.mp, tiles_f);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (p.M > 0) {
        if ((e = transpose((const T *)p.x, p.x_stride, p.M, p.K, xt, (long long)l.mp, st)) != hipSuccess) return e;
        if ((e = transpose((const T *)p.wg, p.w_stride, p.F, p.K, wt, 2LL * fp, st)) != hipSuccess) return e;
        if ((e = transpose((const T *)p.wu, p.w_stride, p.F, p.K, wt + fp, 2LL * fp, st)) != hipSuccess) return e;
        if (fp > p.F) {
            clear_pads_kernel<T><<<dim3(ceil_div((long long)p.K * 2 * (fp - p.F), 256)), dim3(256), 0, st>>>(wt, p.K, p.F, fp);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
        DenseArgs d{};
        d.a = dgu, d.lda = 4LL * fp, d.b = wt, d.ldb = 4LL * fp;
        d.M = p.M, d.N = p.K, d.K = 2 * fp;
        d.out = p.dx, d.ldo = p.dx_stride, d.split = d.valid = p.M;
        if ((e = launch_dense(d, type, st)) != hipSuccess) return e;
    }
    DenseArgs d{};
    d.a = dgu_t, d.lda = 2LL * l.mp, d.b = xt, d.ldb = 2LL * l.mp;
    d.M = 2LL * fp, d.N = p.K, d.K = (int)p.M;
    d.out = p.dwg, d.out2 = p.dwu, d.ldo = p.dw_stride, d.split = fp, d.valid = p.F;
    return launch_dense(d, type, st);
}

}  // namespace

size_t gated_bwd_workspace(long long M, int F, int K) { return layout(M, F, K).bytes; }

hipError_t launch_gated_bwd(const GatedBackArgs &p, int type, hipStream_t st)
{
    return type == XNOR_TYPE_F16 ? run<f16_t>(p, type, st) : run<bf16_t>(p, type, st);
}

}  // namespace xnor
