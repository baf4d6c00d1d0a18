// Around the gated block's products: rows copied to 16-byte boundaries where the products would read them slowly, and the backward
// pass of h = act(g) u, g = x wg^T, u = x wu^T:
//   dg = dh u act'(g)   du = dh act(g)   dx = dg wg + du wu   dwg = dg^T x   dwu = du^T x
// One pass forms [dg du] by token; the two products read it and the block's own operands as they lie, across their rows where the
// contraction goes across.  dg and du are rounded to the block's type, which the matrix instructions take; everything
// else is summed in fp32 and rounded once.  The products are nearly all of it (bf16, 8192 x 4096 x 8192: forming dg and du 136-150 us, 4.5-4.9
// TB/s, and the products 753-882 and 832-927 us, 1.1 TFLOP each); below a few hundred tokens it is the number of launches.
#include <algorithm>

#include "dense_common.hpp"

namespace xnor {
namespace {

size_t pad(long long n, int to) { return (size_t)((n + to - 1) / to * to); }

struct Copy {
    const uint16_t *from;
    uint16_t *to;
    long long rows, stride;
};

// i / n for i < total
__device__ inline long long row_of(long long i, int n, long long total) { return total >> 32 ? i / n : (long long)((uint32_t)i / (uint32_t)n); }

// Up to three matrices of `cols` 16-bit values a row to rows of `stride` values, whole cache lines; what is behind a row's end is zero.
__global__ __launch_bounds__(256) void copy_rows_kernel(const Copy a, const Copy b, const Copy c, int cols, int stride)
{
    const Copy &m = blockIdx.y == 0 ? a : blockIdx.y == 1 ? b : c;
    const int chunks = stride / 8;
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < m.rows * chunks; i += gridDim.x * 256LL) {
        const long long row = row_of(i, chunks, m.rows * chunks);
        const int at = (int)(i - row * chunks) * 8;
        const Chunk<uint16_t> v = load_chunk(m.from + row * m.stride, at, cols);
        __builtin_memcpy(m.to + row * stride + at, &v, 16);
    }
}

hipError_t copy_rows(const Copy (&m)[3], int count, int cols, int stride, hipStream_t st)
{
    long long most = 0;
    for (int i = 0; i < count; ++i) most = std::max(most, m[i].rows * (stride / 8));
    if (most == 0) return hipSuccess;
    const long long blocks = std::min<long long>((most + 255) / 256, 8 * compute_units());
    copy_rows_kernel<<<dim3((unsigned)blocks, (unsigned)count), dim3(256), 0, st>>>(m[0], m[1], m[2], cols, stride);
    return hipGetLastError();
}

// [dg du] by token: rows of 2 fp values, zeros behind F in each half.
template <class T, int ACT>
__global__ __launch_bounds__(256) void gate_back_kernel(const GatedBackArgs p, T *dgu, int fp)
{
    const int chunks = fp / 8;
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < p.M * chunks; i += gridDim.x * 256LL) {
        const long long m = row_of(i, chunks, p.M * chunks);
        const int f = (int)(i - m * chunks) * 8;
        T dg[8] = {}, du[8] = {};
        if (f < p.F) {
            const Chunk<T> dh = load_chunk((const T *)p.dh + m * p.dh_stride, f, p.F);
            const Chunk<T> g = load_chunk((const T *)p.g + m * p.gu_stride, f, p.F);
            const Chunk<T> u = load_chunk((const T *)p.u + m * p.gu_stride, f, p.F);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (f + k >= p.F) break;
                const float d = (float)dh.v[k], gv = (float)g.v[k];
                dg[k] = (T)(d * (float)u.v[k] * act_slope<ACT>(gv));
                du[k] = (T)(d * act_value<ACT, true>(gv));
            }
        }
        __builtin_memcpy(dgu + m * 2 * fp + f, dg, 16);
        __builtin_memcpy(dgu + m * 2 * fp + fp + f, du, 16);
    }
}

// Shares of the contraction of dx, whose sums are added by another launch: where its tiles of 128 x 128 would leave most of the chip idle,
// as many as make two workgroups a unit, of four steps of 64 values at least.  (6 tokens x 1152 x 3200 57 us without, 30 us so; 128 x 4096 x 8192 222 and 122.)
int dx_parts(long long M, int fp, int n)
{
    const long long tiles = (M + 127) / 128 * ceil_div(n, 128);
    const int parts = (int)std::min<long long>(2 * kPlanUnits / std::max(tiles, 1LL), 2 * fp / 64 / 4);
    return parts >= 3 ? parts : 1;
}

// out[m][n] = the sum over parts of sums[part][m][n], four values a thread.
template <class T>
__global__ __launch_bounds__(256) void add_parts_kernel(const float *sums, int parts, long long M, int n, T *out, long long ldo, int out_cols)
{
    const long long total = M * (n / 4);
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < total; i += gridDim.x * 256LL) {
        const long long m = row_of(i, n / 4, total);
        const int at = (int)(i - m * (n / 4)) * 4;
        float v[4] = {};
        for (int part = 0; part < parts; ++part) {
            float4 w;
            __builtin_memcpy(&w, sums + (part * M + m) * n + at, 16);
            v[0] += w.x, v[1] += w.y, v[2] += w.z, v[3] += w.w;
        }
        T to[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) to[k] = (T)v[k];
        store_values(out + m * ldo, at, out_cols, to);
    }
}

// The workspace: copies of x and the weights for rows that do not lie as the products want them, and [dg du].
struct Layout {
    size_t fp, kp, x, wg, wu, dgu, sums, bytes;
};
Layout layout(long long M, int F, int K, bool backward)
{
    Layout l;
    l.fp = pad(F, 64), l.kp = pad(K, 64);          // (rows of whole cache lines)
    size_t at = 0;
    auto take = [&](size_t values) { const size_t here = at; at += (values * 2 + 255) / 256 * 256; return here; };
    l.x = take((size_t)M * l.kp);
    l.wg = take((size_t)F * l.kp);
    l.wu = take((size_t)F * l.kp);
    l.dgu = take(backward ? (size_t)M * 2 * l.fp : 0);
    const int parts = backward ? dx_parts(M, (int)l.fp, (int)l.kp) : 1;        // (of the copies' width: the products' own needs no more)
    l.sums = take(parts > 1 ? 2 * (size_t)parts * M * l.kp : 0);
    l.bytes = at;
    return l;
}

// Rows as launch_dense_across takes them.
bool lies_well(const void *p, long long stride, int K)
{
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && stride % 8 == 0 && K % 8 == 0 && stride >= K && stride < (1 << 23);
}

template <class T>
hipError_t run(GatedBackArgs p, int type, hipStream_t st)
{
    const Layout l = layout(p.M, p.F, p.K, true);
    char *ws = (char *)p.workspace;
    T *dgu = (T *)(ws + l.dgu);
    const int fp = (int)l.fp;
    int n = p.K;            // columns of the products: K, or K and the zeros behind it in the copies
    hipError_t e;
    if (!lies_well(p.x, p.x_stride, p.K) || !lies_well(p.wg, p.w_stride, p.K) || !lies_well(p.wu, p.w_stride, p.K)) {
        const Copy copies[3] = {{(const uint16_t *)p.x, (uint16_t *)(ws + l.x), p.M, p.x_stride}, {(const uint16_t *)p.wg, (uint16_t *)(ws + l.wg), p.F, p.w_stride},
                                {(const uint16_t *)p.wu, (uint16_t *)(ws + l.wu), p.F, p.w_stride}};
        if ((e = copy_rows(copies, 3, p.K, (int)l.kp, st)) != hipSuccess) return e;
        p.x = ws + l.x, p.wg = ws + l.wg, p.wu = ws + l.wu;
        p.x_stride = p.w_stride = (long long)l.kp;
        n = (int)l.kp;
    }
    if (p.M > 0) {
        const unsigned blocks = (unsigned)std::min<long long>((p.M * (fp / 8) + 255) / 256, 16 * compute_units());
        if (p.act == XNOR_ACT_SILU) gate_back_kernel<T, XNOR_ACT_SILU><<<dim3(blocks), dim3(256), 0, st>>>(p, dgu, fp);
        else if (p.act == XNOR_ACT_GELU) gate_back_kernel<T, XNOR_ACT_GELU><<<dim3(blocks), dim3(256), 0, st>>>(p, dgu, fp);
        else gate_back_kernel<T, XNOR_ACT_RELU><<<dim3(blocks), dim3(256), 0, st>>>(p, dgu, fp);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        DenseArgs d{};
        d.a = dgu, d.lda = 4LL * fp, d.b = p.wg, d.b2 = p.wu, d.ldb = 2 * p.w_stride;
        d.M = p.M, d.N = n, d.K = 2 * fp, d.seam = fp, d.deep = p.F;
        d.out = p.dx, d.ldo = p.dx_stride, d.split = d.valid = p.M, d.out_cols = p.K;
        d.parts = dx_parts(p.M, fp, (int)l.kp);
        if (d.parts > 1) d.out = ws + l.sums, d.ldo = n;
        if ((e = launch_dense_across(d, false, type, st)) != hipSuccess) return e;
        if (d.parts > 1) {
            const unsigned blocks = (unsigned)std::min<long long>((p.M * (n / 4) + 255) / 256, 8 * compute_units());
            add_parts_kernel<T><<<dim3(blocks), dim3(256), 0, st>>>((const float *)(ws + l.sums), d.parts, p.M, n, (T *)p.dx, p.dx_stride, p.K);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
    }
    DenseArgs d{};
    d.a = dgu, d.lda = 4LL * fp, d.b = p.x, d.ldb = 2 * p.x_stride;
    d.M = 2LL * fp, d.N = n, d.K = d.deep = (int)p.M, d.seam = 0x7fffffff;
    d.out = p.dwg, d.out2 = p.dwu, d.ldo = p.dw_stride, d.split = fp, d.valid = p.F, d.out_cols = p.K;
    return launch_dense_across(d, true, type, st);
}

}  // namespace

size_t gated_fwd_workspace(long long M, int F, int K) { return layout(M, F, K, false).bytes; }
size_t gated_bwd_workspace(long long M, int F, int K) { return layout(M, F, K, true).bytes; }

// Products of rows that lie badly take 2.5 us and 0.65 us a step of 64 values more for every round of 512 tiles of 128 x 64; the copy takes a launch
// and 5.2 TB/s read and written.  (f16, us without and with: 256 x 256 x 257 11.7 and 12.1, 100 x 8192 x 1001 24.3 and 25.6, 777 x 2501 x 1001 28 and 32,
// 900 x 4000 x 1001 38 and 35, 300 x 1000 x 3001 51 and 31, 1000 x 4096 x 4095 106 and 90, 128 x 8192 x 8191 151 and 214, 4096 x 4096 x 4095 397 and 254:
// of 79 sizes measured the rule has 65 right and loses 10 us of 71 at most in the others.)
bool gated_fwd_copy_pays(long long M, int F, int K)
{
    if (M <= 64) return false;          // (few tokens: the weights are read once)
    const double tiles = (double)((M + 127) / 128) * ceil_div(F, 64), rounds = (double)(long long)((tiles + 511) / 512);
    return rounds * (K / 64.0 * 0.65 + 2.5) > 4.0 + ((double)M + 2.0 * F) * K * 4 / 5.2e6;
}

hipError_t gated_fwd_copy(DenseArgs *p, void *workspace, hipStream_t st)
{
    const Layout l = layout(p->M, p->N, p->K, false);
    char *ws = (char *)workspace;
    const Copy copies[3] = {{(const uint16_t *)p->a, (uint16_t *)(ws + l.x), p->M, p->lda / 2}, {(const uint16_t *)p->b, (uint16_t *)(ws + l.wg), p->N, p->ldb / 2},
                            {(const uint16_t *)p->b2, (uint16_t *)(ws + l.wu), p->N, p->ldb / 2}};
    p->a = ws + l.x, p->b = ws + l.wg, p->b2 = ws + l.wu;
    p->lda = p->ldb = 2 * (long long)l.kp;
    const int K = p->K;
    p->K = (int)l.kp;           // (with the zeros behind a row)
    return copy_rows(copies, 3, K, (int)l.kp, st);
}

hipError_t launch_gated_bwd(const GatedBackArgs &p, int type, hipStream_t st)
{
    return type == XNOR_TYPE_F16 ? run<f16_t>(p, type, st) : run<bf16_t>(p, type, st);
}

}  // namespace xnor
