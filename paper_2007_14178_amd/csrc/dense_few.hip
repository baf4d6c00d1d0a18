// Products for few tokens (a decoding step): b is read once, by as many waves as there are, and that is what they take (gated, one token x 4096 x
// 8192 bf16 27.4 us, 4.9 TB/s, 8 bits 15.3 us, 4.4 TB/s, and 13.0-13.6 us where the weights are in the last-level cache from the pass before; one token x
// 4096 x 4096 on 8 bits with its quantisation 6.8-7.6 us, where a launch and the latency of
// one round of loads are most of it: those of the token and the first of b's are on their way together).
//
// A workgroup has 16 rows of b (of each matrix in the gated block), its eight waves an eighth of the contraction each, whose sums are
// added in LDS.  The tokens are columns of the matrix instruction: up to 16 cost what one costs.
#include <type_traits>

#include "dense_tile.hpp"

namespace xnor {
namespace {

constexpr int kWaves = 8, kThreads = kWaves * kWave;
// Real tokens that can be quantised in the product's launch, by every workgroup for itself: one or two by all its waves together, shorter ones by a
// wave each, up to eight, or, still shorter, by a wave each two.
constexpr int kTogether = 2, kTogetherCols = 8192, kRealTokens = 2 * kWaves, kRealCols = 2048, kRealColsOfTwo = 1280;

// X: the type of real tokens, quantised by every workgroup for itself; void: a holds T.
template <class T, class O, int EPI, int TT, class X>
__global__ __launch_bounds__(kThreads) void few_kernel(const DenseArgs p)
{
    constexpr bool GATED = EPI == kGated || EPI == kInt8Gated, REAL = !std::is_void<X>::value;
    // U: steps whose loads are on their way together (gated, one token x 4096 x 8192 8 bits: 13.6 us, with four 14.9).
    constexpr int MATS = GATED ? 2 : 1, U = TT < 4 && !GATED ? 4 : 2;
    typedef Mat<T> Mul;
    typedef typename Mul::acc Acc;
    __shared__ Acc sums[kWaves][MATS][TT][kWave];
    __shared__ float tops[kTogether][kWaves], scales[kRealTokens];
    extern __shared__ __align__(16) int8_t levels[];        // real tokens: [M][whole steps]
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, r = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16;
    const int steps = (int)(((long long)p.K * (int)sizeof(T) + kStep - 1) / kStep), share = (steps + kWaves - 1) / kWaves;
    const int from = wave * share, to = min(steps, from + share);
    const int held_bytes = steps * kStep;

    const long long row = min(n0 + r, p.N - 1);
    const T *b[MATS];
    b[0] = (const T *)((const char *)p.b + row * p.ldb);
    if constexpr (GATED) b[1] = (const T *)((const char *)p.b2 + row * p.ldb);
    const T *a[TT];
#pragma unroll
    for (int j = 0; j < TT; ++j) {
        const long long m = min((long long)j * 16 + r, p.M - 1);
        a[j] = (const T *)((const char *)p.a + m * p.lda);
    }

    i32x4 vb[MATS][U][2];
    auto load_b = [&](int s) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < MATS; ++k)
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int at = ((s + u) * kStep + g * 32 + i * 16) / (int)sizeof(T);
                    if (s + u < to) vb[k][u][i] = __builtin_bit_cast(i32x4, load_chunk(b[k], at, p.K));
                }
    };

    float scale[TT] = {};
    if constexpr (REAL) {
        // the tokens first, b's first rows on their way while the tokens are quantised
        constexpr int XV = 16 / (int)sizeof(X);
        if (p.M <= kTogether) {
            constexpr int CHUNKS = kTogetherCols / (kThreads * XV);
            Chunk<X> held[kTogether][CHUNKS];
#pragma unroll
            for (int m = 0; m < kTogether; ++m)
                if (m < p.M)
#pragma unroll
                    for (int c = 0; c < CHUNKS; ++c)
                        held[m][c] = load_chunk((const X *)((const char *)p.a + m * p.lda), (t + c * kThreads) * XV, p.K);
            load_b(from);
#pragma unroll
            for (int m = 0; m < kTogether; ++m)
                if (m < p.M) {
                    float top = 0.f;
#pragma unroll
                    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                        for (int k = 0; k < XV; ++k) top = MaxNan()(fabsf((float)held[m][c].v[k]), top);
                    top = wave_reduce(top, MaxNan());
                    if (lane == 0) tops[m][wave] = top;
                }
            __syncthreads();
#pragma unroll
            for (int m = 0; m < kTogether; ++m)
                if (m < p.M) {
                    float top = tops[m][0];
#pragma unroll
                    for (int w = 1; w < kWaves; ++w) top = MaxNan()(tops[m][w], top);
                    const RowLevels l = row_levels(top);
                    if (r == m) scale[0] = l.scale;
#pragma unroll
                    for (int c = 0; c < CHUNKS; ++c) {
                        const int at = (t + c * kThreads) * XV;
                        int8_t q[XV];
#pragma unroll
                        for (int k = 0; k < XV; ++k) q[k] = level_of((float)held[m][c].v[k], l);
                        if (at < held_bytes) __builtin_memcpy(levels + m * held_bytes + at, q, XV);        // (zeros behind the token's end)
                    }
                }
            __syncthreads();
        } else {
            constexpr int CHUNKS = kRealCols / (kWave * XV);
            Chunk<X> held[2][CHUNKS];
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (wave + i * kWaves < p.M)
#pragma unroll
                    for (int c = 0; c < CHUNKS; ++c)
                        held[i][c] = load_chunk((const X *)((const char *)p.a + (wave + i * kWaves) * p.lda), (lane + c * kWave) * XV, p.K);
            load_b(from);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int m = wave + i * kWaves;
                if (m >= p.M) continue;
                float top = 0.f;
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                    for (int k = 0; k < XV; ++k) top = MaxNan()(fabsf((float)held[i][c].v[k]), top);
                const RowLevels l = row_levels(wave_reduce(top, MaxNan()));
                if (lane == 0) scales[m] = l.scale;
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) {
                    const int at = (lane + c * kWave) * XV;
                    int8_t q[XV];
                    if (at >= held_bytes) continue;
#pragma unroll
                    for (int k = 0; k < XV; ++k) q[k] = level_of((float)held[i][c].v[k], l);
                    __builtin_memcpy(levels + m * held_bytes + at, q, XV);
                }
            }
            __syncthreads();
            scale[0] = scales[min(r, (int)p.M - 1)];
        }
    } else {
        load_b(from);
#pragma unroll
        for (int j = 0; j < TT; ++j) {
            const long long m = j * 16 + r;
            scale[j] = p.a_scale && m < p.M ? p.a_scale[m] : 1.f;
        }
    }

    Columns<EPI> columns;
    columns.load(p, n0 + g * 4);
    Acc acc[MATS][TT] = {};
    for (int s = from; s < to; s += U) {
        if (s > from) load_b(s);
        i32x4 va[U][2][TT];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (s + u < to) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < TT; ++j) {
                        const int at = (s + u) * kStep + g * 32 + i * 16;
                        if constexpr (REAL) va[u][i][j] = *(const i32x4 *)(levels + min(r, (int)p.M - 1) * held_bytes + at);
                        else va[u][i][j] = __builtin_bit_cast(i32x4, load_chunk(a[j], at / (int)sizeof(T), p.K));
                    }
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (s + u < to) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < TT; ++j)
#pragma unroll
                        for (int k = 0; k < MATS; ++k) acc[k][j] = Mul::mul(vb[k][u][i], va[u][i][j], acc[k][j]);
            }
    }
#pragma unroll
    for (int k = 0; k < MATS; ++k)
#pragma unroll
        for (int j = 0; j < TT; ++j) sums[wave][k][j][lane] = acc[k][j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < TT; ++j) {
        const long long m = j * 16 + r;
        const int n = n0 + g * 4;
        if (wave != j % kWaves || m >= p.M || n >= p.N) continue;       // (a wave a tile of tokens)
        Acc v[MATS];
#pragma unroll
        for (int k = 0; k < MATS; ++k) {
            v[k] = sums[0][k][j][lane];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) v[k] += sums[w][k][j][lane];
        }
        finish<T, O, EPI>(p, m, scale[j], n, columns, v[0], v[MATS - 1]);
    }
}

}  // namespace

template <class T, class O, int EPI>
hipError_t launch_few(const DenseArgs &p, hipStream_t st)
{
    const dim3 grid((unsigned)ceil_div(p.N, 16));
    if (p.M <= 16) few_kernel<T, O, EPI, 1, void><<<grid, dim3(kThreads), 0, st>>>(p);
    else if (p.M <= 32) few_kernel<T, O, EPI, 2, void><<<grid, dim3(kThreads), 0, st>>>(p);
    else few_kernel<T, O, EPI, 4, void><<<grid, dim3(kThreads), 0, st>>>(p);
    return hipGetLastError();
}

template hipError_t launch_few<int8_t, float, kInt8>(const DenseArgs &, hipStream_t);
template hipError_t launch_few<int8_t, f16_t, kInt8>(const DenseArgs &, hipStream_t);
template hipError_t launch_few<int8_t, bf16_t, kInt8>(const DenseArgs &, hipStream_t);
template hipError_t launch_few<int8_t, float, kInt8Gated>(const DenseArgs &, hipStream_t);
template hipError_t launch_few<int8_t, f16_t, kInt8Gated>(const DenseArgs &, hipStream_t);
template hipError_t launch_few<int8_t, bf16_t, kInt8Gated>(const DenseArgs &, hipStream_t);
template hipError_t launch_few<f16_t, f16_t, kGated>(const DenseArgs &, hipStream_t);
template hipError_t launch_few<bf16_t, bf16_t, kGated>(const DenseArgs &, hipStream_t);

bool dense_few_real_supports(long long M, int K)
{
    return M <= kTogether ? K <= kTogetherCols : M <= kWaves ? K <= kRealCols : M <= kRealTokens && K <= kRealColsOfTwo;
}

// Two workgroups fit on a unit, and those of a second round quantise all tokens once more behind the first: then a launch of its own for the
// tokens is the faster form, for one token from the third round on.  With more than eight tokens already a second workgroup on a unit costs more than
// the host's 4 us for another launch, which passes of this size take.  GPU time in us by one launch and by two, f16 (the host's call 7 and 11):
//     tokens x inner    N = 4096         8192           10240          16384          49152
//     1 x 4096          7.5  9.0     10.4  12.4     14.3  15.5     17.7  18.4     45.6  43.6
//     3 x 1280          6.0  6.8      7.3   7.6     10.8   9.2     12.1  10.5     30.6  21.4
//     8 x 2048          7.0  7.9      9.2   9.4     12.3  11.5     15.7  13.6     36.6  28.1
//    16 x 256           7.5  5.7      9.4   5.9     13.4   6.8     16.1   7.7     42.4  14.5
//    16 x 1280          8.9  7.4     11.5   8.6     16.6  10.4     19.9  11.9     50.9  24.8
bool dense_few_real_pays(long long M, int N)
{
    return ceil_div(N, 16) <= (M == 1 ? 4 : M <= kWaves ? 2 : 1) * kPlanUnits;
}

template <class X>
static hipError_t few_real(const DenseArgs &p, int out_type, hipStream_t st)
{
    const dim3 grid((unsigned)ceil_div(p.N, 16));
    const size_t lds = (size_t)p.M * ceil_div(p.K, kStep) * kStep;
    if (out_type == XNOR_TYPE_FP32) few_kernel<int8_t, float, kInt8, 1, X><<<grid, dim3(kThreads), lds, st>>>(p);
    else if (out_type == XNOR_TYPE_F16) few_kernel<int8_t, f16_t, kInt8, 1, X><<<grid, dim3(kThreads), lds, st>>>(p);
    else few_kernel<int8_t, bf16_t, kInt8, 1, X><<<grid, dim3(kThreads), lds, st>>>(p);
    return hipGetLastError();
}

hipError_t launch_dense_few_real(const DenseArgs &p, int x_type, int out_type, hipStream_t st)
{
    return x_type == XNOR_TYPE_FP32 ? few_real<float>(p, out_type, st)
           : x_type == XNOR_TYPE_F16 ? few_real<f16_t>(p, out_type, st) : few_real<bf16_t>(p, out_type, st);
}

}  // namespace xnor
