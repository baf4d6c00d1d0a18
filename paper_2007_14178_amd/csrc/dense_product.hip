// Products of the dense operators on the matrix cores: out = a b^T for rows of 8-bit integers, f16 or bf16, and the gated
// block's pair of products with its activation.
//
// A tile of TM tokens x TN rows of b is one workgroup's.  128 bytes of each row's contraction are staged in LDS at a time; the
// three types differ only in the instruction that takes 16 bytes a lane.  b's rows are the instruction's first operand, so that a lane
// ends up with four consecutive outputs of one token.
#include <algorithm>

#include "dense_common.hpp"

namespace xnor {
namespace {

enum Epilogue { kPlain, kGated, kInt8, kInt8Gated };

template <class T> struct Mat;
template <> struct Mat<int8_t> {
    typedef i32x4 acc;
    static __device__ acc mul(i32x4 a, i32x4 b, acc c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
};
template <> struct Mat<f16_t> {
    typedef f32x4 acc;
    static __device__ acc mul(i32x4 a, i32x4 b, acc c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};
template <> struct Mat<bf16_t> {
    typedef f32x4 acc;
    static __device__ acc mul(i32x4 a, i32x4 b, acc c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};

constexpr int kStep = 128;      // bytes of a row staged at a time

// Row r of a tile's b operand, whose first row stands for output n0: in the gated block 16 rows of the first matrix and the 16 of
// the second for the same outputs take turns.
template <bool GATED>
__device__ inline const char *b_row(const DenseArgs &p, int n0, int r)
{
    if (!GATED) return (const char *)p.b + (long long)min(n0 + r, p.N - 1) * p.ldb;
    const int n = min(n0 + (r >> 5) * 16 + (r & 15), p.N - 1);
    return (const char *)(r & 16 ? p.b2 : p.b) + n * p.ldb;
}

// Four consecutive outputs n .. n+3 of token m.  Every value is formed in fp32 and rounded once, where it is stored.
template <class T, class O, int EPI, class Acc>
__device__ inline void finish(const DenseArgs &p, long long m, int n, const Acc &v, const Acc &w)
{
    O out[4];
    if constexpr (EPI == kInt8) {
        const float s = p.a_scale[m];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = min(n + i, p.N - 1);
            const float y = (float)v[i] * (s * p.b_scale[at]);
            out[i] = (O)(p.bias ? y + p.bias[at] : y);
        }
        store_values((O *)p.out + m * p.ldo, n, p.N, out);
    } else if constexpr (EPI == kPlain) {
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = (O)v[i];
        const bool second = m >= p.split;
        const long long r = second ? m - p.split : m;
        if (r < p.valid) store_values((O *)(second ? p.out2 : p.out) + r * p.ldo, n, p.N, out);
    } else {
        float g[4], u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            g[i] = (float)v[i];
            u[i] = (float)w[i];
            if constexpr (EPI == kInt8Gated) {
                const int at = min(n + i, p.N - 1);
                const float s = p.a_scale[m];
                g[i] *= s * p.b_scale[at];
                u[i] *= s * p.b2_scale[at];
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = p.act == XNOR_ACT_SILU ? act_value<XNOR_ACT_SILU>(g[i])
                            : p.act == XNOR_ACT_GELU ? act_value<XNOR_ACT_GELU>(g[i]) : act_value<XNOR_ACT_RELU>(g[i]);
            out[i] = (O)(a * u[i]);
        }
        store_values((O *)p.out + m * p.ldo, n, p.N, out);
        if constexpr (EPI == kGated) {
            if (p.out2) {
#pragma unroll
                for (int i = 0; i < 4; ++i) out[i] = (O)g[i];
                store_values((O *)p.out2 + m * p.ldo2, n, p.N, out);
#pragma unroll
                for (int i = 0; i < 4; ++i) out[i] = (O)u[i];
                store_values((O *)p.out3 + m * p.ldo2, n, p.N, out);
            }
        }
    }
}

// 128 tokens x 128 rows of b, four waves of 64 x 64, rows of any alignment and length staged through registers.
template <class T, class O, int EPI>
__global__ __launch_bounds__(256, 2) void dense_tile_kernel(const DenseArgs p, int tiles_n)
{
    constexpr bool GATED = EPI == kGated || EPI == kInt8Gated;
    constexpr int TN = GATED ? 64 : 128;        // outputs n of a tile
    typedef Mat<T> X;
    __shared__ __align__(16) char lds[2 * 128 * kStep];
    char *la = lds, *lb = lds + 128 * kStep;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int n0 = (int)(blockIdx.x % (unsigned)tiles_n) * TN;
    const long long m0 = p.first + (long long)(blockIdx.x / (unsigned)tiles_n) * 128;
    const int wm = (wave & 1) * 64, wn = (wave >> 1) * 64;

    typename X::acc acc[4][4] = {};
    const int steps = (int)(((long long)p.K * (int)sizeof(T) + kStep - 1) / kStep);
    for (int s = 0; s < steps; ++s) {
        i32x4 va[4], vb[4];
        const int chunk = t & 7, at = (s * kStep + chunk * 16) / (int)sizeof(T);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (t >> 3) + 32 * i;
            const long long m = m0 + r < p.M ? m0 + r : p.M - 1;
            const Chunk<T> ca = load_chunk((const T *)((const char *)p.a + m * p.lda), at, p.K);
            const Chunk<T> cb = load_chunk((const T *)b_row<GATED>(p, n0, r), at, p.K);
            va[i] = __builtin_bit_cast(i32x4, ca);
            vb[i] = __builtin_bit_cast(i32x4, cb);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (t >> 3) + 32 * i, to = r * kStep + ((chunk ^ (r & 7)) << 4);
            *(i32x4 *)(la + to) = va[i];
            *(i32x4 *)(lb + to) = vb[i];
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            i32x4 fa[4], fb[4];
            const int c = h * 4 + (lane >> 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int ra = wm + i * 16 + (lane & 15), rb = wn + i * 16 + (lane & 15);
                fa[i] = *(const i32x4 *)(la + ra * kStep + ((c ^ (ra & 7)) << 4));
                fb[i] = *(const i32x4 *)(lb + rb * kStep + ((c ^ (rb & 7)) << 4));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = X::mul(fb[i], fa[j], acc[i][j]);
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const long long m = m0 + wm + j * 16 + (lane & 15);
        if (m >= p.M) continue;
        if constexpr (GATED) {
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                const int n = n0 + wn / 2 + i * 8 + (lane >> 4) * 4;
                if (n < p.N) finish<T, O, EPI>(p, m, n, acc[i][j], acc[i + 1][j]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int n = n0 + wn + i * 16 + (lane >> 4) * 4;
                if (n < p.N) finish<T, O, EPI>(p, m, n, acc[i][j], acc[i][j]);
            }
        }
    }
}

template <class T, class O, int EPI>
hipError_t launch(const DenseArgs &p, hipStream_t st)
{
    constexpr int TN = EPI == kGated || EPI == kInt8Gated ? 64 : 128;
    if (p.M == 0) return hipSuccess;
    const int tiles_n = ceil_div(p.N, TN);
    // (a launch has fewer than 2^32 threads: more tokens than that gives in several)
    const long long rows = std::max<long long>(1, kMaxBlocks / tiles_n) * 128;
    for (long long m = 0; m < p.M; m += rows) {
        DenseArgs q = p;
        q.first = m;
        q.M = std::min(p.M, m + rows);
        dense_tile_kernel<T, O, EPI><<<dim3((unsigned)(tiles_n * ((q.M - m + 127) / 128))), dim3(256), 0, st>>>(q, tiles_n);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_dense(const DenseArgs &p, int type, hipStream_t st)
{
    return type == XNOR_TYPE_F16 ? launch<f16_t, f16_t, kPlain>(p, st) : launch<bf16_t, bf16_t, kPlain>(p, st);
}

hipError_t launch_dense_gated(const DenseArgs &p, int type, hipStream_t st)
{
    return type == XNOR_TYPE_F16 ? launch<f16_t, f16_t, kGated>(p, st) : launch<bf16_t, bf16_t, kGated>(p, st);
}

hipError_t launch_dense_int8(const DenseArgs &p, int out_type, hipStream_t st)
{
    return out_type == XNOR_TYPE_FP32  ? launch<int8_t, float, kInt8>(p, st)
           : out_type == XNOR_TYPE_F16 ? launch<int8_t, f16_t, kInt8>(p, st) : launch<int8_t, bf16_t, kInt8>(p, st);
}

hipError_t launch_dense_int8_gated(const DenseArgs &p, int out_type, hipStream_t st)
{
    return out_type == XNOR_TYPE_FP32  ? launch<int8_t, float, kInt8Gated>(p, st)
           : out_type == XNOR_TYPE_F16 ? launch<int8_t, f16_t, kInt8Gated>(p, st) : launch<int8_t, bf16_t, kInt8Gated>(p, st);
}

}  // namespace xnor
