// How the products' kernels see their operands and finish their outputs.
#pragma once

#include "dense_common.hpp"

namespace xnor {

enum Epilogue { kPlain, kGated, kInt8, kInt8Gated, kSums };     // kSums: fp32 sums over a part of the contraction

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

constexpr int kStep = 128;      // bytes of a row that are taken together

// Row r of a tile's b operand, whose first row stands for output n0: in the gated block 16 rows of the first matrix and the 16 of
// the second for the same outputs take turns.
template <bool GATED>
__device__ inline const char *b_row(const DenseArgs &p, int n0, int r)
{
    if (!GATED) return (const char *)p.b + (long long)min(n0 + r, p.N - 1) * p.ldb;
    const int n = min(n0 + (r >> 5) * 16 + (r & 15), p.N - 1);
    return (const char *)(r & 16 ? p.b2 : p.b) + n * p.ldb;
}

// What four consecutive outputs n .. n+3 of a lane have in common for all its tokens.
template <int EPI>
struct Columns {
    float scale[4], scale2[4], bias[4];
    __device__ inline void load(const DenseArgs &p, int n)
    {
        if constexpr (EPI == kInt8 || EPI == kInt8Gated) load_params(p.b_scale, n, p.N, 0.f, scale);
        if constexpr (EPI == kInt8Gated) load_params(p.b2_scale, n, p.N, 0.f, scale2);
        if constexpr (EPI == kInt8) load_params(p.bias, n, p.N, 0.f, bias);
    }
};

// These outputs of token m.  Every value is formed in fp32 and rounded once, where it is stored.  s: the token's scale (8-bit operands).
template <class T, class O, int EPI, class Acc>
__device__ inline void finish(const DenseArgs &p, long long m, float s, int n, const Columns<EPI> &c, const Acc &v, const Acc &w)
{
    O out[4];
    if constexpr (EPI == kInt8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float y = (float)v[i] * (s * c.scale[i]);
            out[i] = (O)(p.bias ? y + c.bias[i] : y);
        }
        // fp32 outputs whose rows are whole cache lines go past the caches, which the tokens that the next tiles read stay in (100352 x 512 x 512
        // with its quantisation 131 -> 122 us; rows of 4000 bytes would reach memory in pieces, 16384 x 1000 x 1024 27 -> 54 us, as would 16-bit
        // outputs, 32 bytes of a token at a time)
        O *const to = (O *)p.out + m * p.ldo + n;
        const bool lines = sizeof(O) == 4 && ((reinterpret_cast<uintptr_t>(p.out) | (uintptr_t)p.ldo * 4) & 127) == 0;
        if (lines && n + 4 <= p.N) {
            __builtin_nontemporal_store(f32x4{(float)out[0], (float)out[1], (float)out[2], (float)out[3]}, (f32x4 *)to);
        } else {
            store_values((O *)p.out + m * p.ldo, n, p.N, out);
        }
    } else if constexpr (EPI == kSums) {
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = v[i];
        store_values((O *)p.out + m * p.ldo, n, p.N, out);
    } else if constexpr (EPI == kPlain) {
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = (O)v[i];
        const bool second = m >= p.split;
        const long long r = second ? m - p.split : m;
        if (r < p.valid) store_values((O *)(second ? p.out2 : p.out) + r * p.ldo, n, p.out_cols, out);
    } else {
        float g[4], u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            g[i] = (float)v[i];
            u[i] = (float)w[i];
            if constexpr (EPI == kInt8Gated) {
                g[i] *= s * c.scale[i];
                u[i] *= s * c.scale2[i];
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            constexpr bool SHORT = sizeof(O) == 2;
            const float a = p.act == XNOR_ACT_SILU ? act_value<XNOR_ACT_SILU, SHORT>(g[i])
                            : p.act == XNOR_ACT_GELU ? act_value<XNOR_ACT_GELU, SHORT>(g[i]) : act_value<XNOR_ACT_RELU, SHORT>(g[i]);
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

// Tokens up to which a product goes to the kernel for few tokens, and its launcher (EPI an Epilogue).
constexpr int kFewTokens = 64;
template <class T, class O, int EPI>
hipError_t launch_few(const DenseArgs &p, hipStream_t st);

}  // namespace xnor
