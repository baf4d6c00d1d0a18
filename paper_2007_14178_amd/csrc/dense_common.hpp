// What the dense operators (8-bit and 16-bit products, layer norm, the gated block) share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>

#include "xnor_internal.hpp"

namespace xnor {

typedef _Float16 f16_t;
typedef __bf16 bf16_t;
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef f16_t f16x8 __attribute__((ext_vector_type(8)));
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kWave = 64;

// 16 bytes of values as one load or store.  Any byte address will do: global accesses need no alignment on this target.
template <class T>
struct Chunk {
    static constexpr int kCount = 16 / (int)sizeof(T);
    T v[kCount];
};

// The chunk that starts `at` values into a row of `n`; values behind the row's end are zero.
template <class T>
__device__ inline Chunk<T> load_chunk(const T *row, int at, int n)
{
    Chunk<T> c;
    if (at + Chunk<T>::kCount <= n) {
        __builtin_memcpy(&c, row + at, 16);
    } else {
#pragma unroll
        for (int i = 0; i < Chunk<T>::kCount; ++i) c.v[i] = at + i < n ? row[at + i] : T(0);
    }
    return c;
}

// COUNT values to row[at ..], as far as the row goes.
template <class T, int COUNT>
__device__ inline void store_values(T *row, int at, int n, const T (&v)[COUNT])
{
    if (at + COUNT <= n) {
        __builtin_memcpy(row + at, v, sizeof v);
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
            if (at + i < n) row[at + i] = v[i];
    }
}

// V parameters from `at` on as fp32; `none` where there are no parameters, and anything behind the end.
template <int V, class P>
__device__ inline void load_params(const P *p, int at, int n, float none, float (&to)[V])
{
    P raw[V];
    if (p && at + V <= n) {
        __builtin_memcpy(raw, p + at, sizeof raw);
#pragma unroll
        for (int k = 0; k < V; ++k) to[k] = (float)raw[k];
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k) to[k] = p && at + k < n ? (float)p[at + k] : none;
    }
}

// v of the lane that CTRL names, within 16 lanes.
template <int CTRL>
__device__ inline float dpp(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

// Over a wave, to all lanes: the other of each pair, pair of pairs, half and whole row of 16 lanes by DPP, then two exchanges.
template <class Op>
__device__ inline float wave_reduce(float v, Op op)
{
    v = op(v, dpp<0xb1>(v));
    v = op(v, dpp<0x4e>(v));
    v = op(v, dpp<0x141>(v));
    v = op(v, dpp<0x140>(v));
    v = op(v, __shfl_xor(v, 16));
    return op(v, __shfl_xor(v, 32));
}

struct Sum {
    __device__ float operator()(float a, float b) const { return a + b; }
};

// fmaxf drops a NaN; a row's largest magnitude keeps it.
struct MaxNan {
    __device__ float operator()(float a, float b) const { return a > b || a != a ? a : b; }
};

// Rows whose largest magnitude is below this are quantised to zeros: 127 / max and max / 127 stay normal numbers.
constexpr float kQuantFloor = 0x1p-100f;

// The factor that takes a row to its levels, and the size of a level.  A row that holds a NaN or an infinity has neither: its
// levels are 0 and its scale is NaN, so that whatever is computed from it is NaN.
struct RowLevels {
    float to, scale;
};
__device__ inline RowLevels row_levels(float top)
{
    if (top < kQuantFloor) return {0.f, 0.f};
    if (!(top <= 3.402823466e38f)) return {0.f, __uint_as_float(0x7fc00000u)};
    return {127.f / top, top / 127.f};
}
__device__ inline int8_t level_of(float x, const RowLevels &r)
{
    // (r.to 0: whatever x is, NaN and infinity among them, its level is 0)
    return r.to == 0.f ? (int8_t)0 : (int8_t)(int)rintf(x * r.to);
}

// erfc(z) for z >= 0 as t exp(p(t) - z^2) with t = 1 / (1 + z/2), the substitution of Numerical Recipes (Press et al., section 6.2):
// log(erfc(z) e^(z^2) / t) is smooth in t, and p is its fit of degree 7 by least squares at 4000 Chebyshev nodes of t in [1/8, 1] (z up to 14), the
// weights multiplied by |error| / mean |error| + 0.001 sixty times over, towards the least greatest error: 7e-7.  In fp32, with an exact
// exponential, it is 1.1e-6 up to z = 2, 3.5e-6 to 5 and 1.2e-5 to 9, where rounding z^2 is what is left.
__device__ inline float erfc_short(float z)
{
    const float x = fabsf(z), t = __builtin_amdgcn_rcpf(1.f + 0.5f * x);
    float p = -0.187363292f;
    p = p * t + 0.750145849f;
    p = p * t - 0.9993171f;
    p = p * t + 0.349105959f;
    p = p * t - 0.0398076377f;
    p = p * t + 0.394194611f;
    p = p * t + 0.998510106f;
    p = p * t - 1.26546918f;
    const float e = t * __builtin_amdgcn_exp2f((p - x * x) * 1.44269504f);
    return z < 0.f ? 2.f - e : e;
}

// Activations of the gated block and their derivatives, in fp32.  ACT: an xnor_act.  SHORT: for results that are rounded to 16 bits: by the
// exponential and reciprocal instructions, within a few roundings of |g|, a fortieth of the results' own at most (2000 x 4096 x 8192 silu on 8 bits
// 123 us with the functions, 115 us so; 4096 x 4096 x 8192 on f16 gelu 455 us and 433, silu 438 and 430).
template <bool SHORT>
__device__ inline float sigmoid(float g)
{
    if constexpr (SHORT) return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(g * -1.44269504f));
    return 1.f / (1.f + expf(-g));
}
template <int ACT, bool SHORT>
__device__ inline float act_value(float g)
{
    if constexpr (ACT == XNOR_ACT_SILU) return SHORT ? g * sigmoid<SHORT>(g) : g / (1.f + expf(-g));
    if constexpr (ACT == XNOR_ACT_GELU) return 0.5f * g * (SHORT ? erfc_short(g * -0.70710678118654752f) : erfcf(g * -0.70710678118654752f));
    return g > 0.f ? g : (g != g ? g : 0.f);
}
// For the backward pass, whose dg and du are rounded to 16 bits.
template <int ACT>
__device__ inline float act_slope(float g)
{
    if constexpr (ACT == XNOR_ACT_SILU) {
        const float s = sigmoid<true>(g);
        return s * (1.f + g * (1.f - s));
    }
    if constexpr (ACT == XNOR_ACT_GELU)
        return 0.5f * erfc_short(g * -0.70710678118654752f) + g * __builtin_amdgcn_exp2f(g * g * -0.72134752f) * 0.39894228040143268f;
    return g > 0.f ? 1.f : (g != g ? g : 0.f);
}

// One product of the dense operators: out[m][n] = sum_k a[m][k] b[n][k], both operands with the contraction along their rows (or
// across them: launch_dense_across).  Strides of a and b are in bytes, of outputs in values.
struct DenseArgs {
    const void *a;              // [M][K]
    const void *b, *b2;         // [N][K]; b2: the gated block's second matrix
    long long lda, ldb;
    long long M;
    int N, K;                   // K in values
    void *out, *out2, *out3;    // gated: h, and g and u or NULL.  Plain: rows from `split` on go to out2
    long long ldo, ldo2;
    long long split, valid;     // plain: of the rows of either output the first `valid` are written, and of a row `out_cols` values
    int out_cols;
    int parts;                  // b across, a not: > 1: out is fp32 [parts][M][N], each the sums over a share of the contraction
    int seam, deep;             // b across: contraction values from `seam` on are b2's rows, of which, as of b's, there are `deep`
    const float *a_scale, *b_scale, *b2_scale, *bias;
    int act;
    long long first;            // (set by the launchers: the launch's first token)
};

constexpr long long kMaxBlocks = 1 << 22;      // of a launch, for up to 512 threads each: fewer than 2^32 threads

// 16-bit out = a b^T with b as [K][N], and a as [M][K] or [K][M] (a_across): rows at multiples of 16 bytes, N and (a_across) M of 8 values,
// a stride of b that holds its rows; seam a multiple of 64 values.  Rows of 64 contraction values within 31 bits.
hipError_t launch_dense_across(const DenseArgs &p, bool a_across, int type, hipStream_t st);
// Whether the products' rows are where the fast kernels take them (16-byte boundaries); elsewhere they run slower.
bool dense_direct_supports(const DenseArgs &p, int type);
hipError_t launch_dense_gated(const DenseArgs &p, int type, hipStream_t st);                 // 16-bit
hipError_t launch_dense_int8(const DenseArgs &p, int out_type, hipStream_t st);
hipError_t launch_dense_int8_gated(const DenseArgs &p, int out_type, hipStream_t st);
// The 8-bit product of real tokens, a and lda theirs, quantised in the kernel; where it takes them, and where it is not slower for that.
bool dense_few_real_supports(long long M, int K);
bool dense_few_real_pays(long long M, int N);
hipError_t launch_dense_few_real(const DenseArgs &p, int x_type, int out_type, hipStream_t st);

struct RowArgs {
    const void *x;
    long long rows;
    int cols;
    long long x_stride;
    const void *gamma, *beta;
    float eps;
    void *y;
    int8_t *q;
    long long y_stride;          // of y or q
    float *scale, *mean, *rstd;
};
hipError_t launch_quantize(const RowArgs &p, int x_type, hipStream_t st);
hipError_t launch_layer_norm(const RowArgs &p, int x_type, int p_type, hipStream_t st);      // y or q
struct NormBackArgs {
    const void *dy, *x, *gamma;
    long long rows;
    int cols;
    long long dy_stride, x_stride, dx_stride;
    const float *mean, *rstd;
    void *dx, *dgamma, *dbeta;
    float *partial;              // workspace
};
size_t layer_norm_bwd_workspace(int x_type, long long rows, int cols);
hipError_t launch_layer_norm_bwd(const NormBackArgs &p, int x_type, int p_type, hipStream_t st);

struct GatedBackArgs {
    const void *dh, *x, *wg, *wu, *g, *u;
    long long dh_stride, x_stride, w_stride, gu_stride, dx_stride, dw_stride;
    int act;
    long long M;
    int F, K;
    void *dx, *dwg, *dwu;
    void *workspace;
};
constexpr int kMaxGatedBack = 1 << 20;         // F and K of the backward pass: 255 rows of [dg du] within 31 bits
size_t gated_fwd_workspace(long long M, int F, int K);
bool gated_fwd_copy_pays(long long M, int F, int K);
size_t gated_bwd_workspace(long long M, int F, int K);
// The operands of a gated product copied to 16-byte boundaries in `workspace`, and p changed to them.
hipError_t gated_fwd_copy(DenseArgs *p, void *workspace, hipStream_t st);
hipError_t launch_gated_bwd(const GatedBackArgs &p, int type, hipStream_t st);

}  // namespace xnor
