// Products of few tokens with 4-bit weights (a decoding step): the weights are read once, and that is what they take.
//
// A workgroup has 16 rows of the weights (of each matrix in the gated block), its eight waves an eighth of the contraction each, whose sums are added
// in LDS.  A step is 128 values, 64 bytes of a row: lane (r, g) loads 16 bytes, row r's values 32 g .. 32 g + 31, and two exchanges across the wave
// turn the four words of the four lanes of a row about, so that instruction i takes the values 32 i .. 32 i + 31, which have one scale.
// A group's sum is multiplied by its scale in fp32: the weights are never rounded.
#include <algorithm>

#include "int4_common.hpp"

namespace xnor {
namespace {

constexpr int kWaves = 8, kThreads = kWaves * kWave, kValues = 128;

// d[i] of the 16 lanes g to d[g] of the 16 lanes i.
__device__ inline void turn_about(uint32_t (&d)[4])
{
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const auto v = __builtin_amdgcn_permlane32_swap(d[i], d[i + 2], false, false);
        d[i] = v[0], d[i + 2] = v[1];
    }
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        const auto v = __builtin_amdgcn_permlane16_swap(d[i], d[i + 1], false, false);
        d[i] = v[0], d[i + 1] = v[1];
    }
#endif
}

// TT: tiles of 16 tokens.  GROUPS: of a step.
template <class T, bool GATED, int TT, int GROUPS>
__global__ __launch_bounds__(kThreads) void int4_few_kernel(const Int4Args p)
{
    // U: steps whose weights are on their way together
    constexpr int MATS = GATED ? 2 : 1, U = GATED || TT == 4 || GROUPS == 4 ? 2 : 4;
    typedef Mat<T> Mul;
    typedef Levels<T> Level;
    __shared__ f32x4 sums[kWaves][MATS][TT][kWave];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), r = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16;

    Int4View view[MATS];
    view[0] = p.w;
    if constexpr (GATED) view[1] = p.w2;
    long long m0 = (p.first + blockIdx.y) * (16 * TT);
    int count = (int)min(p.M - m0, 16LL * TT);
    if (p.offsets) {
        ExpertTile tile;
        if (!expert_tile(p.offsets, p.E, 16 * TT, p.first + blockIdx.y, &tile)) return;
        m0 = tile.first, count = tile.count;
#pragma unroll
        for (int k = 0; k < MATS; ++k) view[k] = of_stack(view[k], p, tile.expert);
    }

    const int steps = (p.K + kValues - 1) / kValues, share = (steps + kWaves - 1) / kWaves, words = (p.K + 7) / 8;
    const int from = wave * share, to = min(steps, from + share);
    const int groups = (p.K + p.group - 1) / p.group;
    const int row = min(n0 + r, p.N - 1);
    const uint32_t *w[MATS];
#pragma unroll
    for (int k = 0; k < MATS; ++k) w[k] = (const uint32_t *)(view[k].q + row * p.ldq);
    const T *x[TT];
#pragma unroll
    for (int j = 0; j < TT; ++j) {
        const long long m = m0 + min(j * 16 + r, count - 1);
        x[j] = (const T *)((const char *)p.x + (p.order_x ? p.order_x[m] / p.chosen : m) * p.ldx);
    }

    auto accumulate = [&](f32x4 (&acc)[MATS][TT], auto exact) __attribute__((always_inline)) {
        constexpr bool EXACT = decltype(exact)::value;
#pragma unroll
        for (int k = 0; k < MATS; ++k)
#pragma unroll
            for (int j = 0; j < TT; ++j) acc[k][j] = f32x4{};
        for (int s = from; s < to; s += U) {
            uint32_t held[MATS][U][4];
            float scale[MATS][U][GROUPS][4];
            uint32_t zero[MATS][U][GROUPS];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < MATS; ++k) {
                    if (s + u >= to) continue;
                    const Chunk<uint32_t> c = load_chunk(w[k], (s + u) * (kValues / 8) + g * 4, words);
#pragma unroll
                    for (int i = 0; i < 4; ++i) held[k][u][i] = c.v[i];
#pragma unroll
                    for (int i = 0; i < GROUPS; ++i) {
                        const long long at = min((s + u) * GROUPS + i, groups - 1);
                        load_scales(view[k], p.scale_type, at, n0 + g * 4, p.N, scale[k][u][i]);
                        zero[k][u][i] = view[k].zero ? view[k].zero[at * p.N + row] & 15u : 8u;
                    }
                }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (s + u >= to) continue;
                i32x4 vx[4][TT];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < TT; ++j) vx[i][j] = __builtin_bit_cast(i32x4, load_chunk(x[j], (s + u) * kValues + i * 32 + g * 8, p.K));
#pragma unroll
                for (int k = 0; k < MATS; ++k) {
                    turn_about(held[k][u]);
#pragma unroll
                    for (int i = 0; i < GROUPS; ++i) {
                        const typename Level::Zero z = Level::zero(zero[k][u][i]);
                        f32x4 part[TT] = {};
#pragma unroll
                        for (int q = i * (4 / GROUPS); q < (i + 1) * (4 / GROUPS); ++q) {
                            const i32x4 levels = Level::template operand<EXACT>(held[k][u][q], z);
#pragma unroll
                            for (int j = 0; j < TT; ++j) {
                                part[j] = Mul::mul(levels, vx[q][j], part[j]);
                                if constexpr (Level::kOffset && !EXACT) part[j] = Mul::mul(Level::offset(z), vx[q][j], part[j]);
                            }
                        }
#pragma unroll
                        for (int j = 0; j < TT; ++j)
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[k][j][e] += (EXACT && Level::kOffset ? scale[k][u][i][e] * 0x1p16f : scale[k][u][i][e]) * part[j][e];
                    }
                }
            }
        }
    };
    f32x4 acc[MATS][TT];
    accumulate(acc, std::false_type{});
    if constexpr (Level::kOffset) {
        auto is_odd = [](float v) { return !(fabsf(v) <= 3.402823466e38f); };
        bool odd = false;
#pragma unroll
        for (int k = 0; k < MATS; ++k)
#pragma unroll
            for (int j = 0; j < TT; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) odd |= is_odd(acc[k][j][e]);
        if (__any(odd)) {
            f32x4 exact[MATS][TT];
            accumulate(exact, std::true_type{});
#pragma unroll
            for (int k = 0; k < MATS; ++k)
#pragma unroll
                for (int j = 0; j < TT; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (is_odd(acc[k][j][e])) acc[k][j][e] = exact[k][j][e];
        }
    }
#pragma unroll
    for (int k = 0; k < MATS; ++k)
#pragma unroll
        for (int j = 0; j < TT; ++j) sums[wave][k][j][lane] = acc[k][j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < TT; ++j) {
        const int n = n0 + g * 4;
        if (wave != j % kWaves || j * 16 + r >= count || n >= p.N) continue;       // (a wave a tile of tokens)
        f32x4 v[MATS];
#pragma unroll
        for (int k = 0; k < MATS; ++k) {
            v[k] = sums[0][k][j][lane];
#pragma unroll
            for (int i = 1; i < kWaves; ++i) v[k] += sums[i][k][j][lane];
        }
        float out[4], bias[4];
        load_params(p.bias, n, p.N, 0.f, bias);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (GATED) out[e] = gate(p.act, p.out_type != XNOR_TYPE_FP32, v[0][e]) * v[1][e];
            else out[e] = p.bias ? v[0][e] + bias[e] : v[0][e];
        }
        const long long m = m0 + j * 16 + r;
        store_outputs(p, p.order_out ? p.order_out[m] : m, n, out);
    }
}

template <class T, bool GATED, int TT>
hipError_t few(const Int4Args &p, hipStream_t st)
{
    constexpr long long kMost = 32768;          // tiles of tokens in a launch
    const int TM = 16 * TT;
    const long long tiles = p.offsets ? std::min<long long>(p.E, p.M) + p.M / TM : (p.M + TM - 1) / TM;
    const long long each = std::max<long long>(1, std::min<long long>(kMost, kMaxBlocks / ceil_div(p.N, 16)));
    for (long long m = 0; m < tiles; m += each) {
        Int4Args q = p;
        q.first = m;
        const dim3 grid((unsigned)ceil_div(p.N, 16), (unsigned)std::min(each, tiles - m)), block(kThreads);
        if (p.group == 128) int4_few_kernel<T, GATED, TT, 1><<<grid, block, 0, st>>>(q);
        else if (p.group == 64) int4_few_kernel<T, GATED, TT, 2><<<grid, block, 0, st>>>(q);
        else int4_few_kernel<T, GATED, TT, 4><<<grid, block, 0, st>>>(q);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class T, bool GATED>
hipError_t few_by_tokens(const Int4Args &p, hipStream_t st)
{
    const long long each = p.offsets ? (p.M + p.E - 1) / p.E : p.M;
    return each <= 16 ? few<T, GATED, 1>(p, st) : each <= 32 ? few<T, GATED, 2>(p, st) : few<T, GATED, 4>(p, st);
}

}  // namespace

hipError_t launch_int4_few(const Int4Args &p, int type, bool gated, hipStream_t st)
{
    if (p.M == 0) return hipSuccess;
    if (type == XNOR_TYPE_F16) return gated ? few_by_tokens<f16_t, true>(p, st) : few_by_tokens<f16_t, false>(p, st);
    return gated ? few_by_tokens<bf16_t, true>(p, st) : few_by_tokens<bf16_t, false>(p, st);
}

hipError_t launch_int4(const Int4Args &p, int type, bool gated, hipStream_t st)
{
    const long long each = p.offsets ? p.M / p.E : p.M;
    return each > 64 ? launch_int4_tiles(p, type, gated, st) : launch_int4_few(p, type, gated, st);
}

}  // namespace xnor
