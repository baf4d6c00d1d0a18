// Products of few tokens with 4-bit weights (a decoding step): the weights are read once, and that is what they take.
//
// A workgroup has 16 rows of the weights (of each matrix in the gated block), its eight waves an eighth of the contraction each (or four a quarter), whose sums are added
// in LDS.  A step is 128 values, 64 bytes of a row: lane (r, g) loads 16 bytes, row r's values 32 g .. 32 g + 31, and two exchanges across the wave
// turn the four words of the four lanes of a row about, so that instruction i takes the values 32 i .. 32 i + 31, which have one scale.
// A group's sum is multiplied by its scale in fp32: the weights are never rounded.  Some steps' loads are on their way together, behind no branch; their
// scales and zero points come with one load each, and reach the lanes that need them through LDS.
// (GPU time, bf16, weights in the last-level cache and from memory: 1 x 4096 x 4096 5.7 and 7.3 us, a launch and two loads' latencies; gated 1 x 4096 x 8192 in groups of 64
// with zero points 14.0-14.9 and 15.6 us, 2.4 TB/s: 70 vector instructions a step and matrix are about 7 us of it, and a wave has one step of loads on its way.  16, 32 and
// 64 x 8192 x 8192 17.6, 24.7 and 39.0 us, whose tokens each workgroup reads again.)
#include <algorithm>
#include <cstddef>

#include "int4_common.hpp"

namespace xnor {
namespace {

constexpr int kValues = 128;
constexpr int kMostGroups = 4;          // whose scales a wave holds at a time: one a lane

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

// A wave's scales and zero points of some groups' 16 rows.  (Scales are read four at a time.)
struct alignas(16) Held {
    float scale[kMostGroups * 16];
    uint32_t zero[kMostGroups * 16];
};
static_assert(sizeof(Held) % 16 == 0 && offsetof(Held, scale) % 16 == 0, "");

// What a wave multiplies.
template <class T, int MATS, int TT>
struct Span {
    Int4View view[MATS];
    const uint32_t *w[MATS];        // the lane's row
    const T *x[TT];                 // the lane's token (or another's, where there is none)
    int row[MATS];                  // the lane's
    int N, K, groups, scale_type;
    Held *held;                     // [MATS]
};

// U steps as they are loaded.
template <int MATS, int TT, int U>
struct Stage {
    uint32_t w[MATS][U][4];
    uint16_t low[MATS], high[MATS];     // halves of a scale (16-bit ones: both the same)
    uint8_t zero[MATS];
    i32x4 x[U][4][TT];
};
// (Four tiles of tokens are loaded where they are used: there are no registers for them.)
template <int TT> constexpr bool kEarly = TT < 4;

template <class T, int MATS, int TT, int U, bool WHOLE>
__device__ inline void load_x(const Span<T, MATS, TT> &p, int s, int u, Stage<MATS, TT, U> &to)
{
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int j = 0; j < TT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int from = (s + u) * kValues + i * 32 + g * 8;
            if constexpr (WHOLE) __builtin_memcpy(&to.x[u][i][j], p.x[j] + from, 16);
            else to.x[u][i][j] = load_end(p.x[j], from, p.K);
        }
}

// U steps from s on.  WHOLE: all of their values are there.
template <class T, int MATS, int TT, int GROUPS, int U, bool WHOLE>
__device__ inline void load_stage(const Span<T, MATS, TT> &p, int s, Stage<MATS, TT, U> &to)
{
    static_assert(U * GROUPS <= kMostGroups, "");
    const int lane = threadIdx.x & 63, g = lane >> 4;
    // group lane / 16's of row lane % 16; no branch by the scales' type or for want of zero points
    const long long group = (long long)min(s * GROUPS + min(g, U * GROUPS - 1), p.groups - 1) * p.N;
    const bool wide = p.scale_type == XNOR_TYPE_FP32;
#pragma unroll
    for (int k = 0; k < MATS; ++k) {
        const long long at = group + p.row[k];
        const uint16_t *const scale = (const uint16_t *)p.view[k].scale + (wide ? 2 * at : at);
        to.low[k] = scale[0], to.high[k] = scale[wide ? 1 : 0];
        to.zero[k] = *(p.view[k].zero ? p.view[k].zero + at : (const uint8_t *)scale);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < MATS; ++k) {
            if constexpr (WHOLE) {
                __builtin_memcpy(to.w[k][u], p.w[k] + (s + u) * (kValues / 8) + g * 4, 16);
            } else {
                // (words behind the last one: any levels, as the tokens' values are zeros there)
#pragma unroll
                for (int i = 0; i < 4; ++i) to.w[k][u][i] = p.w[k][min((s + u) * (kValues / 8) + g * 4 + i, (p.K - 1) / 8)];
            }
        }
    if constexpr (kEarly<TT>)
#pragma unroll
        for (int u = 0; u < U; ++u) load_x<T, MATS, TT, U, WHOLE>(p, s, u, to);
}

template <class T, int MATS, int TT, int GROUPS, int U, bool WHOLE>
__device__ inline void use_stage(const Span<T, MATS, TT> &p, int s, Stage<MATS, TT, U> &from, f32x4 (&acc)[MATS][TT])
{
    typedef Mat<T> Mul;
    typedef Levels<T> Level;
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int k = 0; k < MATS; ++k) {
        const uint32_t bits = p.scale_type == XNOR_TYPE_FP32 ? (uint32_t)from.high[k] << 16 | from.low[k] : (uint32_t)from.low[k] << 16;
        const float half = (float)__builtin_bit_cast(f16_t, from.low[k]);
        p.held[k].scale[lane] = (p.scale_type == XNOR_TYPE_F16 ? half : __uint_as_float(bits)) * Level::kBack;
        p.held[k].zero[lane] = p.view[k].zero ? from.zero[k] & 15u : 8u;
    }
    // (a wave's own: its LDS instructions come in order)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if constexpr (!kEarly<TT>) load_x<T, MATS, TT, U, WHOLE>(p, s, u, from);
#pragma unroll
        for (int k = 0; k < MATS; ++k) {
            turn_about(from.w[k][u]);
#pragma unroll
            for (int i = 0; i < GROUPS; ++i) {
                const int of = u * GROUPS + i;
                const typename Level::Zero z = Level::zero(p.held[k].zero[of * 16 + r]);
                const f32x4 by = *(const f32x4 *)&p.held[k].scale[of * 16 + g * 4];
                f32x4 part[TT] = {};
#pragma unroll
                for (int q = i * (4 / GROUPS); q < (i + 1) * (4 / GROUPS); ++q) {
                    const i32x4 levels = Level::operand(from.w[k][u][q], z);
#pragma unroll
                    for (int j = 0; j < TT; ++j) part[j] = Mul::mul(levels, from.x[u][q][j], part[j]);
                }
#pragma unroll
                for (int j = 0; j < TT; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[k][j][e] += by[e] * part[j][e];
            }
            __builtin_amdgcn_sched_barrier(0);          // (all groups' operands at a time would not fit the registers)
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Steps from .. to - 1, U at a time: those of the next time are on their way while these are used, loaded in straight lines of code (behind a branch the wait
// for one would be a wait for both).
template <class T, int MATS, int TT, int GROUPS, int U>
__device__ inline void accumulate(const Span<T, MATS, TT> &p, int from, int to, f32x4 (&acc)[MATS][TT])
{
#pragma unroll
    for (int k = 0; k < MATS; ++k)
#pragma unroll
        for (int j = 0; j < TT; ++j) acc[k][j] = f32x4{};
    const int whole = min(to, p.K / kValues);
    int s = from;
    if (s + U <= whole) {
        Stage<MATS, TT, U> a, b;
        load_stage<T, MATS, TT, GROUPS, U, true>(p, s, a);
        for (; s + 3 * U <= whole; s += 2 * U) {
            load_stage<T, MATS, TT, GROUPS, U, true>(p, s + U, b);
            use_stage<T, MATS, TT, GROUPS, U, true>(p, s, a, acc);
            load_stage<T, MATS, TT, GROUPS, U, true>(p, s + 2 * U, a);
            use_stage<T, MATS, TT, GROUPS, U, true>(p, s + U, b, acc);
        }
        if (s + 2 * U <= whole) {
            load_stage<T, MATS, TT, GROUPS, U, true>(p, s + U, b);
            use_stage<T, MATS, TT, GROUPS, U, true>(p, s, a, acc);
            use_stage<T, MATS, TT, GROUPS, U, true>(p, s + U, b, acc);
            s += 2 * U;
        } else {
            use_stage<T, MATS, TT, GROUPS, U, true>(p, s, a, acc);
            s += U;
        }
    }
    if constexpr (U > 1)
        for (; s < whole; ++s) {
            Stage<MATS, TT, 1> a;
            load_stage<T, MATS, TT, GROUPS, 1, true>(p, s, a);
            use_stage<T, MATS, TT, GROUPS, 1, true>(p, s, a, acc);
        }
    if (s < to) {
        Stage<MATS, TT, 1> a;
        load_stage<T, MATS, TT, GROUPS, 1, false>(p, s, a);
        use_stage<T, MATS, TT, GROUPS, 1, false>(p, s, a, acc);
    }
}

// The first of a workgroup's `rows` rows: the last workgroup's are the matrix's last ones, some of them another's too, which come out alike.
__device__ inline int first_row(int block, int rows, int N) { return max(0, min(block * rows, N - rows)); }

// TT: tiles of 16 tokens.  GROUPS: of a step.  MATS: 2: the gated block's matrices, or two times 16 rows of one, which share the tokens' values (from
// five tokens on these are most of what is read).
template <class T, bool GATED, int TT, int GROUPS, int WAVES, int MATS>
__global__ __launch_bounds__(WAVES * kWave, TT == 1 ? 4 : 2) void int4_few_kernel(const Int4Args p)
{
    static_assert(!GATED || MATS == 2, "");
    constexpr int ROWS = GATED ? 16 : 16 * MATS;
    // Tokens in terms: the tiles of 16 columns hold one term after the other of `own` tiles of tokens (of three terms in four, the last one's twice).
    constexpr bool TERMS = !GATED && TT > 1 && std::is_same<T, bf16_t>::value;
    const int own = !TERMS || p.terms == 0 ? TT : p.terms == 2 ? TT / 2 : 1;
    __shared__ f32x4 sums[WAVES][MATS][TT][kWave];
    __shared__ Held held[WAVES][MATS];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), r = lane & 15, g = lane >> 4;
    const int n0 = first_row(blockIdx.x, ROWS, p.N);

    Span<T, MATS, TT> span;
#pragma unroll
    for (int k = 0; k < MATS; ++k) span.view[k] = GATED && k ? p.w2 : p.w;
    long long m0 = (p.first + blockIdx.y) * (16 * TT);
    int count = (int)min(p.M - m0, 16LL * TT);
    int expert = -1;
    if (p.pairs) {
        m0 = p.first + blockIdx.y, count = 1;
        expert = p.pairs[m0];
        if (expert < 0 || expert >= p.E) return;
    } else if (p.tiles) {
        const long long at = p.first + blockIdx.y;
        if constexpr (TERMS) {
            const int cut = (int)(at % p.cuts) * 16 * own;
            if (at / p.cuts >= p.tiles[0].count) return;
            const ExpertTile tile = p.tiles[1 + at / p.cuts];
            m0 = tile.first + cut, count = min(tile.count - cut, 16 * own), expert = tile.expert;
            if (count <= 0) return;
        } else {
            if (at >= p.tiles[0].count) return;
            const ExpertTile tile = p.tiles[1 + at];
            m0 = tile.first, count = tile.count, expert = tile.expert;
        }
    }
#pragma unroll
    for (int k = 0; k < MATS; ++k) {
        if (expert >= 0) span.view[k] = of_stack(span.view[k], p, expert);
        span.row[k] = min(n0 + (GATED ? 0 : 16 * k) + r, p.N - 1);
        span.w[k] = (const uint32_t *)(span.view[k].q + span.row[k] * p.ldq);
    }
#pragma unroll
    for (int j = 0; j < TT; ++j) {
        const long long m = m0 + min((TERMS ? j & (own - 1) : j) * 16 + r, count - 1);
        const long long from = p.pairs ? m / p.chosen : p.order_x ? p.order_x[m] / p.chosen : m;
        span.x[j] = (const T *)((const char *)p.x + from * p.ldx) + (TERMS && p.terms ? (long long)min(j / own, p.terms - 1) * hidden_stride(p.K) : 0);
    }
    span.N = p.N, span.K = p.K, span.groups = (p.K + p.group - 1) / p.group, span.scale_type = p.scale_type, span.held = held[wave];

    const int steps = (p.K + kValues - 1) / kValues;
    f32x4 acc[MATS][TT];
    accumulate<T, MATS, TT, GROUPS, (MATS == 2 || TT > 1 || GROUPS == 4 ? 1 : 2)>(span, steps * wave / WAVES, steps * (wave + 1) / WAVES, acc);
    if constexpr (TERMS) {
#pragma unroll
        for (int k = 0; k < MATS; ++k) {
            if (p.terms == 2) {
#pragma unroll
                for (int j = 0; j < TT / 2; ++j) acc[k][j] += acc[k][j + TT / 2];
            } else if (TT == 4 && p.terms == 3) {
                acc[k][0] += acc[k][1] + acc[k][TT / 2];
            }
        }
    }
#pragma unroll
    for (int k = 0; k < MATS; ++k)
#pragma unroll
        for (int j = 0; j < TT; ++j) sums[wave][k][j][lane] = acc[k][j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < TT; ++j) {
        if (wave != j % WAVES || j * 16 + r >= count) continue;       // (a wave a tile of tokens)
        f32x4 v[MATS];
#pragma unroll
        for (int k = 0; k < MATS; ++k) {
            v[k] = sums[0][k][j][lane];
#pragma unroll
            for (int i = 1; i < WAVES; ++i) v[k] += sums[i][k][j][lane];
        }
        const long long m = m0 + j * 16 + r, to = p.order_out ? p.order_out[m] : m;
#pragma unroll
        for (int k = 0; k < (GATED ? 1 : MATS); ++k) {
            const int n = n0 + 16 * k + g * 4;
            if (n >= p.N) continue;
            float out[4], bias[4];
            load_params(p.bias, n, p.N, 0.f, bias);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (GATED) out[e] = gate(p.act, p.out_type != XNOR_TYPE_FP32, v[0][e]) * v[1][e];
                else out[e] = p.bias ? v[k][e] + bias[e] : v[k][e];
            }
            if (GATED && p.out_terms) store_terms(p, to, n, out);
            else store_outputs(p, to, n, out);
        }
    }
}

template <class T, bool GATED, int TT, int WAVES, int MATS>
hipError_t few_of(const Int4Args &p, hipStream_t st)
{
    constexpr long long kMost = 32768;          // tiles of tokens in a launch
    const int TM = 16 * TT, own = p.terms == 0 ? TM : p.terms == 2 ? TM / 2 : 16, cuts = p.tiles ? std::max(1, p.tile / own) : 1;
    const long long tiles = p.pairs ? p.M : p.tiles ? most_tiles(p.M, p.E, p.tile) * cuts : (p.M + TM - 1) / TM;
    const long long each = std::max<long long>(1, std::min<long long>(kMost, kMaxBlocks / ceil_div(p.N, GATED ? 16 : 16 * MATS)));
    for (long long m = 0; m < tiles; m += each) {
        Int4Args q = p;
        q.first = m, q.cuts = cuts;
        const dim3 grid((unsigned)ceil_div(p.N, GATED ? 16 : 16 * MATS), (unsigned)std::min(each, tiles - m)), block(WAVES * kWave);
        if (p.group == 128) int4_few_kernel<T, GATED, TT, 1, WAVES, MATS><<<grid, block, 0, st>>>(q);
        else if (p.group == 64) int4_few_kernel<T, GATED, TT, 2, WAVES, MATS><<<grid, block, 0, st>>>(q);
        else int4_few_kernel<T, GATED, TT, 4, WAVES, MATS><<<grid, block, 0, st>>>(q);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class T, bool GATED, int TT>
hipError_t few(const Int4Args &p, hipStream_t st)
{
    // Four waves where there is a workgroup for each unit (24 tokens to 3 of 30 experts, 1100 x 777, in groups of 32, hidden values in f16: 16.9 and 13.4 us, with eight 19.9
    // and 16.0; 1 x 4096 x 4096 6.1 and 6.0), eight where there are fewer
    const long long tiles = p.pairs || p.tiles ? p.M : (p.M + 16 * TT - 1) / (16 * TT);
    // (and of one matrix twice 16 rows where that leaves a workgroup a unit: 64 x 8192 x 8192 41 us, by 16 rows 67, x 4096 x 4096 21.8 and 20.4)
    const long long units = compute_units();
    if constexpr (!GATED)
        if (!p.pairs && (TT > 1 || (p.tiles ? p.tile : p.M) > 4) && tiles * ceil_div(p.N, 32) >= units) return tiles * ceil_div(p.N, 32) >= 2 * units ? few_of<T, GATED, TT, 4, 2>(p, st) : few_of<T, GATED, TT, 8, 2>(p, st);
    constexpr int MATS = GATED ? 2 : 1;
    return tiles * ceil_div(p.N, 16) >= units * (TT == 1 ? 1 : 2) ? few_of<T, GATED, TT, 4, MATS>(p, st) : few_of<T, GATED, TT, 8, MATS>(p, st);
}

template <class T, bool GATED>
hipError_t few_by_tokens(const Int4Args &p, hipStream_t st)
{
    if constexpr (!GATED)
        if (p.terms) return p.terms == 2 && p.tile <= 16 ? few<T, GATED, 2>(p, st) : few<T, GATED, 4>(p, st);
    const long long each = p.pairs ? 1 : p.tiles ? p.tile : p.M;
    return each <= 16 ? few<T, GATED, 1>(p, st) : each <= 32 ? few<T, GATED, 2>(p, st) : few<T, GATED, 4>(p, st);
}

// ---- a token's experts' second products and their sum -------------------------------------------------------------------
// A workgroup has 16 rows of every chosen expert's matrix for one token; a wave has a share of the contraction of one of them, or of several in turn.
// The matrix instruction's columns, which would all be the one token, are its terms: they cost nothing.
// Sums are multiplied by their slot's weight before they are added, slots in order within a wave, then the waves'.

constexpr int kDownWaves = 16;

template <int GROUPS>
__global__ __launch_bounds__(kDownWaves * kWave) void int4_down_kernel(const Int4Args p, const float *weights, int shares)
{
    typedef bf16_t T;
    __shared__ f32x4 sums[kDownWaves][4][kMostTerms];
    __shared__ Held held[kDownWaves];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), r = lane & 15, g = lane >> 4;
    const int n0 = first_row(blockIdx.x, 16, p.N), row = min(n0 + r, p.N - 1);
    const long long token = p.first + blockIdx.y;
    const int steps = (p.K + kValues - 1) / kValues;
    f32x4 sum = {};
    float none = 0.f;           // of slots without an expert: weight * 0
    for (int item = wave; item < p.chosen * shares; item += kDownWaves) {
        const int slot = item / shares, part = item % shares;
        const long long m = token * p.chosen + slot;
        const int expert = __builtin_amdgcn_readfirstlane(p.pairs[m]);
        const float weight = weights[m];
        if (expert < 0 || expert >= p.E) {
            none += weight * 0.f;
            continue;
        }
        Span<T, 1, 1> span;
        span.view[0] = of_stack(p.w, p, expert);
        span.w[0] = (const uint32_t *)(span.view[0].q + row * p.ldq);
        span.x[0] = (const T *)((const char *)p.x + m * p.ldx) + (long long)min(r, p.terms - 1) * hidden_stride(p.K);
        span.row[0] = row, span.N = p.N, span.K = p.K, span.groups = (p.K + p.group - 1) / p.group, span.scale_type = p.scale_type, span.held = &held[wave];
        f32x4 acc[1][1];
        accumulate<T, 1, 1, GROUPS, (GROUPS == 4 ? 1 : 2)>(span, steps * part / shares, steps * (part + 1) / shares, acc);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += weight * acc[0][0][e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] += none;
    if (r < kMostTerms) sums[wave][g][r] = sum;
    __syncthreads();
    const int n = n0 + t * 4;
    if (t >= 4 || n >= p.N) return;
    float out[4] = {};
#pragma unroll
    for (int w = 0; w < kDownWaves; ++w)
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] += p.terms == 2 ? sums[w][t][0][e] + sums[w][t][1][e] : sums[w][t][0][e] + (sums[w][t][1][e] + sums[w][t][2][e]);
    store_outputs(p, token, n, out);
}

hipError_t down(const Int4Args &p, const float *weights, hipStream_t st)
{
    const int shares = std::max(1, kDownWaves / p.chosen);
    constexpr long long kMost = 32768;
    const long long each = std::max<long long>(1, std::min<long long>(kMost, kMaxBlocks / 2 / ceil_div(p.N, 16)));
    for (long long m = 0; m < p.M; m += each) {
        Int4Args q = p;
        q.first = m;
        const dim3 grid((unsigned)ceil_div(p.N, 16), (unsigned)std::min(each, p.M - m)), block(kDownWaves * kWave);
        if (p.group == 128) int4_down_kernel<1><<<grid, block, 0, st>>>(q, weights, shares);
        else if (p.group == 64) int4_down_kernel<2><<<grid, block, 0, st>>>(q, weights, shares);
        else int4_down_kernel<4><<<grid, block, 0, st>>>(q, weights, shares);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_int4_few(const Int4Args &p, int type, bool gated, hipStream_t st)
{
    if (p.M == 0) return hipSuccess;
    if (type == XNOR_TYPE_F16) return gated ? few_by_tokens<f16_t, true>(p, st) : few_by_tokens<f16_t, false>(p, st);
    return gated ? few_by_tokens<bf16_t, true>(p, st) : few_by_tokens<bf16_t, false>(p, st);
}

hipError_t launch_int4_down(const Int4Args &p, const float *weights, hipStream_t st) { return down(p, weights, st); }

hipError_t launch_int4(const Int4Args &p, int type, bool gated, hipStream_t st)
{
    const bool many = p.tiles ? p.tile > kInt4Few : !p.pairs && int4_many(p.M, p.N, p.K, gated, p.parts) && int4_tiles_support(p);
    return many ? launch_int4_tiles(p, type, gated, st) : launch_int4_few(p, type, gated, st);
}

}  // namespace xnor
