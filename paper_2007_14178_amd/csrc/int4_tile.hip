// Products of many tokens with 4-bit weights: 128 or 256 tokens x 128 rows of the weights (gated: 64 of each matrix) by four or eight waves of 64 x 64.
//
// Tokens and weights go through registers into LDS, 64 values of a row at a time, the weights as levels less their zero point, which the tokens' type
// holds exactly; a step's sums (of groups of 32: of each half) are multiplied by their scales in fp32 and added.  Two steps' rows are on their way, a step's are
// turned into operands and written to one half of LDS while the other is multiplied.
// Bound by the operands' way out of LDS, 64 KB a step of 128 x 128: without those reads 4096 x 8192 x 4096 bf16 takes 185 us of 335, without the conversions 290.
// 4096 x 8192 x 8192 bf16 640-755 us, 0.73-0.86 PFLOP/s.  With weights rounded to the tokens' type on their way, (level - zero) * scale, there are no scales to
// multiply by and it takes 560-640, but outputs are up to 1.6 times as far from the exact ones as those of products in fp32.
#include <algorithm>
#include <cmath>

#include "int4_common.hpp"

namespace xnor {
namespace {

constexpr int kRows = 128, kDeep = 64;       // rows of the weights a tile, values of a step

// Loads from a buffer: a lane's offset and a scalar one.  (The host's pass does not know the builtins.)
typedef int i32x2 __attribute__((ext_vector_type(2)));
__device__ inline auto buffer(const void *p, int size) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, size, 0x00027000); }
#ifdef __HIP_DEVICE_COMPILE__
template <class R> __device__ inline i32x4 load_16(R r, int at, int from) { return __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at, from, 0)); }
template <class R> __device__ inline i32x2 load_8(R r, int at, int from) { return __builtin_bit_cast(i32x2, __builtin_amdgcn_raw_buffer_load_b64(r, at, from, 0)); }
template <class R> __device__ inline uint32_t load_4(R r, int at, int from) { return __builtin_amdgcn_raw_buffer_load_b32(r, at, from, 0); }
template <class R> __device__ inline uint16_t load_2(R r, int at, int from) { return __builtin_amdgcn_raw_buffer_load_b16(r, at, from, 0); }
template <class R> __device__ inline uint8_t load_1(R r, int at, int from) { return __builtin_amdgcn_raw_buffer_load_b8(r, at, from, 0); }
#else
template <class R> __device__ inline i32x4 load_16(R, int, int) { return {}; }
template <class R> __device__ inline i32x2 load_8(R, int, int) { return {}; }
template <class R> __device__ inline uint32_t load_4(R, int, int) { return 0; }
template <class R> __device__ inline uint16_t load_2(R, int, int) { return 0; }
template <class R> __device__ inline uint8_t load_1(R, int, int) { return 0; }
#endif

// SHORT: groups of 32, two of them in a step.
// TERMS: 2 or 3: a token is the sum of so many rows, which stand in a wave's tiles of 16 one term after the other (of three in four, the last one's twice,
// which is not multiplied) and are added where they are multiplied: a workgroup has the tokens that its TM rows make.  (32768 pairs of 64 experts, 1024 hidden values to 2048
// outputs, two terms, 256 rows: 546 us; one term, 128 rows: 347.)
template <class T, bool GATED, bool SHORT, int TM, int TERMS>
__global__ __launch_bounds__(2 * TM, 2) void int4_tile_kernel(const Int4Args p, int tiles_n, long long tiles)
{
    constexpr int TN = GATED ? 64 : 128;        // outputs n of a tile
    constexpr int OWN = TERMS == 0 ? 4 : TERMS == 2 ? 2 : 1, TOKENS = TM / 4 * OWN;         // a wave's tiles of tokens, and the workgroup's tokens
    constexpr int kThreads = 2 * TM, A = 4, B = 512 / kThreads;         // chunks of the tokens and word pairs of the weights that a thread stages
    typedef Mat<T> Mul;
    __shared__ __align__(16) char lds[2][(TM + kRows) * kStep];
    __shared__ __align__(16) float by[2][2][kRows];         // a step's scales, of its first and its second 32 values
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    // Workgroups go round the eight XCDs by their index: each takes a run of consecutive tiles, groups of eight tiles of tokens for a tile of the
    // weights' rows, so that what its units work on at a time shares both in its L2.  (Experts: of the tiles that there are.)
    if (p.tiles) tiles = min(tiles, ((long long)p.tiles[0].count * (TERMS ? p.cuts : 1) - p.first) * tiles_n);
    const long long eighth = (tiles + 7) >> 3, index = (blockIdx.x & 7) * eighth + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= eighth || index >= tiles) return;
    const int rows = (int)(tiles / tiles_n), group8 = (int)(index / (8 * tiles_n)), in = (int)(index - (long long)group8 * 8 * tiles_n);
    const int high = min(8, rows - group8 * 8);
    const int tn = __builtin_amdgcn_readfirstlane(in / high), tm = __builtin_amdgcn_readfirstlane(group8 * 8 + in % high);
    const int n0 = tn * TN;
    Int4View view[2] = {p.w, GATED ? p.w2 : p.w};
    long long m0 = (p.first + tm) * TOKENS;
    int count = (int)min(p.M - m0, (long long)TOKENS);
    if (p.tiles) {
        const long long at = p.first + tm;
        const int cut = TERMS ? (int)(at % p.cuts) * TOKENS : 0;
        const ExpertTile tile = p.tiles[1 + (TERMS ? at / p.cuts : at)];
        m0 = tile.first + cut, count = tile.count - cut;
        if (TERMS) {
            if (count <= 0) return;
            count = min(count, TOKENS);
        }
        view[0] = of_stack(view[0], p, tile.expert), view[1] = of_stack(view[1], p, tile.expert);
    }

    // Tokens: chunk `chunk` of rows t / 8 + TM / 4 i.  Weights: word pair `pair` (16 values) of rows t / 4 + TM / 2 i.  All through buffers, a lane's offsets staying as
    // they are and a step's a scalar.
    const int chunk = t & 7, pair = t & 3;
    const long long from_x = p.order_x ? 0 : m0 * p.ldx;
    const auto x = buffer((const char *)p.x + from_x, 0x7fffffff);
    int a[A];
#pragma unroll
    for (int i = 0; i < A; ++i) {
        const int r = (t >> 3) + TM / 4 * i, m = min(TERMS ? r / 64 * (16 * OWN) + r % (16 * OWN) : r, count - 1);
        a[i] = (int)((p.order_x ? p.order_x[m0 + m] / p.chosen : m) * p.ldx) + (TERMS ? min(r % 64 / (16 * OWN), TERMS - 1) * hidden_stride(p.K) * 2 : 0) + chunk * 16;
    }
    const int words = (p.K + 7) / 8, groups = (p.K + p.group - 1) / p.group, shift = __builtin_ctz(p.group);
    const bool has_zero = view[0].zero != nullptr, half = p.scale_type == XNOR_TYPE_F16;
    const bool wide = p.scale_type == XNOR_TYPE_FP32;
    const int scale_bytes = wide ? 4 : 2;
    // (a lane's matrix: in the gated block that of its row's 16; a wave's rows t / 4 are 16 of one)
    const bool second = GATED && (wave & 1);
    const Int4View &mine = second ? view[1] : view[0];
    const auto q = buffer(mine.q + (long long)n0 * p.ldq, 0x7fffffff);
    const auto scales = buffer(mine.scale, 0x7fffffff);
    const auto zeros = buffer(has_zero ? (const void *)mine.zero : mine.scale, 0x7fffffff);        // (loaded in any case: a branch would part the step)
    int b[B], of_scale[B], of_zero[B];
#pragma unroll
    for (int i = 0; i < B; ++i) {
        const int r = (t >> 2) + TM / 2 * i, row = min(GATED ? (r >> 5) * 16 + (r & 15) : r, p.N - 1 - n0);
        const int value = n0 + row + (SHORT ? (pair >> 1) * p.N : 0);
        b[i] = row * (int)p.ldq + pair * 8, of_scale[i] = value * scale_bytes, of_zero[i] = has_zero ? value : 0;
    }
    // Steps in the order that they are taken: one that the contraction ends inside comes first.
    // (parts: of the contraction's whole steps a share, the last one's after an end that is the first's.)
    const int all = p.K / kDeep, before = all * (int)blockIdx.y / p.parts;
    const int whole = all * ((int)blockIdx.y + 1) / p.parts - before, part = p.K % kDeep && blockIdx.y == 0 ? 1 : 0, steps = whole + part;

    // Two steps' rows are on their way.
    struct Rows {
        i32x4 a[A];
        i32x2 b[B];
        uint32_t low[B], high[B], zero[B];        // (halves of a scale, 16-bit ones twice) as they are loaded: a conversion beside the loads would wait for them
    };
    Rows held[2];
    auto fetch = [&](int s, Rows &to, auto ends) __attribute__((always_inline)) {
        const int deep = (decltype(ends)::value ? all : before + min(s - part, whole - 1)) * kDeep;      // (behind the last step: that one again)
        // weights first: at the tile's begin the tokens' rows are not known yet
        const int g = deep >> shift, back = decltype(ends)::value && SHORT && g + (pair >> 1) >= groups ? p.N : 0;
#pragma unroll
        for (int i = 0; i < B; ++i) {
            if constexpr (!decltype(ends)::value) {
                to.b[i] = load_8(q, b[i], deep / 2);
            } else {        // (levels behind the last one may be any)
#pragma unroll
                for (int j = 0; j < 2; ++j) to.b[i][j] = load_4(q, b[i] - pair * 8 + min(deep / 8 + pair * 2 + j, words - 1) * 4, 0);
            }
            to.low[i] = load_2(scales, of_scale[i] - back * scale_bytes, g * p.N * scale_bytes);
            to.high[i] = load_2(scales, of_scale[i] - back * scale_bytes + (wide ? 2 : 0), g * p.N * scale_bytes);
            to.zero[i] = load_1(zeros, has_zero ? of_zero[i] - back : 0, has_zero ? g * p.N : 0);
        }
        if constexpr (!decltype(ends)::value) {
#pragma unroll
            for (int i = 0; i < A; ++i) to.a[i] = load_16(x, a[i], deep * 2);
        } else {            // tokens' values there are zeros
#pragma unroll
            for (int i = 0; i < A; ++i) {
                const T *const row = (const T *)((const char *)p.x + from_x + (a[i] - chunk * 16));
                to.a[i] = load_end(row, deep + chunk * 8, p.K);
            }
        }
    };
    auto put = [&](int s, const Rows &from) __attribute__((always_inline)) {
        char *const la = lds[s & 1], *const lb = la + TM * kStep;
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const int r = (t >> 2) + TM / 2 * i;
            const float of_half = (float)__builtin_bit_cast(f16_t, (uint16_t)from.low[i]);
            const float scale = half ? of_half : __uint_as_float(wide ? from.high[i] << 16 | from.low[i] : from.low[i] << 16);
            by[s & 1][pair >> 1][r] = scale * Levels<T>::kBack;         // (pairs 0 and 1, 2 and 3 are of one group)
            const typename Levels<T>::Zero zero = Levels<T>::zero(has_zero ? from.zero[i] & 15u : 8u);
#pragma unroll
            for (int j = 0; j < 2; ++j) *(i32x4 *)(lb + r * kStep + (((pair * 2 + j) ^ (r & 7)) << 4)) = Levels<T>::operand(from.b[i][j], zero);
        }
#pragma unroll
        for (int i = 0; i < A; ++i) {
            const int r = (t >> 3) + TM / 4 * i;
            *(i32x4 *)(la + r * kStep + ((chunk ^ (r & 7)) << 4)) = from.a[i];
        }
    };

    const int wm = (TM == 256 ? wave & 3 : wave >> 1) * 64, wn = (TM == 256 ? wave >> 2 : wave & 1) * 64;
    const int own = wm / 4 * OWN;       // the wave's first token
    const bool busy = own < count;      // whether it has any
    f32x4 acc[4][OWN] = {};
    auto step = [&](int s, Rows &rows_of, auto more) __attribute__((always_inline)) {
        if (busy) {
            const char *const la = lds[s & 1], *const lb = la + TM * kStep;
            i32x4 fa[2][4], fb[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int c = h * 4 + (lane >> 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int ra = wm + i * 16 + (lane & 15), rb = wn + i * 16 + (lane & 15);
                    fa[h][i] = *(const i32x4 *)(la + ra * kStep + ((c ^ (ra & 7)) << 4));
                    fb[h][i] = *(const i32x4 *)(lb + rb * kStep + ((c ^ (rb & 7)) << 4));
                }
            }
            // (not for some steps alone: the wait for a step's rows would be one for all that are on their way)
            if constexpr (decltype(more)::value) put(s + 1, rows_of), fetch(s + 3, rows_of, std::false_type{});
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 first = *(const f32x4 *)&by[s & 1][0][wn + i * 16 + (lane >> 4) * 4];
                const f32x4 then = SHORT ? *(const f32x4 *)&by[s & 1][1][wn + i * 16 + (lane >> 4) * 4] : first;
#pragma unroll
                for (int j = 0; j < OWN; ++j) {
                    f32x4 sum = Mul::mul(fb[0][i], fa[0][j], f32x4{});
#pragma unroll
                    for (int of = 1; of < TERMS; ++of) sum = Mul::mul(fb[0][i], fa[0][j + of * OWN], sum);
                    if constexpr (SHORT) {
                        f32x4 more = Mul::mul(fb[1][i], fa[1][j], f32x4{});
#pragma unroll
                        for (int of = 1; of < TERMS; ++of) more = Mul::mul(fb[1][i], fa[1][j + of * OWN], more);
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j][e] += first[e] * sum[e] + then[e] * more[e];
                    } else {
                        sum = Mul::mul(fb[1][i], fa[1][j], sum);
#pragma unroll
                        for (int of = 1; of < TERMS; ++of) sum = Mul::mul(fb[1][i], fa[1][j + of * OWN], sum);
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j][e] += first[e] * sum[e];
                    }
                }
            }
        } else if constexpr (decltype(more)::value) {
            put(s + 1, rows_of), fetch(s + 3, rows_of, std::false_type{});
        }
        __builtin_amdgcn_sched_barrier(0);
        // (LDS alone is waited for: the fetches are not)
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    if (part) fetch(0, held[0], std::true_type{});
    else fetch(0, held[0], std::false_type{});
    if (whole > 0) {
        fetch(1, held[1], std::false_type{});
        put(0, held[0]);
        fetch(2, held[0], std::false_type{});
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
        int s = 0;
        for (; s + 1 < steps; s += 2) step(s, held[1], std::true_type{}), step(s + 1, held[0], std::true_type{});
        if (s < steps) step(s, held[1], std::false_type{});
    } else {
        put(0, held[0]);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
        step(0, held[1], std::false_type{});
    }
#pragma unroll
    for (int i = 0; i < 4; i += GATED ? 2 : 1) {
        const int n = n0 + (GATED ? wn / 2 + i * 8 : wn + i * 16) + (lane >> 4) * 4;
        if (n >= p.N) continue;
        float bias[4];
        load_params(p.bias, n, p.N, 0.f, bias);
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
            const int at = own + j * 16 + (lane & 15);
            if (at >= count) continue;
            if (p.parts > 1) {          // [part][matrix][M][N]
#pragma unroll
                for (int k = 0; k < (GATED ? 2 : 1); ++k) {
                    const float v[4] = {acc[i + k][j][0], acc[i + k][j][1], acc[i + k][j][2], acc[i + k][j][3]};
                    store_values(p.sums + (((long long)blockIdx.y * (GATED ? 2 : 1) + k) * p.M + m0 + at) * p.N, n, p.N, v);
                }
                continue;
            }
            float out[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (GATED) out[e] = gate(p.act, p.out_type != XNOR_TYPE_FP32, acc[i][j][e]) * acc[i + 1][j][e];
                else out[e] = p.bias ? acc[i][j][e] + bias[e] : acc[i][j][e];
            }
            const long long m = m0 + at;
            if (GATED && p.out_terms) store_terms(p, m, n, out);
            else store_outputs(p, p.order_out ? p.order_out[m] : m, n, out);
        }
    }
}

// The parts' sums, in order, and what becomes of them.
template <bool GATED>
__global__ __launch_bounds__(256) void int4_join_kernel(const Int4Args p, int blocks_n)
{
    const long long m = blockIdx.x / (unsigned)blocks_n;
    const int n = ((int)(blockIdx.x % (unsigned)blocks_n) * 256 + threadIdx.x) * 4;
    if (n >= p.N) return;
    float sum[GATED ? 2 : 1][4] = {}, bias[4];
    constexpr int MATS = GATED ? 2 : 1, U = 4;            // U parts' sums on their way together
    for (int part = 0; part < p.parts; part += U) {
        float v[U][MATS][4];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < MATS; ++k) {
                const float *const row = p.sums + ((long long)(min(part + u, p.parts - 1) * MATS + k) * p.M + m) * p.N;
                if (n + 4 <= p.N) __builtin_memcpy(v[u][k], row + n, 16);
                else load_params(row, n, p.N, 0.f, v[u][k]);
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < MATS; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[k][e] += part + u < p.parts ? v[u][k][e] : 0.f;
    }
    load_params(p.bias, n, p.N, 0.f, bias);
    float out[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (GATED) out[e] = gate(p.act, p.out_type != XNOR_TYPE_FP32, sum[0][e]) * sum[1][e];
        else out[e] = p.bias ? sum[0][e] + bias[e] : sum[0][e];
    }
    store_outputs(p, m, n, out);
}

template <class T, bool GATED, int TM, int TERMS>
hipError_t tiles(const Int4Args &p, hipStream_t st)
{
    constexpr int TOKENS = TERMS == 0 ? TM : TERMS == 2 ? TM / 2 : TM / 4;
    const int tiles_n = ceil_div(p.N, GATED ? 64 : 128), cuts = p.tiles ? std::max(1, p.tile / TOKENS) : 1;
    const long long all = p.tiles ? most_tiles(p.M, p.E, p.tile) * cuts : (p.M + TOKENS - 1) / TOKENS;
    const long long each = std::max<long long>(1, kMaxBlocks / tiles_n);
    for (long long m = 0; m < all; m += each) {
        Int4Args q = p;
        q.first = m, q.cuts = cuts;
        const long long n = std::min(each, all - m) * tiles_n;
        const dim3 grid((unsigned)((n + 7) / 8 * 8), p.parts), block(2 * TM);
        if (p.group == 32) int4_tile_kernel<T, GATED, true, TM, TERMS><<<grid, block, 0, st>>>(q, tiles_n, n);
        else int4_tile_kernel<T, GATED, false, TM, TERMS><<<grid, block, 0, st>>>(q, tiles_n, n);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class T, bool GATED>
hipError_t by_tiles(const Int4Args &p, hipStream_t st)
{
    if constexpr (!GATED && std::is_same<T, bf16_t>::value)
        if (p.terms) return p.terms == 2 ? tiles<T, GATED, 256, 2>(p, st) : tiles<T, GATED, 256, 3>(p, st);
    // the larger tile where there is one for each unit: half the conversions for a product (4096 x 8192 x 8192 bf16 a fifth more on the smaller than on
    // the larger), but one workgroup a unit, with nothing beside its begin and end (32768 pairs of 64 experts, 2048 x 1024, 976 and 982 us in all on
    // the smaller and the larger ones, of 8 experts with 1024 pairs each 252 and 267)
    const bool large = !p.tiles && p.parts == 1 && p.M > 128 && (p.M + 255) / 256 * ceil_div(p.N, GATED ? 64 : 128) >= compute_units();
    const hipError_t e = large ? tiles<T, GATED, 256, 0>(p, st) : tiles<T, GATED, 128, 0>(p, st);
    if (e != hipSuccess || p.parts == 1) return e;
    const int blocks_n = ceil_div(p.N, 1024);
    int4_join_kernel<GATED><<<dim3((unsigned)(p.M * blocks_n)), dim3(256), 0, st>>>(p, blocks_n);
    return hipGetLastError();
}

}  // namespace

// Whether a tile's operands are within 31 bits of where its buffers begin.
bool int4_tiles_support(const Int4Args &p)
{
    constexpr long long kMost = kTileReach;
    if (p.M == 0) return true;
    const long long groups = (p.K + p.group - 1) / p.group, last = p.order_x ? p.M / p.chosen : 256;
    return last * p.ldx + 2LL * p.K <= kMost && kRows * p.ldq <= kMost && (groups + 1) * p.N * 4 <= kMost;
}

int int4_expert_tile(long long pairs, int E)
{
    const long long each = (pairs + E - 1) / E;
    return each <= 16 ? 16 : each <= 32 ? 32 : each <= 64 ? 64 : 128;
}

// Shares of the contraction for few tiles: a step takes a workgroup 1.1 us, whether it is alone on its unit or not quite.  As many as make a workgroup a unit,
// of at least four steps, or two a unit where that leaves 20 steps each; at most 16.  us of GPU time with 1, 2, 4, 8, 16 shares (bf16, groups of 128):
//     128 x 2048 x 8192  134  73  43  30  25      128 x 4096 x 4096  71  43  30  27  30      128 x 8192 x 2048    40  26  20  26  36
//     192 x 8192 x 8192  136  78  62  69  86      384 x 8192 x 2048  40  40  43  58  90      gated 192 x 8192 x 2048  42  43  55  81
//     512 x 4096 x 4096   72  47  42  52  73      640 x 4096 x 4096  73  61  57  63  89      gated 128 x 8192 x 8192 136  82  69  82
static int shares(long long M, int N, int K, bool gated)
{
    const long long tiles = (M + 127) / 128 * ceil_div(N, gated ? 64 : 128), units = compute_units(), steps = K / kDeep;
    return (int)std::min<long long>(16, std::max<long long>({1, std::min(units / tiles, steps / 4), std::min(2 * units / tiles, steps / 20)}));
}

// By what both kernels take in us of GPU time, which these two forms meet within a tenth (926 products of 33 to 100000 tokens, 64 to 65536 rows, contractions of 60 to
// 16384, linear and gated, bf16): of each a round of workgroups, a contraction and what a workgroup begins and ends with, then the rounds that follow, and the
// shares' sums.  The kernel for few has to be a tenth faster: of two that are near the tiles are taken (the loss to the faster of both is then 1.0 % on the mean
// and 30 % at most, without that margin 0.4 %; of a limit on M N K and one on K it is 4.4 % and a factor of 3.5).  Few and tiles:
//     64 x 1024 x 4096   18.7 15.2    64 x 2048 x 8184  23.8 22.1     64 x 4096 x 4096  19.1 20.4     64 x 8192 x 8192  39.5 39.3     33 x 8192 x 8192  28.9 37.1
//     128 x 2048 x 4096  19.3 22.9   128 x 4096 x 6144  29.8 27.9    256 x 4096 x 4096  38.5 31.4    256 x 2048 x 2048  13.3 22.4     64 x 512 x 8192   34.1 18.3
//     8200 x 1030 x 70   59.0 25.9  4096 x 512 x 512    17.7 24.8    4096 x 8192 x 64     191 40.2    8192 x 512 x 1024  45.9 27.8   32768 x 64 x 1024 29.0 27.7
bool int4_many(long long M, int N, int K, bool gated, int parts)
{
    if (M <= kInt4Few / 2) return false;
    const double units = compute_units();
    const long long rows = (M + 63) / 64, wide = rows * ceil_div(N, 32);
    const double groups = (double)(gated || wide < units ? rows * ceil_div(N, 16) : wide);
    const double few = 2.2 + (2.5 + K / 1024. * (0.86 + 0.053 * std::min<long long>(M, 64) + (gated ? 0.17 : 0.))) * (1. + 0.74 * (std::ceil(groups / units) - 1.));
    const double tiles = (double)((M + 127) / 128) * ceil_div(N, gated ? 64 : 128) * parts;
    const double sums = parts > 1 ? 2.31e-6 * parts * M * N * (gated ? 2 : 1) - 2.1 : 0.;
    const double many = (11.4 + 1.06 * std::ceil(K / 64.) / parts) * (1. + 0.39 * std::max(0., tiles / units - 1.)) - 1. + sums;
    return few > 0.9 * many;
}

int int4_tile_parts(long long M, int N, int K, bool gated)
{
    const int parts = M > 0 ? shares(M, N, K, gated) : 1;
    return int4_many(M, N, K, gated, parts) ? parts : 1;
}

hipError_t launch_int4_tiles(const Int4Args &p, int type, bool gated, hipStream_t st)
{
    if (p.M == 0) return hipSuccess;
    if (type == XNOR_TYPE_F16) return gated ? by_tiles<f16_t, true>(p, st) : by_tiles<f16_t, false>(p, st);
    return gated ? by_tiles<bf16_t, true>(p, st) : by_tiles<bf16_t, false>(p, st);
}

}  // namespace xnor
