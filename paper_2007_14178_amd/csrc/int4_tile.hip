// Products of many tokens with 4-bit weights: 128 tokens x 128 rows of the weights (gated: 64 of each matrix) by four waves of 64 x 64.
//
// Tokens and weights go through registers into LDS, 64 values of a row at a time, the weights as values of the tokens' type: (level - zero) * scale
// in fp32, rounded once, which is what the matrix instructions take.  A step's rows are on their way while the one before is multiplied, and are
// turned into values and written to the other half of LDS between its instructions.
#include <algorithm>

#include "int4_common.hpp"

namespace xnor {
namespace {

constexpr int kThreads = 256, kRows = 128, kDeep = 64;       // values of a step

// The values of a word: level * scale - zero * scale.
template <class T>
__device__ inline i32x4 values_of(uint32_t w, float scale, float minus)
{
    uint32_t even = w & 0x0f0f0f0fu, odd = w >> 4 & 0x0f0f0f0fu;
    // (so that a byte's conversion is one instruction)
    asm("" : "+v"(even));
    asm("" : "+v"(odd));
    auto at = [&](uint32_t v, int byte) { return (T)__builtin_fmaf((float)(v >> 8 * byte & 255u), scale, minus); };
    const T to[8] = {at(even, 0), at(even, 2), at(odd, 0), at(odd, 2), at(even, 1), at(even, 3), at(odd, 1), at(odd, 3)};
    return __builtin_bit_cast(i32x4, to);
}

template <class T, bool GATED>
__global__ __launch_bounds__(kThreads, 2) void int4_tile_kernel(const Int4Args p, int tiles_n, long long tiles)
{
    constexpr int TN = GATED ? 64 : 128;        // outputs n of a tile
    typedef Mat<T> Mul;
    __shared__ __align__(16) char lds[2][2 * kRows * kStep];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    // Workgroups go round the eight XCDs by their index: each takes a run of consecutive tiles, groups of eight tiles of tokens for a tile of the
    // weights' rows, so that what its units work on at a time shares both in its L2.
    const long long eighth = (tiles + 7) >> 3, index = (blockIdx.x & 7) * eighth + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= eighth || index >= tiles) return;
    const int rows = (int)(tiles / tiles_n), group8 = (int)(index / (8 * tiles_n)), in = (int)(index - (long long)group8 * 8 * tiles_n);
    const int high = min(8, rows - group8 * 8);
    const int tn = __builtin_amdgcn_readfirstlane(in / high), tm = __builtin_amdgcn_readfirstlane(group8 * 8 + in % high);
    const int n0 = tn * TN;
    Int4View view[2] = {p.w, GATED ? p.w2 : p.w};
    long long m0 = (p.first + tm) * kRows;
    int count = (int)min(p.M - m0, (long long)kRows);
    if (p.offsets) {
        ExpertTile tile;
        if (!expert_tile(p.offsets, p.E, kRows, p.first + tm, &tile)) return;
        m0 = tile.first, count = tile.count;
        view[0] = of_stack(view[0], p, tile.expert), view[1] = of_stack(view[1], p, tile.expert);
    }

    // Tokens: chunk `chunk` of rows t / 8 + 32 i.  Weights: word pair `pair` (16 values) of rows t / 4 + 64 i.
    const int chunk = t & 7, pair = t & 3;
    const T *a[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const long long m = m0 + min((t >> 3) + 32 * i, count - 1);
        a[i] = (const T *)((const char *)p.x + (p.order_x ? p.order_x[m] / p.chosen : m) * p.ldx);
    }
    const uint32_t *b[2];
    int row[2];
    const Int4View *of[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = (t >> 2) + 64 * i;
        row[i] = min(n0 + (GATED ? (r >> 5) * 16 + (r & 15) : r), p.N - 1);
        of[i] = &view[GATED ? r >> 4 & 1 : 0];
        b[i] = (const uint32_t *)(of[i]->q + row[i] * p.ldq);
    }
    const int words = (p.K + 7) / 8, groups = (p.K + p.group - 1) / p.group, shift = __builtin_ctz(p.group);
    const int steps = (p.K + kDeep - 1) / kDeep;

    Chunk<T> va[4];
    uint32_t vb[2][2];
    float scale[2], minus[2];
    auto fetch = [&](int s, auto whole) __attribute__((always_inline)) {
        const int at = s * kDeep + chunk * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (decltype(whole)::value) __builtin_memcpy(&va[i], a[i] + at, 16);
            else va[i] = load_chunk(a[i], at, p.K);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int w = s * (kDeep / 8) + pair * 2;
            const long long g = (long long)min((s * kDeep + pair * 16) >> shift, groups - 1) * p.N + row[i];
            if constexpr (decltype(whole)::value) {
                __builtin_memcpy(vb[i], b[i] + w, 8);
            } else {
                vb[i][0] = w < words ? b[i][w] : 0;
                vb[i][1] = w + 1 < words ? b[i][w + 1] : 0;
            }
            scale[i] = load_real(of[i]->scale, g, p.scale_type);
            minus[i] = of[i]->zero ? (float)(of[i]->zero[g] & 15) : 8.f;
        }
    };
    auto put = [&](int s) __attribute__((always_inline)) {
        char *const la = lds[s & 1], *const lb = la + kRows * kStep;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (t >> 3) + 32 * i;
            *(i32x4 *)(la + r * kStep + ((chunk ^ (r & 7)) << 4)) = __builtin_bit_cast(i32x4, va[i]);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = (t >> 2) + 64 * i;
            const float less = -minus[i] * scale[i];
#pragma unroll
            for (int j = 0; j < 2; ++j)
                *(i32x4 *)(lb + r * kStep + (((pair * 2 + j) ^ (r & 7)) << 4)) = values_of<T>(vb[i][j], scale[i], less);
        }
    };
    auto fetch_any = [&](int s) __attribute__((always_inline)) {
        if ((s + 1) * kDeep <= p.K) fetch(s, std::true_type{});
        else fetch(s, std::false_type{});
    };

    const int wm = (wave & 1) * 64, wn = (wave >> 1) * 64;
    f32x4 acc[4][4] = {};
    fetch_any(0);
    put(0);
    if (steps > 1) fetch_any(1);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
    for (int s = 0; s < steps; ++s) {
        const char *const la = lds[s & 1], *const lb = la + kRows * kStep;
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
                for (int j = 0; j < 4; ++j) acc[i][j] = Mul::mul(fb[i], fa[j], acc[i][j]);
        }
        if (s + 1 < steps) {
            put(s + 1);
            if (s + 2 < steps) fetch_any(s + 2);
        }
        // (LDS alone is waited for: the fetches are not)
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
    }
#pragma unroll
    for (int i = 0; i < 4; i += GATED ? 2 : 1) {
        const int n = n0 + (GATED ? wn / 2 + i * 8 : wn + i * 16) + (lane >> 4) * 4;
        if (n >= p.N) continue;
        float bias[4];
        load_params(p.bias, n, p.N, 0.f, bias);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int at = wm + j * 16 + (lane & 15);
            if (at >= count) continue;
            float out[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (GATED) out[e] = gate(p.act, p.out_type != XNOR_TYPE_FP32, acc[i][j][e]) * acc[i + 1][j][e];
                else out[e] = p.bias ? acc[i][j][e] + bias[e] : acc[i][j][e];
            }
            const long long m = m0 + at;
            store_outputs(p, p.order_out ? p.order_out[m] : m, n, out);
        }
    }
}

template <class T, bool GATED>
hipError_t tiles(const Int4Args &p, hipStream_t st)
{
    const int tiles_n = ceil_div(p.N, GATED ? 64 : 128);
    const long long all = p.offsets ? std::min<long long>(p.E, p.M) + p.M / kRows : (p.M + kRows - 1) / kRows;
    const long long each = std::max<long long>(1, kMaxBlocks / tiles_n);
    for (long long m = 0; m < all; m += each) {
        Int4Args q = p;
        q.first = m;
        const long long n = std::min(each, all - m) * tiles_n;
        int4_tile_kernel<T, GATED><<<dim3((unsigned)((n + 7) / 8 * 8)), dim3(kThreads), 0, st>>>(q, tiles_n, n);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_int4_tiles(const Int4Args &p, int type, bool gated, hipStream_t st)
{
    if (p.M == 0) return hipSuccess;
    if (type == XNOR_TYPE_F16) return gated ? tiles<f16_t, true>(p, st) : tiles<f16_t, false>(p, st);
    return gated ? tiles<bf16_t, true>(p, st) : tiles<bf16_t, false>(p, st);
}

}  // namespace xnor
