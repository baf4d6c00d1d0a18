// What routing to experts and the products with 4-bit weights share.
#pragma once

#include <algorithm>

#include "dense_common.hpp"

namespace xnor {

constexpr int kMaxExperts = 1024, kMaxChosen = 32;

struct RouteArgs {
    const void *logits;
    long long T, stride;
    int E;
    const float *bias;
    int score, groups, kept, top, k, renorm;
    float factor;
    int32_t *experts;
    float *weights;
    const float *dweights;          // backward
    void *dlogits;
    long long dstride;
};
hipError_t launch_route(const RouteArgs &p, int type, hipStream_t st);
hipError_t launch_route_bwd(const RouteArgs &p, int type, hipStream_t st);

struct ListArgs {
    const int32_t *experts;
    long long pairs;
    int E;
    int32_t *offsets, *order, *counts;      // counts: workspace
    int tile;                               // > 0: the lists cut into tiles of so many pairs,
    struct ExpertTile *tiles;               // one after the other; tiles[0].count is their number
};
// A tile of an expert's sorted positions.
struct ExpertTile {
    int expert, first, count, unused;
};
inline long long most_tiles(long long pairs, int E, int tile) { return std::min<long long>(E, pairs) + pairs / tile; }
size_t route_lists_workspace(long long pairs, int E);
hipError_t launch_route_lists(const ListArgs &p, hipStream_t st);

// A matrix of 4-bit weights, or a stack of them, as the kernels see it.
struct Int4View {
    const uint8_t *q;
    const void *scale;
    const uint8_t *zero;
};
struct Int4Args {
    const void *x;              // [M][K], or the experts' tokens: sorted position i's row is order[i] / chosen, or i (order_x NULL)
    long long ldx;              // bytes
    Int4View w, w2;             // w2: the gated block's second matrix
    long long ldq;              // bytes
    int scale_type, group;
    long long M;
    int N, K, act;
    const float *bias;
    void *out;                  // row m; experts: row i, or order_out[i]
    long long ldo;              // values
    int out_type;
    const ExpertTile *tiles;    // of experts' sorted positions, NULL: one matrix for all of x's rows
    int tile;                   // their tokens
    const int32_t *order_x, *order_out;
    const int32_t *pairs;       // experts' pairs, each by itself (tiles NULL): row m is that of expert pairs[m], x's row m / chosen
    int E, chosen;
    int terms;                  // > 0: x's rows are so many rows of bf16 each, hidden_stride(K) values from one another, whose sum is the token
    int out_terms;              // > 0 (gated): outputs are left as such rows; out_type is then that of what is computed from them
    int cuts;                   // (terms; set by the launchers: workgroups for a tile's pairs)
    int parts;                  // > 1: shares of the contraction, their sums fp32 [parts][matrices][M][N] in `sums`, joined by a second launch
    float *sums;
    long long first;            // (set by the launchers: the launch's first tile of tokens)
};
// Between the experts' two products a value is held as the sum of bf16 ones: two hold 16 bits of it (outputs in 16 bits are then as far from the definition as
// those of products in fp32; rounded to the tokens' type they are 1.35 to 1.5 times as far), three the 24 of fp32, for outputs in fp32.  bf16 for f16 tokens
// too: a block's outputs may pass f16's largest value.  (4096 tokens to 8 of 64 experts, 2048 x 1024, bf16: 1030-1075 us, with hidden values in bf16 837; 24 tokens to 3 of 30
// 37.9 and 32.8, one token to 8 of 64 18.9 and 17.2.)
constexpr int kMostTerms = 3;
inline int hidden_terms(int out_type) { return out_type == XNOR_TYPE_FP32 ? 3 : 2; }
__host__ __device__ inline int hidden_stride(int F) { return (F + 7) / 8 * 8; }

// Tiles of more of an expert's tokens than this go to the kernel for many.
constexpr int kInt4Few = 64;
// Whether a product of all of x's rows goes there, in so many shares of the contraction.
bool int4_many(long long M, int N, int K, bool gated, int parts);
// Whether so few pairs are better taken each by itself, without lists: experts of several are read for each of theirs, from the caches mostly.  us of GPU time, by
// lists and by pairs, for tokens to k of E experts, width x hidden (bf16, groups of 128):
//     8 of 64, 2048 x 1024    1: 23.6 18.8    4: 45.9 40.3    6: 51.7 55.9        2 of 8, 4096 x 2048     1: 22.0 17.6    2: 31.2 28.0    3: 30.9 36.8
//     8 of 128, 2048 x 512    1: 20.0 13.9    8: 48.2 48.0   12: 58.4 67.2        4 of 32, 1024 x 768     4: 20.4 14.9    6: 22.7 23.0    8: 22.5 24.4
//     8 of 256, 2048 x 512    4: 35.4 28.1    8: 52.3 47.9   12: 64.9 67.4        4 of 16, 2048 x 2048    2: 31.0 24.5    3: 36.1 36.2    6: 43.4 55.6
inline bool int4_pairs_pay(long long pairs, int E) { return pairs <= 4 || (2 * pairs <= E && pairs <= 64); }
// A token's chosen experts' second products and their sum in one launch: x holds the rows of the pairs, weights their shares, M the tokens.
hipError_t launch_int4_down(const Int4Args &p, const float *weights, hipStream_t st);
// GATED: w and w2 with the activation.
hipError_t launch_int4_few(const Int4Args &p, int type, bool gated, hipStream_t st);
constexpr long long kTileReach = 0x7fffffff;     // bytes from where a tile's buffers begin
bool int4_tiles_support(const Int4Args &p);
hipError_t launch_int4_tiles(const Int4Args &p, int type, bool gated, hipStream_t st);
// By the number of tokens (experts: by the tiles that they were cut into).
hipError_t launch_int4(const Int4Args &p, int type, bool gated, hipStream_t st);
int int4_tile_parts(long long M, int N, int K, bool gated);
int int4_expert_tile(long long pairs, int E);

struct Int4Make {
    const void *from;           // weights, levels, or (dequantize) nothing
    long long rows, stride;
    int cols, group;
    uint8_t *q;
    long long q_stride;
    void *scale;
    uint8_t *zero;
    int scale_type;
    void *out;
    int out_type;
};
hipError_t launch_int4_quantize(const Int4Make &p, int w_type, hipStream_t st);
hipError_t launch_int4_pack(const Int4Make &p, hipStream_t st);
hipError_t launch_int4_dequantize(const Int4Make &p, hipStream_t st);

// out[t] = sum over slots of weights[t][s] * pairs[t k + s], of slots without an expert weights * 0.
struct CombineArgs {
    const float *pairs;
    const int32_t *experts;
    const float *weights;
    long long T, ldo;
    int k, E, N;
    void *out;
    int out_type;
};
hipError_t launch_combine(const CombineArgs &p, hipStream_t st);

__device__ inline float load_real(const void *p, long long at, int type)
{
    return type == XNOR_TYPE_FP32 ? ((const float *)p)[at] : type == XNOR_TYPE_F16 ? (float)((const f16_t *)p)[at] : (float)((const bf16_t *)p)[at];
}
__device__ inline void store_real(void *p, long long at, int type, float v)
{
    if (type == XNOR_TYPE_FP32) ((float *)p)[at] = v;
    else if (type == XNOR_TYPE_F16) ((f16_t *)p)[at] = (f16_t)v;
    else ((bf16_t *)p)[at] = (bf16_t)v;
}

}  // namespace xnor
