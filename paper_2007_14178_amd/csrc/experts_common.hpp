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
    long long first;            // (set by the launchers: the launch's first tile of tokens)
};
// Tiles of more tokens than this go to the kernel for many.
constexpr int kInt4Few = 64;
// Whether so few pairs are better taken each by itself, without lists.
inline bool int4_pairs_pay(long long pairs, int E) { return pairs <= 64 && pairs <= E; }
// A token's chosen experts' second products and their sum in one launch: x holds the rows of the pairs, weights their shares, M the tokens.
hipError_t launch_int4_down(const Int4Args &p, const float *weights, int type, hipStream_t st);
// GATED: w and w2 with the activation.
hipError_t launch_int4_few(const Int4Args &p, int type, bool gated, hipStream_t st);
bool int4_tiles_support(const Int4Args &p);
hipError_t launch_int4_tiles(const Int4Args &p, int type, bool gated, hipStream_t st);
// By the number of tokens (experts: by the tiles that they were cut into).
hipError_t launch_int4(const Int4Args &p, int type, bool gated, hipStream_t st);
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
