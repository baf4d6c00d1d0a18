// Routing of tokens to experts: the choice with its weights, the experts' lists, the logits' gradient, and the sum over a token's experts.
#include <algorithm>
#include <atomic>

#include "experts_common.hpp"

namespace xnor {
namespace {

constexpr int kThreads = 256;

template <int CTRL>
__device__ inline int dpp_int(int v)
{
    return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true);
}
template <int CTRL>
__device__ inline double dpp_double(double v)
{
    return __hiloint2double(dpp_int<CTRL>(__double2hiint(v)), dpp_int<CTRL>(__double2loint(v)));
}

// Over the LANES (16 or 64) lanes of a token, to all of them.  step(ask): ask(v) is the value v of the lane's partner.
template <int LANES, class Step>
__device__ inline void over_lanes(Step step)
{
    step([](auto v) { if constexpr (sizeof(v) == 8) return dpp_double<0xb1>(v); else return dpp_int<0xb1>(v); });
    step([](auto v) { if constexpr (sizeof(v) == 8) return dpp_double<0x4e>(v); else return dpp_int<0x4e>(v); });
    step([](auto v) { if constexpr (sizeof(v) == 8) return dpp_double<0x141>(v); else return dpp_int<0x141>(v); });
    step([](auto v) { if constexpr (sizeof(v) == 8) return dpp_double<0x140>(v); else return dpp_int<0x140>(v); });
    if constexpr (LANES == 64) {
        step([](auto v) { return __shfl_xor(v, 16); });
        step([](auto v) { return __shfl_xor(v, 32); });
    }
}

template <int LANES>
__device__ inline double sum_lanes(double v)
{
    over_lanes<LANES>([&](auto ask) { v += ask(v); });
    return v;
}
template <int LANES>
__device__ inline double max_lanes(double v)
{
    over_lanes<LANES>([&](auto ask) { const double o = ask(v); v = o > v ? o : v; });
    return v;
}
template <int LANES>
__device__ inline bool any_lane(bool b)
{
    int v = b;
    over_lanes<LANES>([&](auto ask) { v |= ask(v); });
    return v != 0;
}
// The largest, and of equals the one with the lowest index.
template <int LANES>
__device__ inline void best_lanes(double *v, int *at)
{
    over_lanes<LANES>([&](auto ask) {
        const double o = ask(*v);
        const int oa = ask(*at);
        if (o > *v || (o == *v && oa < *at)) *v = o, *at = oa;
    });
}

constexpr double kNone = -__builtin_huge_val();

// A lane's values of a row of n, the first at `at`: `each` of them, none behind the row's end.  Full rows by 16 bytes at a time.
template <class X, int EACH>
__device__ inline void load_logits(const X *row, int at, int each, int n, int lanes, float none, float (&to)[EACH])
{
    if (n == EACH * lanes) {
        constexpr int V = 16 / sizeof(X) < EACH ? 16 / sizeof(X) : EACH;
        X raw[EACH];
#pragma unroll
        for (int i = 0; i < EACH; i += V) __builtin_memcpy(raw + i, row + at + i, V * sizeof(X));
#pragma unroll
        for (int i = 0; i < EACH; ++i) to[i] = (float)raw[i];
    } else {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const float v = (float)row[min(at + i, n - 1)];
            to[i] = i < each && at + i < n ? v : none;
        }
    }
}

__device__ inline double score_of(const RouteArgs &p, double logit, double top, double total)
{
    return p.score == XNOR_SCORE_SOFTMAX ? exp(logit - top) / total : 1. / (1. + exp(-logit));
}

// LANES lanes to a token, of whose experts each has EACH consecutive ones: up to LANES * EACH experts.
//
// Scores in 64 bits, as which of two nearly equal ones is the larger decides whole numbers: a quarter of the time is the exponentials' (16384 x 256 in fp32,
// 8 of 4 of 8 groups: 28 us, at the rate of a copy 3.5).  The k best are taken one after the other, each by a scan of a lane's own and a tree over the lanes
// by DPP; lane n keeps the n-th.
template <class X, int LANES, int EACH>
__global__ __launch_bounds__(kThreads) void route_kernel(const RouteArgs p, long long first)
{
    constexpr int TOKENS = kThreads / LANES, SLOTS = (kMaxChosen + LANES - 1) / LANES;
    const int l = threadIdx.x % LANES;
    const long long t = first + (long long)blockIdx.x * TOKENS + threadIdx.x / LANES;
    const bool there = t < p.T;
    const X *const logits = (const X *)p.logits + (there ? t : p.T - 1) * p.stride;
    const int each = (p.E + LANES - 1) / LANES, e0 = l * each;

    double c[EACH];             // what the choice goes by
    bool unfit = false;
    double top = kNone, total = 1.;
    {
        float v[EACH];
        load_logits<X, EACH>(logits, e0, each, p.E, LANES, -__builtin_huge_valf(), v);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            unfit |= v[i] != v[i] || (p.score == XNOR_SCORE_SOFTMAX && v[i] == __builtin_huge_valf());
            c[i] = v[i];
            top = c[i] > top ? c[i] : top;
        }
    }
    unfit = any_lane<LANES>(unfit);
    if (p.score == XNOR_SCORE_SOFTMAX) {
        top = max_lanes<LANES>(top);
        total = 0.;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            c[i] = c[i] == kNone ? kNone : exp(c[i] - top);
            total += c[i] == kNone ? 0. : c[i];
        }
        total = sum_lanes<LANES>(total);
#pragma unroll
        for (int i = 0; i < EACH; ++i) c[i] = c[i] == kNone ? kNone : c[i] / total;
    } else {
#pragma unroll
        for (int i = 0; i < EACH; ++i) c[i] = c[i] == kNone ? kNone : 1. / (1. + exp(-c[i]));
    }
    if (p.bias) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            c[i] += (double)p.bias[min(e0 + i, p.E - 1)];
            if (!(c[i] > kNone)) c[i] = kNone;
        }
    }
    if (p.kept < p.groups) {
        const int size = p.E / p.groups, lanes = size / each;
        uint32_t stay = 0;                      // of the lane's experts
        if (size % each == 0 && (lanes & (lanes - 1)) == 0 && lanes <= 16) {
            // a lane's experts are of one group, a group's lanes neighbours: its two largest, over 1, 2, 4, 8 or 16 lanes
            double a = kNone, b = kNone;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const double v = i < each ? c[i] : kNone;
                const double low = v > a ? a : v;
                b = low > b ? low : b;
                a = v > a ? v : a;
            }
            auto both = [&](auto ask) {
                const double oa = ask(a), ob = ask(b);
                const double low = oa > a ? a : oa, more = ob > b ? ob : b;
                a = oa > a ? oa : a;
                b = low > more ? low : more;
            };
            if (lanes > 1) both([](double v) { return dpp_double<0xb1>(v); });
            if (lanes > 2) both([](double v) { return dpp_double<0x4e>(v); });
            if (lanes > 4) both([](double v) { return dpp_double<0x141>(v); });
            if (lanes > 8) both([](double v) { return dpp_double<0x140>(v); });
            const double score = p.top == 2 && b > kNone ? a + b : a;
            const int group = l / lanes;
            bool open = group < p.groups;       // (the last lanes may have no experts)
            for (int n = 0; n < p.kept; ++n) {
                double best = open ? score : kNone;
                int at = open ? group : kMaxExperts;
                best_lanes<LANES>(&best, &at);
                if (at == group) open = false, stay = ~0u;
            }
        } else {
            // the groups' scores, one after the other, group g's kept by lane g / per
            const int per = (p.groups + LANES - 1) / LANES;
            double score[EACH];
#pragma unroll
            for (int i = 0; i < EACH; ++i) score[i] = kNone;
            for (int g = 0; g < p.groups; ++g) {
                double a = kNone, b = kNone;        // the two largest
#pragma unroll
                for (int i = 0; i < EACH; ++i) {
                    const int e = e0 + i;
                    if (i < each && e >= g * size && e < (g + 1) * size) {
                        b = c[i] > a ? a : c[i] > b ? c[i] : b;
                        a = c[i] > a ? c[i] : a;
                    }
                }
                over_lanes<LANES>([&](auto ask) {
                    const double oa = ask(a), ob = ask(b);
                    const double low = oa > a ? a : oa, more = ob > b ? ob : b;
                    a = oa > a ? oa : a;
                    b = low > more ? low : more;
                });
                const double sum = p.top == 2 && b > kNone ? a + b : a;
#pragma unroll
                for (int i = 0; i < EACH; ++i)
                    if (l * per + i == g && i < per) score[i] = sum;
            }
            uint32_t taken = 0;                     // of the lane's groups
            for (int n = 0; n < p.kept; ++n) {
                double best = kNone;
                int at = kMaxExperts;               // (a group whose score is -inf can be the best that is left)
#pragma unroll
                for (int i = 0; i < EACH; ++i)
                    if (i < per && l * per + i < p.groups && !(taken >> i & 1) && (at == kMaxExperts || score[i] > best)) best = score[i], at = l * per + i;
                best_lanes<LANES>(&best, &at);
                if (at / per == l) taken |= 1u << (at - l * per);
#pragma unroll
                for (int i = 0; i < EACH; ++i)
                    if (e0 + i >= at * size && e0 + i < (at + 1) * size) stay |= 1u << i;
            }
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (!(stay >> i & 1)) c[i] = kNone;
    }

    int mine[SLOTS];                // slot l + i LANES
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) mine[i] = -1;
    for (int n = 0; n < p.k; ++n) {
        double best = kNone;
        int at = kMaxExperts;
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (c[i] > best) best = c[i], at = e0 + i;
        best_lanes<LANES>(&best, &at);
        if (unfit || !(best > kNone)) break;        // (the token's lanes together)
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (e0 + i == at) c[i] = kNone;
#pragma unroll
        for (int i = 0; i < SLOTS; ++i)
            if (n == l + i * LANES) mine[i] = at;
    }
    double w[SLOTS], sum = 0., most = kNone;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        w[i] = mine[i] >= 0 ? (double)(float)logits[mine[i]] : kNone;
        most = w[i] > most ? w[i] : most;
    }
    // (a softmax's shares are those of exponentials relative to the chosen's largest, whatever its own score is)
    if (p.renorm && p.score == XNOR_SCORE_SOFTMAX) top = max_lanes<LANES>(most), total = 1.;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        w[i] = mine[i] >= 0 ? score_of(p, w[i], top, total) : 0.;
        sum += w[i];
    }
    if (p.renorm) sum = sum_lanes<LANES>(sum);
    if (!there) return;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        const int n = l + i * LANES;
        if (n >= p.k) continue;
        const double share = !p.renorm ? w[i] : sum > 0. ? w[i] / sum : 0.;
        p.experts[t * p.k + n] = mine[i];
        p.weights[t * p.k + n] = unfit ? __uint_as_float(0x7fc00000u) : (float)(share * (double)p.factor);
    }
}

// The gradient.  With shares r = p / S of the chosen (renorm) it is r (dw' - sum dw' r), times 1 - p for sigmoids: only the chosen have one, and it is
// formed from their logits alone, r from exponentials relative to the chosen's largest, which keeps scores that fp32 would not hold.  A softmax
// whose weights are the scores themselves has the dense one, p (dw' - sum dw' p).  (16384 x 256 in fp32, dense, 8 chosen: 16 us, 2.1-2.4 TB/s; a row's maximum, sum,
// and slots matched against a lane's experts are one chain.)
template <class X, int LANES, int EACH>
__global__ __launch_bounds__(kThreads) void route_back_kernel(const RouteArgs p, long long first)
{
    constexpr int TOKENS = kThreads / LANES, SLOTS = (kMaxChosen + LANES - 1) / LANES;
    __shared__ float values[TOKENS][kMaxChosen];
    __shared__ int of[TOKENS][kMaxChosen];
    const int l = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    const long long t = first + (long long)blockIdx.x * TOKENS + slot;
    const bool there = t < p.T;
    const long long token = there ? t : p.T - 1;
    const X *const logits = (const X *)p.logits + token * p.stride;
    const int each = (p.E + LANES - 1) / LANES, e0 = l * each;
    const bool softmax = p.score == XNOR_SCORE_SOFTMAX, dense = softmax && !p.renorm;
    constexpr float NONE = -__builtin_huge_valf();
    auto sum_of = [](float v) {
        over_lanes<LANES>([&](auto ask) { v += __int_as_float(ask(__float_as_int(v))); });
        return v;
    };
    auto max_of = [](float v) {
        over_lanes<LANES>([&](auto ask) { v = fmaxf(v, __int_as_float(ask(__float_as_int(v)))); });
        return v;
    };

    float s[EACH];              // dense: the scores
    float top = NONE, total = 1.f;
    if (dense) {
        load_logits<X, EACH>(logits, e0, each, p.E, LANES, NONE, s);
#pragma unroll
        for (int i = 0; i < EACH; ++i) top = fmaxf(top, s[i]);
        top = max_of(top);
        total = 0.f;
#pragma unroll
        for (int i = 0; i < EACH; ++i) total += s[i] = s[i] == NONE ? 0.f : expf(s[i] - top);
        total = sum_of(total);
#pragma unroll
        for (int i = 0; i < EACH; ++i) s[i] = total > 0.f ? s[i] / total : 0.f;
    }
    // a slot a lane: its expert, logit and weight's gradient
    int e[SLOTS];
    float logit[SLOTS], dw[SLOTS], w[SLOTS], most = NONE;
    bool any = false;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        const int n = l + i * LANES;
        e[i] = n < p.k ? p.experts[token * p.k + n] : -1;
        const bool is = e[i] >= 0 && e[i] < p.E;
        any |= is;
        if (!is) e[i] = -1;
        logit[i] = is ? (float)logits[e[i]] : NONE;
        dw[i] = is ? p.factor * p.dweights[token * p.k + n] : 0.f;
        most = fmaxf(most, logit[i]);
    }
    bool empty = !any_lane<LANES>(any);
    if (!dense) {
        top = max_of(most);
        // sigmoids that are all 0 in 64 bits have weights of 0, whatever the logits
        if (!softmax && p.renorm && top < -700.f) empty |= !(1. / (1. + exp(-(double)top)) > 0.);
        if (!softmax) top = fminf(0.f, top);
    }
    float sum = 0.f, dot = 0.f;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        const bool none = logit[i] == NONE;
        // sigmoid: times exp(-top), which is 1 but for logits all below 0
        if (softmax) w[i] = none ? 0.f : expf(logit[i] - top);
        else w[i] = none ? 0.f : p.renorm ? expf(fminf(logit[i], 0.f) - top) / (1.f + expf(-fabsf(logit[i]))) : 1.f / (1.f + expf(-logit[i]));
        sum += w[i];
    }
    if (p.renorm) total = sum_of(sum);
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        w[i] = total > 0.f ? w[i] / total : 0.f;
        dot += dw[i] * w[i];
    }
    dot = dense || p.renorm ? sum_of(dot) : 0.f;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        const int n = l + i * LANES;
        if (n >= p.k) continue;
        const float rest = softmax ? 1.f : 1.f / (1.f + expf(logit[i]));         // 1 - p of a sigmoid
        values[slot][n] = dense ? dw[i] : w[i] * (dw[i] - dot) * rest;
        of[slot][n] = e[i];
    }
    __syncthreads();
    float d[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) d[i] = 0.f;
    for (int n = 0; n < p.k; ++n) {
        const int at = of[slot][n] - e0;
        const float v = values[slot][n];
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (i == at && i < each) d[i] += v;
    }
    if (!there) return;
    X *const out = (X *)p.dlogits + t * p.dstride;
    X to[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) to[i] = (X)(empty ? 0.f : dense ? s[i] * (d[i] - dot) : d[i]);
    if (p.E == EACH * LANES) {
        constexpr int V = 16 / sizeof(X) < EACH ? 16 / sizeof(X) : EACH;
#pragma unroll
        for (int i = 0; i < EACH; i += V) __builtin_memcpy(out + e0 + i, to + i, V * sizeof(X));
    } else {
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (i < each && e0 + i < p.E) out[e0 + i] = to[i];
    }
}

template <class X, int LANES, int EACH>
hipError_t route(const RouteArgs &p, hipStream_t st)
{
    constexpr int TOKENS = kThreads / LANES;
    const long long most = (long long)kMaxBlocks * TOKENS;
    for (long long t = 0; t < p.T; t += most) {
        const dim3 grid((unsigned)((std::min(most, p.T - t) + TOKENS - 1) / TOKENS));
        if (p.dlogits) route_back_kernel<X, LANES, EACH><<<grid, dim3(kThreads), 0, st>>>(p, t);
        else route_kernel<X, LANES, EACH><<<grid, dim3(kThreads), 0, st>>>(p, t);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class X>
hipError_t route_by_experts(const RouteArgs &p, hipStream_t st)
{
    if (p.E <= 64) return route<X, 16, 4>(p, st);
    if (p.E <= 128) return route<X, 16, 8>(p, st);
    if (p.E <= 256) return route<X, 16, 16>(p, st);
    if (p.E <= 512) return route<X, 64, 8>(p, st);
    return route<X, 64, 16>(p, st);
}

// ---- the experts' lists ------------------------------------------------------------------------------------------------
// A workgroup has a run of pairs, in chunks of 64 of a wave each.  In a chunk an expert's pairs are the bits of a word, so that a pair's place among
// them is the number of set bits before its own: no order of atomics matters.  (131072 pairs of 256 experts 4.2 + 7.6 us, each workgroup summing all runs' counts;
// up to 1024 pairs one launch of 2.8.)

constexpr int kListWaves = 16, kListThreads = kListWaves * kWave, kMostRuns = 512;

int list_runs(long long pairs) { return (int)std::max<long long>(1, std::min<long long>(kMostRuns, (pairs + kListThreads - 1) / kListThreads)); }
long long list_run(long long pairs)
{
    const long long runs = list_runs(pairs);
    return std::max<long long>(1, ((pairs + runs - 1) / runs + kListThreads - 1) / kListThreads) * kListThreads;
}

__global__ __launch_bounds__(kListThreads) void list_count_kernel(const ListArgs p, long long run)
{
    __shared__ int count[kMaxExperts];
    for (int e = threadIdx.x; e < p.E; e += kListThreads) count[e] = 0;
    __syncthreads();
    const long long from = blockIdx.x * run, to = min(p.pairs, from + run);
    for (long long i = from + threadIdx.x; i < to; i += kListThreads) {
        const int e = p.experts[i];
        if (e >= 0 && e < p.E) atomicAdd(&count[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.E; e += kListThreads) p.counts[(long long)blockIdx.x * p.E + e] = count[e];
}

struct ListSums {
    int pairs[kListWaves], tiles[kListWaves];
};

__global__ __launch_bounds__(kListThreads) void list_kernel(const ListArgs p, long long run)
{
    extern __shared__ unsigned long long bits[];        // [kListWaves][E], then base [E] and room for as many
    int *const base = (int *)(bits + kListWaves * p.E);
    __shared__ ListSums sums;
    int *const wave_sums = sums.pairs, *const wave_tiles = sums.tiles;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const long long from = blockIdx.x * run, to = min(p.pairs, from + run);
    // of expert t: all its pairs, and those of the runs before
    int all = 0, before = 0;
    if (gridDim.x == 1) {
        if (t < p.E) base[t] = 0;
        __syncthreads();
        for (long long i = t; i < p.pairs; i += kListThreads) {
            const int e = p.experts[i];
            if (e >= 0 && e < p.E) atomicAdd(&base[e], 1);
        }
        __syncthreads();
        if (t < p.E) all = base[t];
    } else {
        // (the runs in as many parts as there are threads for, whose sums meet in LDS)
        const int parts = kListThreads / p.E, runs = gridDim.x, part = t / p.E, e = t - part * p.E;
        for (int i = t; i < 2 * p.E; i += kListThreads) base[i] = 0;
        __syncthreads();
        if (part < parts) {
            const int from_run = (int)((long long)runs * part / parts), to_run = (int)((long long)runs * (part + 1) / parts);
            int sum = 0, early = 0;
#pragma unroll 8
            for (int b = from_run; b < to_run; ++b) {
                const int n = p.counts[(long long)b * p.E + e];
                early += b < (int)blockIdx.x ? n : 0;
                sum += n;
            }
            atomicAdd(&base[e], sum), atomicAdd(&base[p.E + e], early);
        }
        __syncthreads();
        if (t < p.E) all = base[t], before = base[p.E + t];
    }
    int upto = all;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int v = __shfl_up(upto, d);
        if (lane >= d) upto += v;
    }
    if (lane == 63) wave_sums[wave] = upto;
    __syncthreads();
    int total = 0;
    for (int w = 0; w < kListWaves; ++w) {
        if (w < wave) upto += wave_sums[w];
        total += wave_sums[w];
    }
    if (t < p.E) {
        base[t] = upto - all + before;
        if (blockIdx.x == 0) p.offsets[t + 1] = upto;
    }
    if (blockIdx.x == 0 && t == 0) p.offsets[0] = 0;
    if (blockIdx.x == 0 && p.tiles) {
        const int mine = (all + p.tile - 1) / max(p.tile, 1);
        int to = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int v = __shfl_up(to, d);
            if (lane >= d) to += v;
        }
        if (lane == 63) wave_tiles[wave] = to;
        __syncthreads();
        int number = 0;
        for (int w = 0; w < kListWaves; ++w) {
            if (w < wave) to += wave_tiles[w];
            number += wave_tiles[w];
        }
        if (t == 0) p.tiles[0] = {0, 0, number, 0};
        for (int i = 0; i < mine; ++i) p.tiles[1 + to - mine + i] = {t, upto - all + i * p.tile, min(p.tile, all - i * p.tile), 0};
    }
    // behind the lists
    for (long long i = from + t; i < to; i += kListThreads)
        if (i >= total) p.order[i] = -1;

    for (long long chunk = from; chunk < to; chunk += kListThreads) {
        for (int i = t; i < kListWaves * p.E; i += kListThreads) bits[i] = 0;
        __syncthreads();
        const long long i = chunk + t;
        const int e = i < to ? p.experts[i] : -1;
        const bool in = e >= 0 && e < p.E;
        if (in) atomicOr(&bits[wave * p.E + e], 1ull << lane);
        __syncthreads();
        if (in) {
            int at = base[e] + __popcll(bits[wave * p.E + e] & ((1ull << lane) - 1));
            for (int w = 0; w < wave; ++w) at += __popcll(bits[w * p.E + e]);
            p.order[at] = (int)i;
        }
        if (chunk + kListThreads >= to) break;
        __syncthreads();
        if (t < p.E)
            for (int w = 0; w < kListWaves; ++w) base[t] += __popcll(bits[w * p.E + t]);
        __syncthreads();
    }
}

// ---- the sum over a token's experts ------------------------------------------------------------------------------------

// Bound by memory: 4096 tokens of 8 pairs of 2048 fp32 values 46 us, 6.2 TB/s.
__global__ __launch_bounds__(kThreads) void combine_kernel(const CombineArgs p, int blocks_n, long long first)
{
    const long long t = first + blockIdx.x / blocks_n;
    const int n = ((int)(blockIdx.x % blocks_n) * kThreads + threadIdx.x) * 4;
    if (n >= p.N) return;
    float sum[4] = {};
    for (int s = 0; s < p.k; ++s) {
        const int e = p.experts[t * p.k + s];
        const float w = p.weights[t * p.k + s];
        float v[4] = {};
        if (e >= 0 && e < p.E) load_params(p.pairs + (t * p.k + s) * p.N, n, p.N, 0.f, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += w * v[i];
    }
    const long long at = t * p.ldo;
    if (p.out_type == XNOR_TYPE_FP32) {
        store_values((float *)p.out + at, n, p.N, sum);
    } else if (p.out_type == XNOR_TYPE_F16) {
        const f16_t to[4] = {(f16_t)sum[0], (f16_t)sum[1], (f16_t)sum[2], (f16_t)sum[3]};
        store_values((f16_t *)p.out + at, n, p.N, to);
    } else {
        const bf16_t to[4] = {(bf16_t)sum[0], (bf16_t)sum[1], (bf16_t)sum[2], (bf16_t)sum[3]};
        store_values((bf16_t *)p.out + at, n, p.N, to);
    }
}

}  // namespace

hipError_t launch_route(const RouteArgs &p, int type, hipStream_t st)
{
    return type == XNOR_TYPE_FP32 ? route_by_experts<float>(p, st) : type == XNOR_TYPE_F16 ? route_by_experts<f16_t>(p, st) : route_by_experts<bf16_t>(p, st);
}

hipError_t launch_route_bwd(const RouteArgs &p, int type, hipStream_t st) { return launch_route(p, type, st); }

size_t route_lists_workspace(long long pairs, int E) { return pairs <= kListThreads ? 0 : (size_t)list_runs(pairs) * E * sizeof(int); }

hipError_t launch_route_lists(const ListArgs &p, hipStream_t st)
{
    const long long run = list_run(p.pairs);
    const int runs = (int)std::max<long long>(1, (p.pairs + run - 1) / run);
    const size_t lds = (size_t)kListWaves * p.E * 8 + p.E * 8;
    if (lds + sizeof(ListSums) > 64 * 1024) {       // (the limit is for both)
        static std::atomic<bool> raised[64];
        int dev = 0;
        hipError_t e = hipGetDevice(&dev);
        if (e != hipSuccess) return e;
        if (dev < 0 || dev >= 64 || !raised[dev].load(std::memory_order_relaxed)) {
            e = hipFuncSetAttribute(reinterpret_cast<const void *>(&list_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kMaxExperts * (kListWaves * 8 + 8));
            if (e != hipSuccess) return e;
            if (dev >= 0 && dev < 64) raised[dev].store(true, std::memory_order_relaxed);
        }
    }
    if (runs > 1) {
        list_count_kernel<<<dim3(runs), dim3(kListThreads), 0, st>>>(p, run);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    list_kernel<<<dim3(runs), dim3(kListThreads), lds, st>>>(p, run);
    return hipGetLastError();
}

hipError_t launch_combine(const CombineArgs &p, hipStream_t st)
{
    const int blocks_n = ceil_div(p.N, kThreads * 4);
    const long long most = std::max<long long>(1, kMaxBlocks / blocks_n);
    for (long long t = 0; t < p.T; t += most) {
        combine_kernel<<<dim3((unsigned)(std::min(most, p.T - t) * blocks_n)), dim3(kThreads), 0, st>>>(p, blocks_n, t);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace xnor
