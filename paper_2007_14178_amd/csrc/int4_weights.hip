// Real weights to levels of 4 bits and back: read once, written once, eight values a lane.  (8192 x 8192 bf16: 69 us to levels, 30 to 39 back, 40 for levels that
// are there; what a program does once.)
#include "experts_common.hpp"

namespace xnor {
namespace {

constexpr int kThreads = 256;

// Over the lanes that share a group: 4, 8 or 16.
template <class Op>
__device__ inline float group_reduce(float v, int lanes, Op op)
{
    v = op(v, dpp<0xb1>(v));
    v = op(v, dpp<0x4e>(v));
    if (lanes >= 8) v = op(v, dpp<0x141>(v));
    if (lanes >= 16) v = op(v, dpp<0x140>(v));
    return v;
}

struct Max {
    __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Min {
    __device__ float operator()(float a, float b) const { return fminf(a, b); }
};

__device__ inline float as_type(float v, int type) { return type == XNOR_TYPE_FP32 ? v : type == XNOR_TYPE_F16 ? (float)(f16_t)v : (float)(bf16_t)v; }

// Eight values of a row of n from `at` on, zeros behind its end.
__device__ inline void load_eight(const void *p, long long row, int at, int n, int type, float (&to)[8])
{
    if (type == XNOR_TYPE_FP32) load_params((const float *)p + row, at, n, 0.f, to);
    else if (type == XNOR_TYPE_F16) load_params((const f16_t *)p + row, at, n, 0.f, to);
    else load_params((const bf16_t *)p + row, at, n, 0.f, to);
}

template <class T>
__device__ inline void store_eight(void *p, long long row, int at, int n, const float (&v)[8])
{
    T to[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) to[i] = (T)v[i];
    store_values((T *)p + row, at, n, to);
}

// A lane makes one word, eight values; the lanes of a group are neighbours.
__global__ __launch_bounds__(kThreads) void int4_quantize_kernel(const Int4Make p, int w_type, long long first)
{
    const long long row = first + blockIdx.x;
    const int words = (p.cols + 7) / 8, lanes = p.group / 8, words_up = (words + lanes - 1) / lanes * lanes;
    for (int at = threadIdx.x; at < words_up; at += kThreads) {
        float v[8];
        load_eight(p.from, row * p.stride, at * 8, p.cols, w_type, v);
        float top = 0.f, low = 0.f, high = 0.f;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            bad |= !(fabsf(v[i]) <= 3.402823466e38f);
            low = fminf(low, v[i]), high = fmaxf(high, v[i]);
        }
        top = fmaxf(-low, high);
        bad = group_reduce(bad ? 1.f : 0.f, lanes, Max()) > 0.f;
        top = group_reduce(top, lanes, Max()), low = group_reduce(low, lanes, Min()), high = group_reduce(high, lanes, Max());
        float scale = as_type(p.zero ? (high - low) / 15.f : top / 7.f, p.scale_type);
        if (bad || !(scale <= 3.402823466e38f)) scale = __uint_as_float(0x7fc00000u);
        const bool none = !(scale > 0.f);           // (NaN among them)
        const float zero = !p.zero || none ? 8.f : fminf(fmaxf(rintf(-low / scale), 0.f), 15.f);
        uint32_t word = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float level = none ? zero : fminf(fmaxf(rintf(v[i] / scale) + zero, 0.f), 15.f);
            if (at * 8 + i < p.cols) word |= (uint32_t)level << (4 * (i >> 1) + 16 * (i & 1));
        }
        if (at < words) *(uint32_t *)(p.q + row * p.q_stride + at * 4) = word;
        if (at % lanes == 0) {
            const long long to = (long long)(at / lanes) * p.rows + row;
            store_real(p.scale, to, p.scale_type, scale);
            if (p.zero) p.zero[to] = (uint8_t)zero;
        }
    }
}

__global__ __launch_bounds__(kThreads) void int4_pack_kernel(const Int4Make p, long long first)
{
    const long long row = first + blockIdx.x;
    const uint8_t *const from = (const uint8_t *)p.from + row * p.stride;
    const int words = (p.cols + 7) / 8;
    for (int at = threadIdx.x; at < words; at += kThreads) {
        uint32_t word = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (at * 8 + i < p.cols) word |= (uint32_t)(from[at * 8 + i] & 15) << (4 * (i >> 1) + 16 * (i & 1));
        *(uint32_t *)(p.q + row * p.q_stride + at * 4) = word;
    }
}

__global__ __launch_bounds__(kThreads) void int4_dequantize_kernel(const Int4Make p, long long first)
{
    const long long row = first + blockIdx.x;
    const int words = (p.cols + 7) / 8;
    for (int at = threadIdx.x; at < words; at += kThreads) {
        const uint32_t word = *(const uint32_t *)(p.q + row * p.q_stride + at * 4);
        const long long g = (long long)(at * 8 / p.group) * p.rows + row;
        const float scale = load_real(p.scale, g, p.scale_type), zero = p.zero ? (float)(p.zero[g] & 15) : 8.f;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = ((float)(word >> (4 * (i >> 1) + 16 * (i & 1)) & 15u) - zero) * scale;
        if (p.out_type == XNOR_TYPE_FP32) store_eight<float>(p.out, row * p.stride, at * 8, p.cols, v);
        else if (p.out_type == XNOR_TYPE_F16) store_eight<f16_t>(p.out, row * p.stride, at * 8, p.cols, v);
        else store_eight<bf16_t>(p.out, row * p.stride, at * 8, p.cols, v);
    }
}

// Rows in launches of fewer than 2^32 threads.
template <class Launch>
hipError_t by_rows(long long rows, Launch launch)
{
    for (long long r = 0; r < rows; r += kMaxBlocks) {
        launch(dim3((unsigned)(rows - r < kMaxBlocks ? rows - r : kMaxBlocks)), r);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_int4_quantize(const Int4Make &p, int w_type, hipStream_t st)
{
    return by_rows(p.rows, [&](dim3 grid, long long first) { int4_quantize_kernel<<<grid, dim3(kThreads), 0, st>>>(p, w_type, first); });
}

hipError_t launch_int4_pack(const Int4Make &p, hipStream_t st)
{
    return by_rows(p.rows, [&](dim3 grid, long long first) { int4_pack_kernel<<<grid, dim3(kThreads), 0, st>>>(p, first); });
}

hipError_t launch_int4_dequantize(const Int4Make &p, hipStream_t st)
{
    return by_rows(p.rows, [&](dim3 grid, long long first) { int4_dequantize_kernel<<<grid, dim3(kThreads), 0, st>>>(p, first); });
}

}  // namespace xnor
