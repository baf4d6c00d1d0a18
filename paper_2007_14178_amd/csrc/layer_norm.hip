// Operators on the rows of a matrix: layer norm forward (real or quantised output) and backward, and the quantisation of rows
// to 8 bits.  All are bound by memory: a row is read once into registers, where its sums are formed, and written once.  (16384 x 4096 f16 47 us,
// 5.7 TB/s; 16384 x 8192 quantised 77 us over and over on the same rows, which the last-level cache holds a part of, 87-90 us right after other work, 5.2 and
// 4.5 TB/s; 100352 x 512 fp32 quantised 41 and 44-46 us, 6.3 and 5.7 TB/s.)
#include <algorithm>

#include "dense_common.hpp"

namespace xnor {
namespace {

enum RowOutput { kReal, kLevels, kQuantize };       // layer norm; layer norm, quantised; quantisation alone

constexpr int kBlock = 256;

// Over the THREADS threads of a row (a wave, or the whole workgroup).  `slots` is not written again before another barrier has passed.
template <int THREADS, class Op>
__device__ inline float row_reduce(float v, float *slots, Op op)
{
    v = wave_reduce(v, op);
    if constexpr (THREADS == kWave) return v;
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    v = slots[0];
#pragma unroll
    for (int i = 1; i < THREADS / kWave; ++i) v = op(v, slots[i]);
    return v;
}

// The chunk that starts `at` values into a row of `cols`, zeros where `there` is false or behind its end, by one load that no branch
// stands before: where one does, a wait for a row is a wait for what was asked for behind it too.  Rows of whole chunks at multiples of 16 bytes;
// the row the same for the whole wave.
template <class T>
__device__ inline Chunk<T> load_whole(const T *row, bool there, int cols, int at)
{
    Chunk<T> c{};
#ifdef __HIP_DEVICE_COMPILE__        // (the host's pass does not know the builtins)
    const auto from = __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(row), 0, there ? cols * (int)sizeof(T) : 0, 0x00027000);
    const auto raw = __builtin_amdgcn_raw_buffer_load_b128(from, at * (int)sizeof(T), 0, 0);
    __builtin_memcpy(&c, &raw, 16);
#endif
    return c;
}
inline bool whole_rows(const void *x, long long stride, int cols, int value_bytes)
{
    return (((uintptr_t)x | (uintptr_t)(stride * value_bytes) | (uintptr_t)cols * value_bytes) & 15) == 0;
}

// v rounded to T from fp32.  The compiler folds the last multiply-add of some values into the conversion to f16, which rounds once where the others
// round twice; it chooses anew in each copy of the code that takes the rows in turns, and a row's output would depend on its place among the rows.
template <class T>
__device__ inline T rounded(float v)
{
#ifdef __HIP_DEVICE_COMPILE__
    if constexpr (std::is_same<T, f16_t>::value) asm("" : "+v"(v));
#endif
    return (T)v;
}

constexpr int block_of(int threads) { return threads < kBlock ? kBlock : threads; }

// Rows by THREADS threads each, NV chunks of 16 bytes of a row in a thread's registers, and with them the parameters of its
// columns, which are read once for all of a workgroup's rows; the next row is on its way while one is worked on.  (NV = 0: rows of any
// length, read again for every sum.)  WHOLE: load_whole takes the rows, and two are on their way.
template <class T, class P, int OUT, int THREADS, int NV, bool WHOLE>
__global__ __launch_bounds__(block_of(THREADS)) void row_kernel(const RowArgs p)
{
    constexpr int V = Chunk<T>::kCount, ROWS = block_of(THREADS) / THREADS, N = NV ? NV : 1;
    __shared__ float slots[2][3][16];
    const int t = threadIdx.x % THREADS;
    const long long step = (long long)gridDim.x * ROWS;
    long long row = (long long)blockIdx.x * ROWS + __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS);
    if (row >= p.rows) return;                  // (rows share no barrier where a workgroup has several)

    float gamma[N][V], beta[N][V];
    constexpr int DEEP = WHOLE ? 2 : 1;
    Chunk<T> next[DEEP][N];
    auto fetch = [&](auto slot, long long r) __attribute__((always_inline)) {
        constexpr int D = decltype(slot)::value;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = (t + i * THREADS) * V;
            if constexpr (WHOLE) next[D][i] = load_whole((const T *)p.x + r * p.x_stride, r < p.rows, p.cols, at);
            else next[D][i] = load_chunk((const T *)p.x + r * p.x_stride, at, p.cols);
        }
    };
    using std::integral_constant;
    fetch(integral_constant<int, 0>(), row);
    if constexpr (WHOLE) fetch(integral_constant<int, 1>(), row + step);
    if constexpr (NV > 0 && OUT != kQuantize) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            load_params((const P *)p.gamma, (t + i * THREADS) * V, p.cols, 1.f, gamma[i]);
            load_params((const P *)p.beta, (t + i * THREADS) * V, p.cols, 0.f, beta[i]);
        }
    }
    auto work = [&](auto slot, int turn) __attribute__((always_inline)) {
        Chunk<T> held[N];
#pragma unroll
        for (int i = 0; i < NV; ++i) held[i] = next[decltype(slot)::value][i];
        if (WHOLE || row + step < p.rows) fetch(slot, row + DEEP * step);
        const T *x = (const T *)p.x + row * p.x_stride;
        auto each = [&](auto f) __attribute__((always_inline)) {        // f(column of the chunk's first value, chunk, its number)
            if constexpr (NV > 0) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if ((t + i * THREADS) * V < p.cols) f((t + i * THREADS) * V, held[i], i);
            } else {
                for (int at = t * V; at < p.cols; at += THREADS * V) f(at, load_chunk(x, at, p.cols), 0);
            }
        };

        float mean = 0.f, rstd = 1.f;
        if constexpr (OUT != kQuantize) {
            float s = 0.f;
            each([&](int, const Chunk<T> &c, int) {
#pragma unroll
                for (int k = 0; k < V; ++k) s += (float)c.v[k];
            });
            mean = row_reduce<THREADS>(s, slots[turn][0], Sum()) / (float)p.cols;
            float d2 = 0.f;         // about the mean: no difference of large squares
            each([&](int at, const Chunk<T> &c, int) {
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const float d = (float)c.v[k] - mean;
                    d2 += WHOLE || at + k < p.cols ? d * d : 0.f;
                }
            });
            rstd = 1.f / sqrtf(row_reduce<THREADS>(d2, slots[turn][1], Sum()) / (float)p.cols + p.eps);
            if (t == 0) {
                if (p.mean) p.mean[row] = mean;
                if (p.rstd) p.rstd[row] = rstd;
            }
        }
        auto values = [&](int at, const Chunk<T> &c, int i, float (&to)[V]) __attribute__((always_inline)) {
            if constexpr (NV == 0 && OUT != kQuantize) {
                load_params((const P *)p.gamma, at, p.cols, 1.f, gamma[0]);
                load_params((const P *)p.beta, at, p.cols, 0.f, beta[0]);
            }
#pragma unroll
            for (int k = 0; k < V; ++k) {
                if constexpr (OUT == kQuantize) to[k] = (float)c.v[k];
                else to[k] = WHOLE || at + k < p.cols ? ((float)c.v[k] - mean) * rstd * gamma[i][k] + beta[i][k] : 0.f;
            }
        };
        if constexpr (OUT == kReal) {
            T *y = (T *)p.y + row * p.y_stride;
            each([&](int at, const Chunk<T> &c, int i) {
                float v[V];
                values(at, c, i, v);
                T out[V];
#pragma unroll
                for (int k = 0; k < V; ++k) out[k] = rounded<T>(v[k]);
                store_values(y, at, p.cols, out);
            });
        } else {
            float top = 0.f;
            each([&](int at, const Chunk<T> &c, int i) {
                float v[V];
                values(at, c, i, v);
#pragma unroll
                for (int k = 0; k < V; ++k) top = MaxNan()(fabsf(v[k]), top);
            });
            top = row_reduce<THREADS>(top, slots[turn][2], MaxNan());
            const RowLevels levels = row_levels(top);
            if (t == 0) p.scale[row] = levels.scale;
            int8_t *q = p.q + row * p.y_stride;
            each([&](int at, const Chunk<T> &c, int i) {
                float v[V];
                values(at, c, i, v);
                int8_t out[V];
#pragma unroll
                for (int k = 0; k < V; ++k) out[k] = level_of(v[k], levels);
                store_values(q, at, p.cols, out);
            });
        }
    };
    if constexpr (WHOLE) {
        while (row < p.rows) {
            work(integral_constant<int, 0>(), 0);
            row += step;
            if (row >= p.rows) break;
            work(integral_constant<int, 1>(), 1);
            row += step;
        }
    } else {
        for (int turn = 0; row < p.rows; row += step, turn ^= 1) work(integral_constant<int, 0>(), turn);
    }
}

template <class T, class P, int OUT>
hipError_t launch_rows(const RowArgs &p, hipStream_t st)
{
    constexpr int V = Chunk<T>::kCount;
    if (p.rows == 0) return hipSuccess;
    const int chunks = ceil_div(p.cols, V);
    auto go = [&](auto threads, auto nv) {
        constexpr int THREADS = decltype(threads)::value, NV = decltype(nv)::value;
        constexpr int ROWS = block_of(THREADS) / THREADS;
        const long long blocks = (p.rows + ROWS - 1) / ROWS;
        const dim3 grid((unsigned)std::min<long long>(blocks, (THREADS >= 512 && OUT == kReal ? 4 : 16) * compute_units())), block(block_of(THREADS));
        // (16-bit rows: 16384 x 8192 bf16 112 us, so 102, quantised norm 149 and 119, 40000 x 1024 41 and 27; fp32 rows, of twice the chunks, have enough
        // on their way: 100352 x 512 quantised 40 us, so 42; nor do levels of 1024 threads gain, 4096 x 16384 bf16 42 and 46)
        if constexpr (V == 8 && NV > 0 && (THREADS < 1024 || OUT == kReal)) {
            if (whole_rows(p.x, p.x_stride, p.cols, (int)sizeof(T))) {
                row_kernel<T, P, OUT, THREADS, NV, true><<<grid, block, 0, st>>>(p);
                return hipGetLastError();
            }
        }
        row_kernel<T, P, OUT, THREADS, NV, false><<<grid, block, 0, st>>>(p);
        return hipGetLastError();
    };
    using std::integral_constant;
    if (chunks <= 64) return go(integral_constant<int, 64>(), integral_constant<int, 1>());
    if (chunks <= 128) return go(integral_constant<int, 64>(), integral_constant<int, 2>());
    if (chunks <= 256) return go(integral_constant<int, 256>(), integral_constant<int, 1>());
    // Real outputs: a chunk a thread (16384 x 4096 bf16, one row on its way: 56 us, with two 67; 16384 x 8192 118 us, with four 169).  Levels take three sums
    // or maxima over the workgroup, and fewer waves wait for each other (16384 x 4096 quantised norm, one row on its way: 63 us, with one chunk 81).
    if constexpr (OUT == kReal) {
        if (chunks <= 512) return go(integral_constant<int, 512>(), integral_constant<int, 1>());
        if (chunks <= 1024) return go(integral_constant<int, 1024>(), integral_constant<int, 1>());
    } else {
        if (chunks <= 512) return go(integral_constant<int, 256>(), integral_constant<int, 2>());
        if (chunks <= 1024) return go(integral_constant<int, 512>(), integral_constant<int, 2>());
    }
    if (chunks <= 2048) return go(integral_constant<int, 1024>(), integral_constant<int, 2>());
    // (four chunks of eight values and their parameters do not fit in registers: 2048 x 30000 bf16 208 us, read again for every sum 108 us)
    if constexpr (OUT == kQuantize || V == 4)
        if (chunks <= 4096) return go(integral_constant<int, 1024>(), integral_constant<int, 4>());
    return go(integral_constant<int, 1024>(), integral_constant<int, 0>());
}

// ------------------------------------------------------------------------------------------------
// Backward.  p = dy gamma, xh = (x - mean) rstd: dx = rstd (p - mean(p) - xh mean(p xh)), dgamma = sum over rows of dy xh,
// dbeta = sum over rows of dy.  A workgroup takes every gridDim.x-th row and keeps its columns' part of the two sums in
// registers; a second launch adds the parts in a fixed order.  Memory bounds it: x and dy read, dx written (16384 x 4096 bf16
// 89 us, 4.5 TB/s; 100000 x 512 f16 71 us, with one row on its way 109).
// ------------------------------------------------------------------------------------------------
// WHOLE: load_whole takes the rows.  Two are then on their way while one is worked on.
template <class T, class P, int THREADS, int NV, bool WHOLE>
__global__ __launch_bounds__(block_of(THREADS)) void norm_back_kernel(const NormBackArgs p)
{
    constexpr int V = Chunk<T>::kCount, ROWS = block_of(THREADS) / THREADS;
    __shared__ float slots[2][2][16];
    const int t = threadIdx.x % THREADS;
    const long long step = (long long)gridDim.x * ROWS;
    long long row = (long long)blockIdx.x * ROWS + __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS);
    float gamma[NV][V], sg[NV][V] = {}, sb[NV][V] = {};
    constexpr int DEEP = WHOLE ? 2 : 1;
    Chunk<T> nx[DEEP][NV], nd[DEEP][NV];
    float next_mean[DEEP], next_rstd[DEEP];
    auto fetch = [&](auto slot, long long r) __attribute__((always_inline)) {
        constexpr int D = decltype(slot)::value;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = (t + i * THREADS) * V;
            if constexpr (WHOLE) {
                nx[D][i] = load_whole((const T *)p.x + r * p.x_stride, r < p.rows, p.cols, at);
                nd[D][i] = load_whole((const T *)p.dy + r * p.dy_stride, r < p.rows, p.cols, at);
            } else {
                nx[D][i] = load_chunk((const T *)p.x + r * p.x_stride, at, p.cols);
                nd[D][i] = load_chunk((const T *)p.dy + r * p.dy_stride, at, p.cols);
            }
        }
        if constexpr (WHOLE) r = r < p.rows ? r : row;
        next_mean[D] = p.mean[r];
        next_rstd[D] = p.rstd[r];
    };
    using std::integral_constant;
    if (row < p.rows) {
        fetch(integral_constant<int, 0>(), row);
        if constexpr (WHOLE) fetch(integral_constant<int, 1>(), row + step);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) load_params((const P *)p.gamma, (t + i * THREADS) * V, p.cols, 1.f, gamma[i]);
    const float share = 1.f / (float)p.cols;
    auto work = [&](auto slot, int turn) __attribute__((always_inline)) {
        constexpr int D = decltype(slot)::value;
        Chunk<T> cx[NV], cd[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) cx[i] = nx[D][i], cd[i] = nd[D][i];
        const float mean = next_mean[D], rstd = next_rstd[D];
        if (WHOLE || row + step < p.rows) fetch(slot, row + DEEP * step);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < V; ++k) {       // (behind the row's end dy is 0, and with it every term)
                const float xh = ((float)cx[i].v[k] - mean) * rstd, d = (float)cd[i].v[k], pv = d * gamma[i][k];
                s1 += pv;
                s2 += pv * xh;
                sg[i][k] += d * xh;
                sb[i][k] += d;
            }
        s1 = wave_reduce(s1, Sum());
        s2 = wave_reduce(s2, Sum());
        if constexpr (THREADS > kWave) {
            if ((threadIdx.x & 63) == 0) {
                slots[turn][0][threadIdx.x >> 6] = s1;
                slots[turn][1][threadIdx.x >> 6] = s2;
            }
            __syncthreads();
            s1 = s2 = 0.f;
#pragma unroll
            for (int i = 0; i < THREADS / kWave; ++i) {
                s1 += slots[turn][0][i];
                s2 += slots[turn][1][i];
            }
        }
        s1 *= share;
        s2 *= share;
        T *dx = (T *)p.dx + row * p.dx_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = (t + i * THREADS) * V;
            if (at >= p.cols) continue;
            T out[V];
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float xh = ((float)cx[i].v[k] - mean) * rstd;
                out[k] = rounded<T>(rstd * ((float)cd[i].v[k] * gamma[i][k] - s1 - xh * s2));
            }
            store_values(dx, at, p.cols, out);
        }
    };
    if constexpr (WHOLE) {
        while (row < p.rows) {
            work(integral_constant<int, 0>(), 0);
            row += step;
            if (row >= p.rows) break;
            work(integral_constant<int, 1>(), 1);
            row += step;
        }
    } else {
        for (int turn = 0; row < p.rows; row += step, turn ^= 1) work(integral_constant<int, 0>(), turn);
    }
    if (!p.partial) return;
    float *to = p.partial + (long long)blockIdx.x * 2 * p.cols;
    if constexpr (ROWS > 1) {       // the waves' sums become the workgroup's: wave after wave, in LDS
        __shared__ float held[2][NV * THREADS * V];
        for (int w = 0; w < ROWS; ++w) {
            if ((int)threadIdx.x / THREADS == w) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        const int at = (i * V + k) * THREADS + t;
                        held[0][at] = w ? held[0][at] + sg[i][k] : sg[i][k];
                        held[1][at] = w ? held[1][at] + sb[i][k] : sb[i][k];
                    }
            }
            __syncthreads();
        }
        if ((int)threadIdx.x >= THREADS) return;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < V; ++k) sg[i][k] = held[0][(i * V + k) * THREADS + t], sb[i][k] = held[1][(i * V + k) * THREADS + t];
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = (t + i * THREADS) * V;
        if (at >= p.cols) continue;
        store_values(to, at, p.cols, sg[i]);
        store_values(to + p.cols, at, p.cols, sb[i]);
    }
}

// Rows that no workgroup holds in registers: dx from two readings, the parameters' sums by column.
constexpr int kLongThreads = 1024;
constexpr long long kMaxLongBlocks = kMaxBlocks / 2;
static_assert(kMaxLongBlocks * kLongThreads < 1LL << 32, "a launch has fewer than 2^32 threads");

template <class T, class P>
__global__ __launch_bounds__(kLongThreads) void norm_back_long_kernel(const NormBackArgs p)
{
    constexpr int V = Chunk<T>::kCount, THREADS = kLongThreads;
    __shared__ float slots[2][2][16];
    int turn = 0;
    for (long long row = blockIdx.x; row < p.rows; row += gridDim.x, turn ^= 1) {
        const T *x = (const T *)p.x + row * p.x_stride, *dy = (const T *)p.dy + row * p.dy_stride;
        const float mean = p.mean[row], rstd = p.rstd[row];
        float s1 = 0.f, s2 = 0.f;
        for (int at = threadIdx.x * V; at < p.cols; at += THREADS * V) {
            const Chunk<T> cx = load_chunk(x, at, p.cols), cd = load_chunk(dy, at, p.cols);
            float gamma[V];
            load_params((const P *)p.gamma, at, p.cols, 1.f, gamma);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float pv = (float)cd.v[k] * gamma[k];
                s1 += pv;
                s2 += pv * (((float)cx.v[k] - mean) * rstd);
            }
        }
        s1 = row_reduce<THREADS>(s1, slots[turn][0], Sum()) / (float)p.cols;
        s2 = row_reduce<THREADS>(s2, slots[turn][1], Sum()) / (float)p.cols;
        T *dx = (T *)p.dx + row * p.dx_stride;
        for (int at = threadIdx.x * V; at < p.cols; at += THREADS * V) {
            const Chunk<T> cx = load_chunk(x, at, p.cols), cd = load_chunk(dy, at, p.cols);
            float gamma[V];
            load_params((const P *)p.gamma, at, p.cols, 1.f, gamma);
            T out[V];
#pragma unroll
            for (int k = 0; k < V; ++k) out[k] = rounded<T>(rstd * ((float)cd.v[k] * gamma[k] - s1 - ((float)cx.v[k] - mean) * rstd * s2));
            store_values(dx, at, p.cols, out);
        }
    }
}

// Part b of the sums over rows b, b + parts, ...: one column a thread.
template <class T>
__global__ __launch_bounds__(kBlock) void norm_back_columns_kernel(const NormBackArgs p, int parts)
{
    const int col = blockIdx.x * kBlock + threadIdx.x;
    if (col >= p.cols) return;
    float g = 0.f, b = 0.f;
    for (long long row = blockIdx.y; row < p.rows; row += parts) {
        const float d = (float)((const T *)p.dy)[row * p.dy_stride + col];
        g += d * (((float)((const T *)p.x)[row * p.x_stride + col] - p.mean[row]) * p.rstd[row]);
        b += d;
    }
    float *to = p.partial + (long long)blockIdx.y * 2 * p.cols + col;
    to[0] = g;
    to[p.cols] = b;
}

// dgamma and dbeta from `parts` parts [part][gamma, beta][cols]: 32 columns a workgroup, eight threads a column.
template <class P>
__global__ __launch_bounds__(kBlock) void norm_back_parts_kernel(const float *partial, int parts, int cols, P *dgamma, P *dbeta)
{
    __shared__ float lds[8][33];
    const int c = threadIdx.x & 31, s = threadIdx.x >> 5;
    const long long col = (long long)blockIdx.x * 32 + c;          // over both vectors
    float v = 0.f;
    if (col < 2LL * cols) {
#pragma unroll 8
        for (int i = s; i < parts; i += 8) v += partial[(long long)i * 2 * cols + col];
    }
    lds[s][c] = v;
    __syncthreads();
    if (s == 0 && col < 2LL * cols) {
#pragma unroll
        for (int i = 1; i < 8; ++i) v += lds[i][c];
        if (col < cols) dgamma[col] = (P)v;
        else dbeta[col - cols] = (P)v;
    }
}

struct BackPlan {
    int threads, nv;            // nv 0: the long rows' kernels
    int blocks, parts;
};

BackPlan back_plan(int x_type, long long rows, int cols)
{
    const int chunks = ceil_div(cols, x_type == XNOR_TYPE_FP32 ? 4 : 8);
    BackPlan b{};
    if (chunks <= 128) b.threads = 64, b.nv = chunks <= 64 ? 1 : 2;
    else if (chunks <= 256) b.threads = 256, b.nv = 1;
    else if (chunks <= 512) b.threads = 512, b.nv = 1;
    else if (chunks <= 2048) b.threads = 1024, b.nv = chunks <= 1024 ? 1 : 2;
    if (b.nv == 0) {
        b.blocks = (int)std::min(rows, kMaxLongBlocks);
        b.parts = (int)std::max<long long>(1, std::min<long long>(rows, 64));       // (without rows too a caller's workspace is one part)
        return b;
    }
    // Two workgroups a unit, of 256 threads three: their registers, and the parts that they leave, have more run slower
    // (16384 x 4096 bf16, one row on its way: 110 us, with three 131; 16384 x 2048 50 us, with two 57); and four rows a thread, where there are fewer.
    const int rows_a_block = b.threads < kBlock ? kBlock / b.threads : 1, most = (b.threads == 256 ? 3 : 2) * kPlanUnits;
    const long long want = std::max<long long>(1, std::min<long long>(most, (rows + rows_a_block * 4 - 1) / (rows_a_block * 4)));
    b.blocks = (int)want;         // (a part each)
    b.parts = b.blocks;
    return b;
}

template <class T, class P>
hipError_t back(const NormBackArgs &p, int x_type, hipStream_t st)
{
    const BackPlan b = back_plan(x_type, p.rows, p.cols);
    int parts = p.rows ? b.parts : 0;
    if (p.rows > 0) {
        using std::integral_constant;
        auto go = [&](auto threads, auto nv) {
            constexpr int THREADS = decltype(threads)::value, NV = decltype(nv)::value;
            if constexpr (THREADS < 1024 || NV == 1)        // (what two chunks of 1024 threads hold leaves no registers for a second row)
                if (whole_rows(p.x, p.x_stride, p.cols, (int)sizeof(T)) && whole_rows(p.dy, p.dy_stride, p.cols, (int)sizeof(T))) return norm_back_kernel<T, P, THREADS, NV, true><<<dim3((unsigned)b.blocks), dim3(block_of(THREADS)), 0, st>>>(p);
            norm_back_kernel<T, P, THREADS, NV, false><<<dim3((unsigned)b.blocks), dim3(block_of(THREADS)), 0, st>>>(p);
        };
        if (b.nv == 0) {
            norm_back_long_kernel<T, P><<<dim3((unsigned)b.blocks), dim3(kLongThreads), 0, st>>>(p);
            if (p.partial) norm_back_columns_kernel<T><<<dim3(ceil_div(p.cols, kBlock), parts), dim3(kBlock), 0, st>>>(p, parts);
        } else if (b.threads == 64) {
            b.nv == 1 ? go(integral_constant<int, 64>(), integral_constant<int, 1>()) : go(integral_constant<int, 64>(), integral_constant<int, 2>());
        } else if (b.threads == 256) {
            go(integral_constant<int, 256>(), integral_constant<int, 1>());
        } else if (b.threads == 512) {
            go(integral_constant<int, 512>(), integral_constant<int, 1>());
        } else {
            b.nv == 1 ? go(integral_constant<int, 1024>(), integral_constant<int, 1>()) : go(integral_constant<int, 1024>(), integral_constant<int, 2>());
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (p.partial) {
        norm_back_parts_kernel<P><<<dim3(ceil_div(2LL * p.cols, 32)), dim3(kBlock), 0, st>>>(p.partial, parts, p.cols, (P *)p.dgamma, (P *)p.dbeta);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_quantize(const RowArgs &p, int x_type, hipStream_t st)
{
    return x_type == XNOR_TYPE_FP32  ? launch_rows<float, float, kQuantize>(p, st)
           : x_type == XNOR_TYPE_F16 ? launch_rows<f16_t, float, kQuantize>(p, st) : launch_rows<bf16_t, float, kQuantize>(p, st);
}

template <int OUT>
static hipError_t norm_forward(const RowArgs &p, int x_type, int p_type, hipStream_t st)
{
    if (x_type == XNOR_TYPE_FP32) return launch_rows<float, float, OUT>(p, st);
    if (x_type == XNOR_TYPE_F16) return p_type == XNOR_TYPE_FP32 ? launch_rows<f16_t, float, OUT>(p, st) : launch_rows<f16_t, f16_t, OUT>(p, st);
    return p_type == XNOR_TYPE_FP32 ? launch_rows<bf16_t, float, OUT>(p, st) : launch_rows<bf16_t, bf16_t, OUT>(p, st);
}

hipError_t launch_layer_norm(const RowArgs &p, int x_type, int p_type, hipStream_t st)
{
    return p.q ? norm_forward<kLevels>(p, x_type, p_type, st) : norm_forward<kReal>(p, x_type, p_type, st);
}

size_t layer_norm_bwd_workspace(int x_type, long long rows, int cols)
{
    return (size_t)back_plan(x_type, rows, cols).parts * 2 * (size_t)cols * sizeof(float);
}

hipError_t launch_layer_norm_bwd(const NormBackArgs &p, int x_type, int p_type, hipStream_t st)
{
    if (x_type == XNOR_TYPE_FP32) return back<float, float>(p, x_type, st);
    if (x_type == XNOR_TYPE_F16) return p_type == XNOR_TYPE_FP32 ? back<f16_t, float>(p, x_type, st) : back<f16_t, f16_t>(p, x_type, st);
    return p_type == XNOR_TYPE_FP32 ? back<bf16_t, float>(p, x_type, st) : back<bf16_t, bf16_t>(p, x_type, st);
}

}  // namespace xnor
