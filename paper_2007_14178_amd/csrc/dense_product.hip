// Products of the dense operators on the matrix cores: out = a b^T for rows of 8-bit integers, f16 or bf16, and the gated
// block's pair of products with its activation.
//
// A tile of TM tokens x TN rows of b is one workgroup's.  128 bytes of each row's contraction are staged in LDS at a time; the
// three types differ only in the instruction that takes 16 bytes a lane.  b's rows are the instruction's first operand, so that a lane
// ends up with four consecutive outputs of one token.
#include <algorithm>
#include <atomic>

#include "dense_tile.hpp"

namespace xnor {
namespace {

// 128 tokens x 128 rows of b, four waves of 64 x 64, rows of any alignment and length staged through registers.
template <class T, class O, int EPI>
__global__ __launch_bounds__(256, 2) void dense_tile_kernel(const DenseArgs p, int tiles_n)
{
    constexpr bool GATED = EPI == kGated || EPI == kInt8Gated;
    constexpr int TN = GATED ? 64 : 128;        // outputs n of a tile
    typedef Mat<T> X;
    __shared__ __align__(16) char lds[2 * 128 * kStep];
    char *la = lds, *lb = lds + 128 * kStep;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int n0 = (int)(blockIdx.x % (unsigned)tiles_n) * TN;
    const long long m0 = p.first + (long long)(blockIdx.x / (unsigned)tiles_n) * 128;
    const int wm = (wave & 1) * 64, wn = (wave >> 1) * 64;

    typename X::acc acc[4][4] = {};
    const int steps = (int)(((long long)p.K * (int)sizeof(T) + kStep - 1) / kStep);
    for (int s = 0; s < steps; ++s) {
        i32x4 va[4], vb[4];
        const int chunk = t & 7, at = (s * kStep + chunk * 16) / (int)sizeof(T);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (t >> 3) + 32 * i;
            const long long m = m0 + r < p.M ? m0 + r : p.M - 1;
            const Chunk<T> ca = load_chunk((const T *)((const char *)p.a + m * p.lda), at, p.K);
            const Chunk<T> cb = load_chunk((const T *)b_row<GATED>(p, n0, r), at, p.K);
            va[i] = __builtin_bit_cast(i32x4, ca);
            vb[i] = __builtin_bit_cast(i32x4, cb);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (t >> 3) + 32 * i, to = r * kStep + ((chunk ^ (r & 7)) << 4);
            *(i32x4 *)(la + to) = va[i];
            *(i32x4 *)(lb + to) = vb[i];
        }
        __syncthreads();
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
                for (int j = 0; j < 4; ++j) acc[i][j] = X::mul(fb[i], fa[j], acc[i][j]);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; i += GATED ? 2 : 1) {
        const int n = n0 + (GATED ? wn / 2 + i * 8 : wn + i * 16) + (lane >> 4) * 4;
        if (n >= p.N) continue;
        Columns<EPI> columns;
        columns.load(p, n);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const long long m = m0 + wm + j * 16 + (lane & 15);
            if (m < p.M) finish<T, O, EPI>(p, m, p.a_scale ? p.a_scale[m] : 1.f, n, columns, acc[i][j], acc[GATED ? i + 1 : i][j]);
        }
    }
}

// ------------------------------------------------------------------------------------------------
// 256 tokens x 256 rows of b, eight waves of 128 x 64 (64 x 32 of each quarter), one workgroup a compute unit.
//
// LDS holds two steps of the contraction, each as four parts of 128 rows: the tokens' halves A0, A1 and b's B0, B1 (in the
// gated block the two matrices' rows for the same outputs).  A step is four phases of 16 matrix instructions a wave, one for each pair
// of halves, in the order A0 P, A0 Q, A1 Q, A1 P with P = B0, Q = B1 in even steps and the reverse in odd ones: each phase then
// needs one half more than the one before, and reads it from LDS while the last one's instructions run:
//     phase     instructions     reads from LDS     its LDS part is refilled in
//       0       A0 P             Q                  the next phase
//       1       A0 Q             A1                 the next phase
//       2       A1 Q             the next A0        the next phase
//       3       A1 P             the next step's first b half (this step's Q place)
// A part's rows are fetched seven phases before they are read, straight into LDS (16 bytes a lane, two instructions a wave and
// part); at a phase's end six younger fetches may be under way, and that is what the wave waits for.
// ------------------------------------------------------------------------------------------------
constexpr int kPart = 128 * kStep, kBuffer = 4 * kPart, kFetches = 2;

typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) void lds_void;

// Row r of b's part `half`: each wave's 32 rows of both parts are 64 consecutive ones of the tile, so that a wave's outputs of a token
// are 64 consecutive values.
__device__ inline int b_row_of(int half, int r) { return (r >> 5) * 64 + half * 32 + (r & 31); }

struct TileMap {
    int tiles_n;
    long long tiles;        // of the launch
};

// The tile of a workgroup.  Workgroups go round the eight XCDs by their index: each XCD takes a run of consecutive tiles, in groups
// of eight rows of tiles, so that what its units work on at a time shares rows of both operands in its L2.
__device__ inline bool tile_of(const TileMap &t, int *tm, int *tn)
{
    const long long eighth = (t.tiles + 7) >> 3, i = (blockIdx.x & 7) * eighth + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= eighth || i >= t.tiles) return false;
    const int rows = (int)(t.tiles / t.tiles_n), group = (int)(i / (8 * t.tiles_n)), in = (int)(i - (long long)group * 8 * t.tiles_n);
    const int high = min(8, rows - group * 8);
    *tn = in / high;
    *tm = group * 8 + in % high;
    return true;
}

template <class T, class O, int EPI>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void dense_large_kernel(const DenseArgs p, const TileMap map)
{
    constexpr bool GATED = EPI == kGated || EPI == kInt8Gated;
    typedef Mat<T> X;
    typedef typename X::acc Acc;
    extern __shared__ __align__(1024) char lds[];
    int tm, tn;
    if (!tile_of(map, &tm, &tn)) return;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), r = lane & 15, g = lane >> 4;
    const long long m0 = p.first + (long long)tm * 256;
    const int n0 = tn * (GATED ? 128 : 256);
    const int wm = (wave & 1) * 64, wn = (wave >> 1) * 32;
    const int bytes = p.K * (int)sizeof(T), steps = bytes / kStep;

    // Fetches: instruction i of a wave fills rows 16 wave + 8 i + lane / 8 of a part, and the lane brings the 16 bytes that
    // belong at its place: chunk c of row r stands at place c ^ (r & 7), which spreads a column of rows over the banks.
    const char *const from_a = (const char *)p.a + m0 * p.lda;
    const char *const from_b[2] = {(const char *)p.b + (long long)n0 * p.ldb, GATED ? (const char *)p.b2 + (long long)n0 * p.ldb : (const char *)p.b + (long long)n0 * p.ldb};
    const int last_m = (int)min(p.M - 1 - m0, 255LL), last_n = min(p.N - 1 - n0, GATED ? 127 : 255);
    const auto rsrc_a = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(from_a), 0, (int)(last_m * p.lda + bytes), 0x00027000);
    const auto rsrc_b0 = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(from_b[0]), 0, (int)(last_n * p.ldb + bytes), 0x00027000);
    const auto rsrc_b1 = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(from_b[1]), 0, (int)(last_n * p.ldb + bytes), 0x00027000);
    int at_a[2][kFetches], at_b[2][kFetches];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < kFetches; ++i) {
            const int row = 16 * wave + 8 * i + (lane >> 3), chunk = ((lane & 7) ^ (lane >> 3)) * 16;
            at_a[h][i] = min(h * 128 + row, last_m) * (int)p.lda + chunk;
            at_b[h][i] = min(GATED ? row : b_row_of(h, row), last_n) * (int)p.ldb + chunk;
        }
    lds_char *const lds_wave = (lds_char *)lds + 16 * wave * kStep;
    // Part `part` (A0, A1, B0, B1) of a step into buffer step & 1; of a step behind the last one, which nothing reads, the last one's.
    auto fetch = [&](auto part, int step) __attribute__((always_inline)) {
        constexpr int PART = decltype(part)::value;
        lds_char *const to = lds_wave + (step & 1) * kBuffer + PART * kPart;
        const int k = min(step, steps - 1) * kStep;
#pragma unroll
        for (int i = 0; i < kFetches; ++i) {
            const int at = PART < 2 ? at_a[PART & 1][i] : at_b[PART & 1][i];
            const auto rsrc = PART < 2 ? rsrc_a : PART == 2 ? rsrc_b0 : rsrc_b1;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void *)(to + i * 8 * kStep), 16, at, k, 0, 0);
        }
    };
    // The lane's places in a part for the two halves of a step; a fragment is 16 rows further on.
    const uint32_t place0 = r * kStep + ((g ^ (r & 7)) << 4), place1 = place0 ^ 64;
    i32x4 a[2][4][2], b[2][2][2];
    auto read_a = [&](int h, int buffer) __attribute__((always_inline)) {
        const char *part = lds + buffer * kBuffer + h * kPart + wm * kStep;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            a[h][j][0] = *(const i32x4 *)(part + place0 + j * 16 * kStep);
            a[h][j][1] = *(const i32x4 *)(part + place1 + j * 16 * kStep);
        }
    };
    auto read_b = [&](int h, int buffer) __attribute__((always_inline)) {
        const char *part = lds + buffer * kBuffer + (2 + h) * kPart + wn * kStep;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            b[h][j][0] = *(const i32x4 *)(part + place0 + j * 16 * kStep);
            b[h][j][1] = *(const i32x4 *)(part + place1 + j * 16 * kStep);
        }
    };
    Acc acc[2][2][4][2] = {};       // [token half][b half][16 tokens][16 rows of b]
    auto multiply = [&](int ha, int hb) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i) acc[ha][hb][j][i] = X::mul(b[hb][i][h], a[ha][j][h], acc[ha][hb][j][i]);
    };
    auto end_phase = [&]() __attribute__((always_inline)) {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(12) lgkmcnt(0)\n\ts_barrier" : : : "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    using std::integral_constant;
    const integral_constant<int, 0> A0{};
    const integral_constant<int, 1> A1{};
    const integral_constant<int, 2> B0{};
    const integral_constant<int, 3> B1{};

    if (steps > 0) {
        fetch(A0, 0), fetch(B0, 0), fetch(B1, 0), fetch(A1, 0), fetch(A0, 1), fetch(B1, 1), fetch(B0, 1);
        end_phase();
        read_a(0, 0);
        fetch(A1, 1);
        end_phase();
        read_b(0, 0);
        fetch(A0, 2);
        end_phase();
        for (int s = 0; s < steps; s += 2) {
            read_b(1, 0);
            fetch(B0, s + 2);
            multiply(0, 0);
            end_phase();
            read_a(1, 0);
            fetch(B1, s + 2);
            multiply(0, 1);
            end_phase();
            read_a(0, 1);
            fetch(A1, s + 2);
            multiply(1, 1);
            end_phase();
            read_b(1, 1);
            fetch(A0, s + 3);
            multiply(1, 0);
            end_phase();
            if (s + 1 >= steps) break;
            read_b(0, 1);
            fetch(B1, s + 3);
            multiply(0, 1);
            end_phase();
            read_a(1, 1);
            fetch(B0, s + 3);
            multiply(0, 0);
            end_phase();
            read_a(0, 0);
            fetch(A1, s + 3);
            multiply(1, 0);
            end_phase();
            read_b(0, 0);
            fetch(A0, s + 4);
            multiply(1, 1);
            end_phase();
        }
        asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" : : : "memory");
    }
    if (steps * kStep < bytes) {        // the contraction's end, through registers
        const int chunk = t & 7, at = (steps * kStep + chunk * 16) / (int)sizeof(T);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = (t >> 3) + 64 * i, to = (row >> 7) * kPart + (row & 127) * kStep + ((chunk ^ (row & 7)) << 4);
            const Chunk<T> ca = load_chunk((const T *)(from_a + (long long)min(row, last_m) * p.lda), at, p.K);
            const Chunk<T> cb = load_chunk((const T *)(from_b[row >> 7] + (long long)min(GATED ? row & 127 : b_row_of(row >> 7, row & 127), last_n) * p.ldb), at, p.K);
            *(i32x4 *)(lds + to) = __builtin_bit_cast(i32x4, ca);
            *(i32x4 *)(lds + 2 * kPart + to) = __builtin_bit_cast(i32x4, cb);
        }
        __syncthreads();
        read_a(0, 0), read_a(1, 0), read_b(0, 0), read_b(1, 0);
        multiply(0, 0), multiply(0, 1), multiply(1, 0), multiply(1, 1);
    }
    float scale[2][4];
#pragma unroll
    for (int ha = 0; ha < 2; ++ha)
#pragma unroll
        for (int j = 0; j < 4; ++j) scale[ha][j] = p.a_scale ? p.a_scale[min(m0 + ha * 128 + wm + j * 16 + r, p.M - 1)] : 1.f;
    constexpr int HB = GATED ? 1 : 2;
    Columns<EPI> columns[HB][2];
    int n[HB][2];
#pragma unroll
    for (int hb = 0; hb < HB; ++hb)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            n[hb][i] = n0 + (GATED ? wn : b_row_of(hb, wn)) + i * 16 + g * 4;
            if (n[hb][i] < p.N) columns[hb][i].load(p, n[hb][i]);
        }
#pragma unroll
    for (int ha = 0; ha < 2; ++ha)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const long long m = m0 + ha * 128 + wm + j * 16 + r;
            if (m >= p.M) continue;
#pragma unroll
            for (int hb = 0; hb < HB; ++hb)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (n[hb][i] < p.N) finish<T, O, EPI>(p, m, scale[ha][j], n[hb][i], columns[hb][i], acc[ha][hb][j][i], acc[ha][GATED ? 1 : hb][j][i]);
        }
}

// Whether the fetches straight into LDS take the operands: rows at multiples of 16 bytes, a tile's rows within 31 bits of its first.
bool large_supports(const DenseArgs &p, int size)
{
    auto fits = [&](const void *q, long long ld) {
        return (reinterpret_cast<uintptr_t>(q) & 15) == 0 && (ld & 15) == 0 && 255 * ld + (long long)p.K * size < 0x7fffffffLL;
    };
    return fits(p.a, p.lda) && fits(p.b, p.ldb) && (!p.b2 || fits(p.b2, p.ldb));
}

template <class T, class O, int EPI>
hipError_t launch_large(const DenseArgs &p, hipStream_t st)
{
    static std::atomic<bool> raised[64];
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= 64 || !raised[dev].load(std::memory_order_relaxed)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void *>(&dense_large_kernel<T, O, EPI>), hipFuncAttributeMaxDynamicSharedMemorySize, 2 * kBuffer);
        if (e != hipSuccess) return e;
        if (dev >= 0 && dev < 64) raised[dev].store(true, std::memory_order_relaxed);
    }
    constexpr int TN = EPI == kGated || EPI == kInt8Gated ? 128 : 256;
    TileMap map{ceil_div(p.N, TN), 0};
    const long long rows = std::max<long long>(1, kMaxBlocks / map.tiles_n) * 256;
    for (long long m = 0; m < p.M; m += rows) {
        DenseArgs q = p;
        q.first = m;
        q.M = std::min(p.M, m + rows);
        map.tiles = map.tiles_n * ((q.M - m + 255) / 256);
        dense_large_kernel<T, O, EPI><<<dim3((unsigned)((map.tiles + 7) / 8 * 8)), dim3(512), 2 * kBuffer, st>>>(q, map);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class T, class O, int EPI>
hipError_t launch(const DenseArgs &p, hipStream_t st)
{
    constexpr int TN = EPI == kGated || EPI == kInt8Gated ? 64 : 128;
    if (p.M == 0) return hipSuccess;
    if (p.M <= kFewTokens) return launch_few<T, O, EPI>(p, st);
    if (large_supports(p, sizeof(T)) && p.M * (long long)p.N >= 256LL * 256 * 128) return launch_large<T, O, EPI>(p, st);
    const int tiles_n = ceil_div(p.N, TN);
    // (a launch has fewer than 2^32 threads: more tokens than that gives in several)
    const long long rows = std::max<long long>(1, kMaxBlocks / tiles_n) * 128;
    for (long long m = 0; m < p.M; m += rows) {
        DenseArgs q = p;
        q.first = m;
        q.M = std::min(p.M, m + rows);
        dense_tile_kernel<T, O, EPI><<<dim3((unsigned)(tiles_n * ((q.M - m + 127) / 128))), dim3(256), 0, st>>>(q, tiles_n);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_dense(const DenseArgs &p, int type, hipStream_t st)
{
    return type == XNOR_TYPE_F16 ? launch<f16_t, f16_t, kPlain>(p, st) : launch<bf16_t, bf16_t, kPlain>(p, st);
}

hipError_t launch_dense_gated(const DenseArgs &p, int type, hipStream_t st)
{
    return type == XNOR_TYPE_F16 ? launch<f16_t, f16_t, kGated>(p, st) : launch<bf16_t, bf16_t, kGated>(p, st);
}

hipError_t launch_dense_int8(const DenseArgs &p, int out_type, hipStream_t st)
{
    return out_type == XNOR_TYPE_FP32  ? launch<int8_t, float, kInt8>(p, st)
           : out_type == XNOR_TYPE_F16 ? launch<int8_t, f16_t, kInt8>(p, st) : launch<int8_t, bf16_t, kInt8>(p, st);
}

hipError_t launch_dense_int8_gated(const DenseArgs &p, int out_type, hipStream_t st)
{
    return out_type == XNOR_TYPE_FP32  ? launch<int8_t, float, kInt8Gated>(p, st)
           : out_type == XNOR_TYPE_F16 ? launch<int8_t, f16_t, kInt8Gated>(p, st) : launch<int8_t, bf16_t, kInt8Gated>(p, st);
}

}  // namespace xnor
