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

// 128 tokens x 128 rows of b, four waves of 64 x 64, rows of any alignment and length staged through registers: a step's rows are on
// their way while the one before is worked on.  Bound by those loads, which come as pieces where rows do not begin at multiples of 16 bytes (gated
// f16 777 x 2501 x 1001 27 us, 290 TFLOP/s).
template <class T, class O, int EPI>
__global__ __launch_bounds__(256, 2) void dense_tile_kernel(const DenseArgs p, int tiles_n)
{
    constexpr bool GATED = EPI == kGated || EPI == kInt8Gated;
    constexpr int TN = GATED ? 64 : 128;        // outputs n of a tile
    typedef Mat<T> X;
    __shared__ __align__(16) char lds[2][2 * 128 * kStep];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int n0 = (int)(blockIdx.x % (unsigned)tiles_n) * TN;
    const long long m0 = p.first + (long long)(blockIdx.x / (unsigned)tiles_n) * 128;
    const int wm = (wave & 1) * 64, wn = (wave >> 1) * 64;

    typename X::acc acc[4][4] = {};
    const int steps = (int)(((long long)p.K * (int)sizeof(T) + kStep - 1) / kStep), chunk = t & 7;
    const T *a[4], *b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = (t >> 3) + 32 * i;
        a[i] = (const T *)((const char *)p.a + min(m0 + r, p.M - 1) * p.lda);
        b[i] = (const T *)b_row<GATED>(p, n0, r);
    }
    Chunk<T> va[4], vb[4];
    auto fetch = [&](int s) __attribute__((always_inline)) {
        const int at = (s * kStep + chunk * 16) / (int)sizeof(T);
#pragma unroll
        for (int i = 0; i < 4; ++i) va[i] = load_chunk(a[i], at, p.K), vb[i] = load_chunk(b[i], at, p.K);
    };
    if (steps > 0) fetch(0);
    for (int s = 0; s < steps; ++s) {
        char *const la = lds[s & 1], *const lb = la + 128 * kStep;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (t >> 3) + 32 * i, to = r * kStep + ((chunk ^ (r & 7)) << 4);
            *(i32x4 *)(la + to) = __builtin_bit_cast(i32x4, va[i]);
            *(i32x4 *)(lb + to) = __builtin_bit_cast(i32x4, vb[i]);
        }
        if (s + 1 < steps) fetch(s + 1);
        // (LDS alone is waited for: the fetches are not)
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
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
// Tiles whose rows are fetched straight into LDS.  WM x WN waves share a tile of 2 P tokens x 2 P rows of b, P = 16 WM WN: 256 x 256 with
// eight waves, one workgroup a compute unit, or 128 x 128 with four.
//
// LDS holds STEPS steps of the contraction, each as four parts of P rows: the tokens' halves A0, A1 and b's B0, B1 (in the
// gated block the two matrices' rows for the same outputs).  A step is four phases, one for each pair of halves, in the order A0 X, A0 Y,
// A1 Y, A1 X with X = B0, Y = B1 in even steps and the reverse in odd ones: each phase then needs one half more than the one
// before, and reads it from LDS while the last one's instructions run:
//     phase     instructions     reads from LDS
//       0       A0 X             Y
//       1       A0 Y             A1
//       2       A1 Y             the next step's A0
//       3       A1 X             the next step's first b half (into Y's registers)
// What a phase has read is refilled in the next one with the rows of STEPS steps further on (16 bytes a lane, two instructions
// a wave and part), 4 STEPS - 1 phases before they are read; at a phase's end the 4 STEPS - 2 youngest fetches may be under way.
//
// Bound by the clock that the card's power leaves the matrix instructions, and by the phases' ends: 8192 x 8192 x 8192 on 8 bits takes 398 us (2.76
// POP/s) at 1.9 GHz, with the matrix pipes busy 68 % of the cycles and no bank conflicts; a third of its waves' cycles are waits and barriers, and two waves
// a SIMD do not always cover for each other.  16384 x 8192 x 8192 811 us over and over on the same operands, 880-965 us right after other work (2.71 and
// 2.28-2.50 POP/s); gated 4096 x 4096 x 8192 f16 430 us, bf16 417 us, 1.28 and 1.32 PFLOP/s.
// Instructions of 32 x 32 were slower: two accumulators' chains a wave depend on themselves, and their reads meet in the banks.
// ------------------------------------------------------------------------------------------------
constexpr int kFetches = 2;

typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) void lds_void;
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4_t lds_short4;
typedef int i32x2 __attribute__((ext_vector_type(2)));

// Eight bytes of each of 16 lanes are four rows of 16 values: lane i gets the four of column i.
__device__ inline i32x2 read_transposed(const lds_char *from)
{
#ifdef __HIP_DEVICE_COMPILE__        // (the host's pass does not know the builtin)
    return __builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4 *)from));
#else
    return i32x2{};
#endif
}

// 16 bytes a lane from a buffer straight into LDS, the wave's 1024 from `to` on.  As an instruction of our own beside transposing reads:
// before each of these the compiler would wait for all such fetches of its builtin.  (It reads the place in LDS from m0, one instruction after that is
// written at the earliest.)
template <class Rsrc>
__device__ inline void fetch_16(Rsrc rsrc, int at, int from, lds_char *to)
{
#ifdef __HIP_DEVICE_COMPILE__
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" : : "{m0}"((uint32_t)(uintptr_t)to), "v"(at), "s"(rsrc), "s"(from) : "memory");
#endif
}

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
    *tn = __builtin_amdgcn_readfirstlane(in / high);         // (a quotient is a vector register otherwise)
    *tm = __builtin_amdgcn_readfirstlane(group * 8 + in % high);
    return true;
}

template <int WM_, int WN_, int STEPS_, int GROUPS_>
struct Shape {
    static constexpr int WM = WM_, WN = WN_, STEPS = STEPS_, WAVES = WM * WN, ROWS = 16 * WAVES;   // ROWS: of a part
    static constexpr int GROUPS = GROUPS_;                          // groups of so many waves, a share of the contraction each
    static constexpr int RM = WN, RN = WM;                          // 16-row fragments of a part that a wave takes
    static constexpr int kPart = ROWS * kStep, kBuffer = 4 * kPart, kLds = STEPS * kBuffer;
    static constexpr int kYoung = (4 * STEPS - 2) * kFetches;
    static_assert(RN == 2 && (STEPS & (STEPS - 1)) == 0 && GROUPS <= 2, "");
};
typedef Shape<2, 4, 2, 1> Large;
typedef Shape<2, 2, 2, 1> Medium;
typedef Shape<2, 2, 2, 2> Split;

//
// TA, TB: that operand (of 16-bit values) lies with the contraction across its rows, as [K][M] or [K][N].  A part of it is then 64 rows
// of P values, and the transposing reads of LDS hand a lane its eight values along the contraction.  32 values c of row k stand
// at place c ^ across_key(k), which spreads the rows of one read over the banks.  Rows behind the contraction's end are beyond what
// the buffer's descriptor admits and arrive as zeros.
__device__ inline int across_key(int k, int places) { return places == 8 ? (k & 3) | (k >> 3 & 1) << 2 : (k >> 1 & 1) | (k >> 3 & 1) << 1; }

template <class T, class O, int EPI, class S, bool TA = false, bool TB = false>
__global__ __launch_bounds__(S::GROUPS * S::WAVES * kWave) __attribute__((amdgpu_waves_per_eu(2, 2))) void dense_direct_kernel(const DenseArgs p, const TileMap map)
{
    constexpr bool GATED = EPI == kGated || EPI == kInt8Gated;
    constexpr int PITCH = S::ROWS * 2, PLACES = PITCH / 32, DEEP = kStep / 2;       // operands across: bytes of a row, its places, rows of a step
    static_assert(!TA || TB, "");
    constexpr int ROWS = S::ROWS, RM = S::RM, RN = S::RN, kPart = S::kPart, kBuffer = S::kBuffer, STEPS = S::STEPS;
    typedef Mat<T> X;
    typedef typename X::acc Acc;
    extern __shared__ __align__(1024) char lds_all[];
    int tm, tn;
    if (!tile_of(map, &tm, &tn)) return;
    const int group = S::GROUPS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / (S::WAVES * kWave));
    const int t = S::GROUPS == 1 ? threadIdx.x : threadIdx.x % (S::WAVES * kWave);
    const int lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), r = lane & 15, g = lane >> 4;
    char *const lds = lds_all + group * S::kLds;
    const long long m0 = p.first + (long long)tm * 2 * ROWS;
    const int n0 = tn * (GATED ? ROWS : 2 * ROWS);
    const int wm = wave % S::WM * RM * 16, wn = wave / S::WM * RN * 16;
    // A group's whole steps; what is left over, whole or not, is a step more for some groups.  END: it is fetched as the others are, and what
    // it brings from behind the contraction's end is masked (the eight waves of the large tile have no registers left for that).
    constexpr bool END = S::WAVES == 4 && !TB;
    // (Operands across have no such step.)
    // (kSums: a workgroup has one of p.parts shares.)
    const int part = EPI == kSums ? blockIdx.y : 0;
    const int bytes = p.K * (int)sizeof(T), whole = (bytes + (TB ? kStep - 1 : 0)) / kStep;
    const int share = EPI == kSums ? (whole + p.parts - 1) / p.parts : (whole + (TB ? S::GROUPS - 1 : 0)) / S::GROUPS;
    const int first = (EPI == kSums ? part : group) * share, steps = EPI == kSums ? min(max(whole - first, 0), share) : share, rest = S::GROUPS * steps, left = TB ? 0 : (bytes + kStep - 1) / kStep - rest;

    // Fetches: instruction i of a wave fills rows 16 wave + 8 i + lane / 8 of a part, and the lane brings the 16 bytes that
    // belong at its place: chunk c of row r stands at place c ^ (r & 7), which spreads a column of rows over the banks.
    const char *const from_a = (const char *)p.a + m0 * (TA ? 2 : p.lda);
    const char *const from_b[2] = {(const char *)p.b + n0 * (TB ? 2 : p.ldb), (const char *)(p.b2 ? p.b2 : p.b) + n0 * (TB ? 2 : p.ldb)};
    const int last_m = (int)min(p.M - 1 - m0, 2LL * ROWS - 1), last_n = min(p.N - 1 - n0, (GATED ? 1 : 2) * ROWS - 1);
    // (END: to the end of the 16 bytes that the last row ends in; rows start at multiples of 16)
    const int upto = END ? (bytes + 15) & ~15 : bytes;
    const auto rsrc_a = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(from_a), 0, (int)(last_m * p.lda + upto), 0x00027000);
    const auto rsrc_b0 = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(from_b[0]), 0, (int)(last_n * p.ldb + upto), 0x00027000);
    const auto rsrc_b1 = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(from_b[1]), 0, (int)(last_n * p.ldb + upto), 0x00027000);
    int at_a[2][kFetches], at_b[2][kFetches];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < kFetches; ++i) {
            const int row = 16 * wave + 8 * i + (lane >> 3), chunk = ((lane & 7) ^ (lane >> 3)) * 16;
            const int l = (2 * wave + i) * 1024 + lane * 16, k = l / PITCH, c = ((l % PITCH / 16) ^ across_key(k, PLACES) << 1) * 8;
            // (operands across: 8 | M, N, so that the last 8 columns of a tile are whole)
            at_a[h][i] = TA ? k * (int)p.lda + min(h * ROWS + c, last_m - 7) * 2 : min(h * ROWS + row, last_m) * (int)p.lda + chunk;
            at_b[h][i] = TB ? k * (int)p.ldb + min(b_row_of(h, c), last_n - 7) * 2 : min(GATED ? row : b_row_of(h, row), last_n) * (int)p.ldb + chunk;
        }
    lds_char *const lds_wave = (lds_char *)lds + 16 * wave * kStep;
    const int last = steps - 1 + (END && group < left ? 1 : 0);
    // Part `part` (A0, A1, B0, B1) of a step into its buffer; of a step behind the last one, which nothing reads, the last one's.
    auto fetch = [&](auto part, int step) __attribute__((always_inline)) {
        constexpr int PART = decltype(part)::value;
        lds_char *const to = lds_wave + (step & (STEPS - 1)) * kBuffer + PART * kPart;
        const int s = min(step, last), at_step = s < steps ? first + s : rest + group;
        if constexpr (PART < 2 ? TA : TB) {
            const int k = at_step * DEEP;
            const bool second = PART >= 2 && k >= p.seam;
            // DEEP rows from `row` on: those that there are, up to the tile's last column
            const long long ld = PART < 2 ? p.lda : p.ldb;
            const int row = second ? k - p.seam : k, there = min(max((PART < 2 ? p.K : p.deep) - row, 0), DEEP);
            const int short_by = (int)ld - ((PART < 2 ? last_m : last_n) + 1) * 2;          // (the last row's columns end with the tile's)
            const int size = __builtin_amdgcn_readfirstlane(max(there * (int)ld - short_by, 0));
            const char *const from = (PART < 2 ? from_a : from_b[second]) + row * ld;
            const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(from), 0, size, 0x00027000);
#pragma unroll
            for (int i = 0; i < kFetches; ++i)
                fetch_16(rsrc, PART < 2 ? at_a[PART & 1][i] : at_b[PART & 1][i], 0, to + i * 8 * kStep);
        } else {
#pragma unroll
            for (int i = 0; i < kFetches; ++i) {
                const int at = PART < 2 ? at_a[PART & 1][i] : at_b[PART & 1][i], k = at_step * kStep;
                const auto rsrc = PART < 2 ? rsrc_a : PART == 2 ? rsrc_b0 : rsrc_b1;
                // (END: the whole offset in the lane's own, as a scalar one does not count where the buffer's end is checked)
                if constexpr (TB) fetch_16(rsrc, at, k, to + i * 8 * kStep);
                else __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void *)(to + i * 8 * kStep), 16, END ? at + k : at, END ? 0 : k, 0, 0);
            }
        }
    };
    // The lane's places in a part for the two halves of a step; a fragment is 16 rows further on.
    const uint32_t place0 = r * kStep + ((g ^ (r & 7)) << 4), place1 = place0 ^ 64;
    // ... and in a part of an operand across: four lanes a row of 16 values, four rows 16 lanes.
    const uint32_t across_row = (g * 8 + (r >> 2)) * PITCH + (r & 3) * 8, key = across_key(g * 8 + (r >> 2), PLACES);
    auto read_across = [&](const char *part, int fragment, i32x4 (&to)[2]) __attribute__((always_inline)) {
        const lds_char *const from = (const lds_char *)part + across_row + ((fragment ^ key) << 5);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const i32x2 low = read_transposed(from + h * 32 * PITCH), high = read_transposed(from + (h * 32 + 4) * PITCH);
            to[h] = i32x4{low.x, low.y, high.x, high.y};
        }
    };
    i32x4 a[2][RM][2], b[2][RN][2];
    auto read_a = [&](int h, int step) __attribute__((always_inline)) {
        const char *const all = lds + (step & (STEPS - 1)) * kBuffer + h * kPart, *const part = all + wm * kStep;
#pragma unroll
        for (int j = 0; j < RM; ++j) {
            if constexpr (TA) {
                read_across(all, wm / 16 + j, a[h][j]);
                continue;
            }
            a[h][j][0] = *(const i32x4 *)(part + place0 + j * 16 * kStep);
            a[h][j][1] = *(const i32x4 *)(part + place1 + j * 16 * kStep);
        }
    };
    auto read_b = [&](int h, int step) __attribute__((always_inline)) {
        const char *const all = lds + (step & (STEPS - 1)) * kBuffer + (2 + h) * kPart, *const part = all + wn * kStep;
#pragma unroll
        for (int j = 0; j < RN; ++j) {
            if constexpr (TB) {
                read_across(all, wn / 16 + j, b[h][j]);
                continue;
            }
            b[h][j][0] = *(const i32x4 *)(part + place0 + j * 16 * kStep);
            b[h][j][1] = *(const i32x4 *)(part + place1 + j * 16 * kStep);
        }
    };
    Acc acc[2][2][RM][RN] = {};     // [token half][b half][16 tokens][16 rows of b]
    auto multiply = [&](int ha, int hb) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < RM; ++j)
#pragma unroll
                for (int i = 0; i < RN; ++i) acc[ha][hb][j][i] = X::mul(b[hb][i][h], a[ha][j][h], acc[ha][hb][j][i]);
    };
    auto end_phase = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 2 * RM * RN; ++i) {         // reads of LDS between the matrix instructions, not before them: 1.5 to 3 %
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(S::kYoung) : "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    using std::integral_constant;
    const integral_constant<int, 0> A0{};
    const integral_constant<int, 1> A1{};
    const integral_constant<int, 2> B0{};
    const integral_constant<int, 3> B1{};

    if (steps > 0 || (END && left > 0)) {
#pragma unroll
        for (int s = 0; s < STEPS; s += 2) {
            fetch(A0, s), fetch(B0, s), fetch(B1, s), fetch(A1, s);
            fetch(A0, s + 1), fetch(B1, s + 1), fetch(B0, s + 1);
            if (s + 2 < STEPS) fetch(A1, s + 1);
        }
        end_phase();
        read_a(0, 0);
        fetch(A1, STEPS - 1);
        end_phase();
        read_b(0, 0);
        fetch(A0, STEPS);
        end_phase();
        for (int s = 0; s < steps; s += 2) {
            read_b(1, s);
            fetch(B0, s + STEPS);
            multiply(0, 0);
            end_phase();
            read_a(1, s);
            fetch(B1, s + STEPS);
            multiply(0, 1);
            end_phase();
            read_a(0, s + 1);
            fetch(A1, s + STEPS);
            multiply(1, 1);
            end_phase();
            read_b(1, s + 1);
            fetch(A0, s + 1 + STEPS);
            multiply(1, 0);
            end_phase();
            if (s + 1 >= steps) break;
            read_b(0, s + 1);
            fetch(B1, s + 1 + STEPS);
            multiply(0, 1);
            end_phase();
            read_a(1, s + 1);
            fetch(B0, s + 1 + STEPS);
            multiply(0, 0);
            end_phase();
            read_a(0, s + 2);
            fetch(A1, s + 1 + STEPS);
            multiply(1, 0);
            end_phase();
            read_b(0, s + 2);
            fetch(A0, s + 2 + STEPS);
            multiply(1, 1);
            end_phase();
        }
        asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" : : : "memory");
    }
    if constexpr (END) {
        if (group < left) {
            auto masked = [&](i32x4 (&v)[2]) __attribute__((always_inline)) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int there = min(max(bytes - ((rest + group) * kStep + (h * 4 + g) * 16 + i * 4), 0), 4);
                        v[h][i] &= there == 4 ? -1 : (1 << 8 * there) - 1;
                    }
            };
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                read_a(h, steps), read_b(h, steps);
#pragma unroll
                for (int j = 0; j < RM; ++j) masked(a[h][j]);
#pragma unroll
                for (int j = 0; j < RN; ++j) masked(b[h][j]);
            }
            multiply(0, 0), multiply(0, 1), multiply(1, 0), multiply(1, 1);
        }
    } else if (!TB && left > 0) {       // through registers
        const int chunk = t & 7, at = (rest * kStep + chunk * 16) / (int)sizeof(T);       // (zeros behind the end)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int row = (t >> 3) + 8 * S::WAVES * i, to = row * kStep + ((chunk ^ (row & 7)) << 4);
                const Chunk<T> ca = load_chunk((const T *)(from_a + (long long)min(h * ROWS + row, last_m) * p.lda), at, p.K);
                const Chunk<T> cb = load_chunk((const T *)(from_b[h] + (long long)min(GATED ? row : b_row_of(h, row), last_n) * p.ldb), at, p.K);
                *(i32x4 *)(lds + h * kPart + to) = __builtin_bit_cast(i32x4, ca);
                *(i32x4 *)(lds + (2 + h) * kPart + to) = __builtin_bit_cast(i32x4, cb);
            }
        __syncthreads();
        read_a(0, 0), read_a(1, 0), read_b(0, 0), read_b(1, 0);
        multiply(0, 0), multiply(0, 1), multiply(1, 0), multiply(1, 1);
    }
    // Two groups: each finishes one half of the tokens, with the other's sums of it.
    constexpr int HALVES = S::GROUPS == 1 ? 2 : 1;
    if constexpr (S::GROUPS == 2) {
        __syncthreads();
        Acc *const slots = (Acc *)lds_all + wave * 2 * RM * RN * kWave + lane;
#pragma unroll
        for (int hb = 0; hb < 2; ++hb)
#pragma unroll
            for (int j = 0; j < RM; ++j)
#pragma unroll
                for (int i = 0; i < RN; ++i) {
                    const int at = ((hb * RM + j) * RN + i) * kWave;
                    slots[group * S::WAVES * 2 * RM * RN * kWave + at] = group ? acc[0][hb][j][i] : acc[1][hb][j][i];
                    if (group) acc[0][hb][j][i] = acc[1][hb][j][i];
                }
        __syncthreads();
#pragma unroll
        for (int hb = 0; hb < 2; ++hb)
#pragma unroll
            for (int j = 0; j < RM; ++j)
#pragma unroll
                for (int i = 0; i < RN; ++i)
                    acc[0][hb][j][i] += slots[(1 - group) * S::WAVES * 2 * RM * RN * kWave + ((hb * RM + j) * RN + i) * kWave];
    }
    float scale[HALVES][RM];
#pragma unroll
    for (int ha = 0; ha < HALVES; ++ha)
#pragma unroll
        for (int j = 0; j < RM; ++j) scale[ha][j] = p.a_scale ? p.a_scale[min(m0 + (group + ha) * ROWS + wm + j * 16 + r, p.M - 1)] : 1.f;
    constexpr int HB = GATED ? 1 : 2;
    Columns<EPI> columns[HB][RN];
    int n[HB][RN];
#pragma unroll
    for (int hb = 0; hb < HB; ++hb)
#pragma unroll
        for (int i = 0; i < RN; ++i) {
            n[hb][i] = n0 + (GATED ? wn : b_row_of(hb, wn)) + i * 16 + g * 4;
            if (n[hb][i] < p.N) columns[hb][i].load(p, n[hb][i]);
        }
#pragma unroll
    for (int ha = 0; ha < HALVES; ++ha)
#pragma unroll
        for (int j = 0; j < RM; ++j) {
            const long long m = m0 + (group + ha) * ROWS + wm + j * 16 + r;
            if (m >= p.M) continue;
#pragma unroll
            for (int hb = 0; hb < HB; ++hb)
#pragma unroll
                for (int i = 0; i < RN; ++i)
                    if (n[hb][i] < p.N)
                        finish<T, O, EPI>(p, m + (EPI == kSums ? part * p.M : 0), scale[ha][j], n[hb][i], columns[hb][i], acc[ha][hb][j][i], acc[ha][GATED ? 1 : hb][j][i]);
        }
}

// Whether the fetches straight into LDS take the operands: rows at multiples of 16 bytes, a tile's rows within 31 bits of its first.
bool direct_supports(const DenseArgs &p, int size)
{
    auto fits = [&](const void *q, long long ld) {
        return (reinterpret_cast<uintptr_t>(q) & 15) == 0 && (ld & 15) == 0 && ld <= (0x7ffffffeLL - (long long)p.K * size) / 255;
    };
    return fits(p.a, p.lda) && fits(p.b, p.ldb) && (!p.b2 || fits(p.b2, p.ldb));
}

template <class T, class O, int EPI, class S, bool TA = false, bool TB = false>
hipError_t launch_direct(const DenseArgs &p, hipStream_t st)
{
    static std::atomic<bool> raised[64];
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= 64 || !raised[dev].load(std::memory_order_relaxed)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void *>(&dense_direct_kernel<T, O, EPI, S, TA, TB>), hipFuncAttributeMaxDynamicSharedMemorySize, S::GROUPS * S::kLds);
        if (e != hipSuccess) return e;
        if (dev >= 0 && dev < 64) raised[dev].store(true, std::memory_order_relaxed);
    }
    constexpr int TM = 2 * S::ROWS, TN = (EPI == kGated || EPI == kInt8Gated ? 1 : 2) * S::ROWS;
    TileMap map{ceil_div(p.N, TN), 0};
    // (a launch has fewer than 2^32 threads: more tokens than that gives in several)
    const long long rows = std::max<long long>(1, kMaxBlocks / map.tiles_n) * TM;
    for (long long m = 0; m < p.M; m += rows) {
        DenseArgs q = p;
        q.first = m;
        q.M = std::min(p.M, m + rows);
        map.tiles = map.tiles_n * ((q.M - m + TM - 1) / TM);
        dense_direct_kernel<T, O, EPI, S, TA, TB><<<dim3((unsigned)((map.tiles + 7) / 8 * 8), EPI == kSums ? p.parts : 1), dim3(S::GROUPS * S::WAVES * kWave), S::GROUPS * S::kLds, st>>>(q, map);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class T, class O, int EPI>
hipError_t launch_tiles(const DenseArgs &p, hipStream_t st)
{
    constexpr int TN = EPI == kGated || EPI == kInt8Gated ? 64 : 128;
    const int tiles_n = ceil_div(p.N, TN);
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

// By which tiles: `small` and `large` of them of 128 x 128 and 256 x 256.  Where a unit gets no more than one small one, two groups of
// waves share its contraction (256 x 4096 x 4096 8 bits 17.0 us, without 19.8).  Else by what the rounds of workgroups take, in steps of a
// large tile: one of these a unit, or two small ones at 0.56 of the time, a step; and some time for the tile's begin and end, which
// only two workgroups on a unit overlap.  (2048 x 4096 x 4096 8 bits 38.7 us on small tiles, 49.5 on large ones; 4096 x 4096 x 4096 70.5 and 67.9;
// 6144: 104 and 110; 16-bit gated block of 3584 x 4096 x 4096 209 and 195; 100352 x 512 x 512 8 bits 65 and 71.)
enum Tiles { kSplit, kMedium, kLarge };
Tiles tiles_of(long long small, long long large, double steps)
{
    const long long units = compute_units();
    if (small <= units) return kSplit;
    const double small_time = (double)((small + 2 * units - 1) / (2 * units)) * (0.56 * steps + 2.5);
    const double large_time = (double)((large + units - 1) / units) * (steps + 5);
    return small_time < large_time ? kMedium : kLarge;
}

template <class T, class O, int EPI, bool TA = false, bool TB = false>
hipError_t launch_by_tiles(const DenseArgs &p, hipStream_t st)
{
    constexpr int MATS = EPI == kGated || EPI == kInt8Gated ? 2 : 1;
    const long long small = ((p.M + 127) / 128) * ceil_div((long long)p.N * MATS, 128), large = ((p.M + 255) / 256) * ceil_div((long long)p.N * MATS, 256);
    switch (tiles_of(small, large, (double)p.K * sizeof(T) / kStep)) {
        case kSplit: return launch_direct<T, O, EPI, Split, TA, TB>(p, st);
        case kMedium: return launch_direct<T, O, EPI, Medium, TA, TB>(p, st);
        default: return launch_direct<T, O, EPI, Large, TA, TB>(p, st);
    }
}

// Which kernel.  Up to 16 tokens the one that reads b once; up to 64 too where it has no more than a workgroup a unit (each of them reads
// all tokens: 64 tokens x 4096 x 4096 12.3 us, on tiles 16.8; x 8192 x 8192 41 us, 28) or rows that the fetches into LDS do not take.
template <class T, class O, int EPI>
hipError_t launch(const DenseArgs &p, hipStream_t st)
{
    if (p.M == 0) return hipSuccess;
    const bool direct = direct_supports(p, sizeof(T));
    if (p.M <= 16 || (p.M <= kFewTokens && (!direct || p.N <= 16 * compute_units()))) return launch_few<T, O, EPI>(p, st);
    return direct ? launch_by_tiles<T, O, EPI>(p, st) : launch_tiles<T, O, EPI>(p, st);
}

}  // namespace

hipError_t launch_dense_across(const DenseArgs &p, bool a_across, int type, hipStream_t st)
{
    if (p.M == 0) return hipSuccess;
    if (p.parts > 1) return type == XNOR_TYPE_F16 ? launch_direct<f16_t, float, kSums, Medium, false, true>(p, st) : launch_direct<bf16_t, float, kSums, Medium, false, true>(p, st);
    if (type == XNOR_TYPE_F16) return a_across ? launch_by_tiles<f16_t, f16_t, kPlain, true, true>(p, st) : launch_by_tiles<f16_t, f16_t, kPlain, false, true>(p, st);
    return a_across ? launch_by_tiles<bf16_t, bf16_t, kPlain, true, true>(p, st) : launch_by_tiles<bf16_t, bf16_t, kPlain, false, true>(p, st);
}

bool dense_direct_supports(const DenseArgs &p, int type) { return direct_supports(p, type == XNOR_TYPE_FP32 ? 4 : 2); }

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
