// Levels of 4 bits on their way to the matrix instructions, and how the products with them finish.
#pragma once

#include "dense_tile.hpp"
#include "experts_common.hpp"

namespace xnor {

// (a & MASK) | SET as one instruction: of its operands only one can be a scalar, so that the compiler, which keeps both constants in scalars, makes two unless one
// of them is hidden from it.  (Not an instruction written as asm: the compiler does not see what that writes, and leaves no wait before it where a matrix
// instruction in flight still has to write or read the same registers.)
template <uint32_t MASK, uint32_t SET>
__device__ inline uint32_t and_or(uint32_t a)
{
    uint32_t set = SET;
#ifdef __HIP_DEVICE_COMPILE__
    asm("" : "+v"(set));
#endif
    return (a & MASK) | set;
}

// Eight values of a word, levels less their zero point, as the operand's four registers: register j holds the values 2 j and 2 j + 1, as f16 or bf16, which hold
// them exactly.  Sums get kBack back with their group's scale.
template <class T> struct Levels;

// f16 has ten bits behind the point: a level in the lowest four of 1024's is 1024 + level, in the next four of 64's 64 + level, and a packed
// addition leaves level - zero: 9 instructions for eight values.
template <> struct Levels<f16_t> {
    static constexpr float kBack = 1.f;
    struct Zero {
        uint32_t far, near;             // -(1024 + zero), -(64 + zero), twice
    };
    static __device__ Zero zero(uint32_t z)
    {
        const uint32_t zz = z | z << 16;
        return {0xe400e400u | zz, 0xd400d400u | zz << 4};
    }
    static __device__ uint32_t add(uint32_t a, uint32_t b)
    {
        typedef f16_t f16x2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, a) + __builtin_bit_cast(f16x2, b));
    }
    static __device__ i32x4 operand(uint32_t w, const Zero &z)
    {
        const uint32_t v = w >> 8;
        return i32x4{(int)add(and_or<0x000f000fu, 0x64006400u>(w), z.far), (int)add(and_or<0x00f000f0u, 0x54005400u>(w), z.near),
                     (int)add(and_or<0x000f000fu, 0x64006400u>(v), z.far), (int)add(and_or<0x00f000f0u, 0x54005400u>(v), z.near)};
    }
};

// bf16 has no packed addition: a byte's conversion to fp32, an addition and half a packing for each value, 23 instructions for eight.  (16 + level, which takes 8,
// with a second matrix instruction that takes (16 + zero) times the tokens off, would cost sums the low bits of 31 times the largest token's magnitude, also
// where that one meets a level that is its zero point.)  Times 2^-11: sums of up to 128 times 15 tokens stay finite for tokens up to the largest.
template <> struct Levels<bf16_t> {
    static constexpr float kBack = 0x1p11f;
    struct Zero {
        float less;
    };
    static __device__ Zero zero(uint32_t z) { return {(float)z * -0x1p-11f}; }
    static __device__ i32x4 operand(uint32_t w, const Zero &z)
    {
        uint32_t even = w & 0x0f0f0f0fu, odd = w >> 4 & 0x0f0f0f0fu;
#ifdef __HIP_DEVICE_COMPILE__
        // (so that a byte's conversion is one instruction)
        asm("" : "+v"(even));
        asm("" : "+v"(odd));
#endif
        auto at = [&](uint32_t v, int byte) { return __float_as_uint(__builtin_fmaf((float)(v >> 8 * byte & 255u), 0x1p-11f, z.less)); };
        auto two = [](uint32_t low, uint32_t high) { return (int)__builtin_amdgcn_perm(high, low, 0x07060302u); };        // (small integers: no bits are lost)
        return i32x4{two(at(even, 0), at(even, 2)), two(at(odd, 0), at(odd, 2)), two(at(even, 1), at(even, 3)), two(at(odd, 1), at(odd, 3))};
    }
};

// Eight 16-bit values of a row of n from `at` on, of which those behind the row's end are zeros: the row's last eight, moved down.
template <class T>
__device__ inline i32x4 load_end(const T *row, int at, int n)
{
    if (n >= 8) {
        unsigned long long v[2];
        __builtin_memcpy(v, row + min(at, n - 8), 16);
        const int by = min(max(at - (n - 8), 0), 8), bits = 16 * (by & 3);
        unsigned long long low = by >= 8 ? 0 : by >= 4 ? v[1] : v[0], high = by >= 4 ? 0 : v[1];
        low = low >> bits | (bits ? high << (64 - bits) : 0);
        high >>= bits;
        return i32x4{(int)low, (int)(low >> 32), (int)high, (int)(high >> 32)};
    }
    T v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        v[e] = row[min(at + e, n - 1)];
        v[e] = at + e < n ? v[e] : T(0);
    }
    return __builtin_bit_cast(i32x4, v);
}

// Scales of rows n .. n + 3 in group g, 0 behind the last row.
__device__ inline void load_scales(const Int4View &w, int type, long long g, int n, int N, float (&to)[4])
{
    const long long at = g * N;
    if (type == XNOR_TYPE_FP32) load_params((const float *)w.scale + at, n, N, 0.f, to);
    else if (type == XNOR_TYPE_F16) load_params((const f16_t *)w.scale + at, n, N, 0.f, to);
    else load_params((const bf16_t *)w.scale + at, n, N, 0.f, to);
}

// The gated block's outputs from its sums.  16-bit ones by the short forms of the activations.
__device__ inline float gate(int act, bool half, float g)
{
    if (half)
        return act == XNOR_ACT_SILU ? act_value<XNOR_ACT_SILU, true>(g) : act == XNOR_ACT_GELU ? act_value<XNOR_ACT_GELU, true>(g) : act_value<XNOR_ACT_RELU, true>(g);
    return act == XNOR_ACT_SILU ? act_value<XNOR_ACT_SILU, false>(g) : act == XNOR_ACT_GELU ? act_value<XNOR_ACT_GELU, false>(g) : act_value<XNOR_ACT_RELU, false>(g);
}

// Outputs n .. n + 3 of row m, as far as the row goes, rounded once.
__device__ inline void store_outputs(const Int4Args &p, long long m, int n, const float (&v)[4])
{
    const long long at = m * p.ldo;
    if (p.out_type == XNOR_TYPE_FP32) {
        store_values((float *)p.out + at, n, p.N, v);
    } else if (p.out_type == XNOR_TYPE_F16) {
        const f16_t to[4] = {(f16_t)v[0], (f16_t)v[1], (f16_t)v[2], (f16_t)v[3]};
        store_values((f16_t *)p.out + at, n, p.N, to);
    } else {
        const bf16_t to[4] = {(bf16_t)v[0], (bf16_t)v[1], (bf16_t)v[2], (bf16_t)v[3]};
        store_values((bf16_t *)p.out + at, n, p.N, to);
    }
}

// Values n .. n + 3 of row m as the sums of p.out_terms bf16 ones, the largest first.  An infinity or a NaN is the first term, and the others are 0; a
// finite value that would round past the largest is cut instead.
__device__ inline void store_terms(const Int4Args &p, long long m, int n, const float (&v)[4])
{
    float rest[4] = {v[0], v[1], v[2], v[3]};
    bf16_t *const to = (bf16_t *)p.out + m * p.ldo;
    const int apart = hidden_stride(p.N);
#pragma unroll
    for (int t = 0; t < kMostTerms; ++t) {
        if (t >= p.out_terms) break;
        bf16_t term[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool finite = fabsf(rest[e]) <= 3.402823466e38f;
            term[e] = (bf16_t)rest[e];
            if (finite && !(fabsf((float)term[e]) <= 3.402823466e38f)) term[e] = (bf16_t)__uint_as_float(__float_as_uint(rest[e]) & 0xffff0000u);
            rest[e] = finite ? rest[e] - (float)term[e] : 0.f;
        }
        store_values(to + t * apart, n, p.N, term);
    }
}

// Matrix e of a stack.
__device__ inline Int4View of_stack(const Int4View &w, const Int4Args &p, int e)
{
    const long long groups = (p.K + p.group - 1) / p.group, values = e * groups * p.N;
    const int size = p.scale_type == XNOR_TYPE_FP32 ? 4 : 2;
    return {w.q + (long long)e * p.N * p.ldq, (const char *)w.scale + values * size, w.zero ? w.zero + values : nullptr};
}

}  // namespace xnor
