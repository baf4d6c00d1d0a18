// Validation of the dense operators' arguments, on the host.
#pragma once

#include "dense_common.hpp"

namespace xnor {

constexpr long long kMaxRows = 0x7fffffffLL;
constexpr int kMaxCols = 1 << 26;          // a launch of a workgroup of 512 for 16 outputs has fewer than 2^32 threads

inline int value_size(int type) { return type == XNOR_TYPE_FP32 ? 4 : type == XNOR_TYPE_F16 || type == XNOR_TYPE_BF16 ? 2 : 0; }

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr long long kMaxStride = 1LL << 60;
inline bool stride_fits(long long rows, long long stride) { return stride >= 0 && (rows <= 1 || stride <= kMaxStride / rows); }

// One matrix operand of a call.
struct Matrix {
    const void *p;
    long long rows;
    int cols;
    long long stride;
    int size;           // of a value
    bool output;
};

// Status of a call's operands, in the order pointers, sizes, alignment.
template <int COUNT>
int check(const Matrix (&m)[COUNT])
{
    for (const Matrix &x : m)
        if (x.rows > 0 && !x.p) return XNOR_E_NULL;
    for (const Matrix &x : m) {
        if (x.rows < 0 || x.rows > kMaxRows || x.cols <= 0 || x.cols > kMaxCols) return XNOR_E_SHAPE;
        if (!stride_fits(x.rows, x.stride) || (x.output && x.stride < x.cols)) return XNOR_E_SHAPE;
    }
    for (const Matrix &x : m)
        if (!aligned(x.p, x.size)) return XNOR_E_ALIGN;
    return XNOR_OK;
}

inline Matrix vec(const void *p, long long n, int size, bool output = false) { return {p, n, 1, 1, size, output}; }

inline bool known_act(int act) { return act == XNOR_ACT_SILU || act == XNOR_ACT_GELU || act == XNOR_ACT_RELU; }

}  // namespace xnor
