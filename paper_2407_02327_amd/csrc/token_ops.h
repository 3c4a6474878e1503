// What the operators with a scale for each token share: the codes' layouts, the scale of a slice, and where the rows of a set (an
// expert's tokens) lie.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"

namespace qsync {

// Codes lie in rows padded with zeros to whole K tiles of the matrix kernels, which then have no remainder to mask.
constexpr int64_t kCodePad = 128;
__host__ __device__ constexpr int64_t code_pad(int64_t n) { return (n + kCodePad - 1) / kCodePad * kCodePad; }

namespace {

// A row or column of values and what its codes stand for.  Its largest magnitude comes as fp32 bits without the sign, which order like
// the values, infinities and NaN behind them.  Below 2^-100 the inverse could overflow and products of two scales lose bits: such a
// slice counts as zero.  One that is not finite has a NaN for its scale, so every output it takes part in is NaN, and codes of 0.
struct CodeScale { float scale, inv; };
__device__ __forceinline__ CodeScale code_scale(uint32_t amax_bits)
{
    if(amax_bits >= 0x7F800000u) return {__uint_as_float(0x7FC00000u), 0.0f};
    if(amax_bits < 0x0D800000u) return {1.0f, 0.0f};      // 2^-100
    const float a = __uint_as_float(amax_bits);
    return {a / 127.0f, 127.0f / a};
}
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// The rows of set e: [first, first + len).  Offsets come from device memory: whatever they hold, the rows lie in [0, rows) and the
// positions below in the buffers.
struct SetRows { int64_t first, len; };
__device__ __forceinline__ SetRows set_rows(const int32_t* offsets, int64_t rows, int64_t sets, int64_t e)
{
    if(!offsets) return {rows / sets * e, rows / sets};
    int64_t a = offsets[e], b = offsets[e + 1];
    a = a < 0 ? 0 : a > rows ? rows : a;
    b = b < a ? a : b > rows ? rows : b;
    return {a, b - a};
}
// Codes whose contraction axis is the rows (weight gradients) hold the sets one behind the other, each a packed matrix [cols][code_pad(len)]:
// set e's starts at position code_pad(first) + 128 e of the rows' axis (times cols).  A position's set is found from the offsets alone, and
// no two overlap: code_pad(f) + code_pad(len) <= code_pad(f + len) + 128.  Sets of the same known size lie without gaps.
__device__ __forceinline__ int64_t set_start(const int32_t* offsets, const SetRows& s, int64_t e)
{
    return offsets ? code_pad(s.first) + kCodePad * e : code_pad(s.len) * e;
}

}  // namespace

__host__ __device__ inline int64_t code_positions(int64_t rows, int64_t sets, bool offsets)
{
    return offsets ? code_pad(rows) + kCodePad * sets : code_pad(rows / sets) * sets;
}

}  // namespace qsync
