// Float products with 4-bit codes on the bfloat16 matrix instruction, without losing the float.
//
// A 4-bit code with its scale is a bfloat16 number, and a float is the sum of three of them.  A query's value is cut, not
// rounded, into its 24 bits' runs of 8: nothing is left behind the third, whatever stands beside the value, and the first
// never passes the type's largest.  Weights are rounded three times, 2^-25 of each at most.  Products of bfloat16 numbers are
// exact, so what is left are the roundings of float sums.
//
// Three pieces a product still take a fifth of the float instruction's time.  2048 tokens over 8192 keys, head_dim 128: 2033 us
// with the float instruction on converted codes, 587 so (410 TFLOP/s); 257 over 9001 380 and 126.  Pieces of 6 bits that share
// a block's exponent, on the instruction for low precisions, took 506 and 112, but a value beside one 2^10 times larger
// kept 14 of its bits.
#pragma once

#include "sekv_page_row.h"

namespace sekv {
namespace page {

constexpr int kPieces = 3;

// The smallest query value whose last piece has all its bits in bfloat16's normal numbers: 2^-102.  Items with values below
// it, but for zeros, are done row by row.
constexpr uint32_t kLeastQuery = 25u << 23;
__device__ inline bool too_small(float x) { return (__float_as_uint(x) & 0x7fffffffu) - 1u < kLeastQuery - 1u; }

// Two floats' three pieces, the first value in the low halves.  An infinity is its own first piece and its others are zeros,
// so that products keep its sign; NaN is NaN.
__device__ inline void cut2(float x, float y, uint32_t (&piece)[kPieces]) {
    float v[2] = {x, y};
    uint32_t h[2][kPieces];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bool finite = fabsf(v[i]) <= 3.402823466e38f;
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            h[i][p] = __float_as_uint(v[i]) & 0xffff0000u;
            if (p == 0) h[i][p] = v[i] == v[i] ? h[i][p] : 0x7fc00000u;
            v[i] = finite ? v[i] - __uint_as_float(h[i][p]) : 0.f;
        }
    }
#pragma unroll
    for (int p = 0; p < kPieces; ++p) piece[p] = h[0][p] >> 16 | h[1][p];
}

// The next bfloat16 piece of two weights, which keep what it leaves.
__device__ inline uint32_t take_bf16(float &x, float &y) {
    const uint32_t w = bf16_pack(x, y);
    x -= bf16_up(w & 0xffffu);
    y -= __uint_as_float(w & 0xffff0000u);
    return w;
}

}  // namespace page
}  // namespace sekv
