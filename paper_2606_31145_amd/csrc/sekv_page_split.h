// Float products with 4-bit codes on the matrix cores' low-precision paths, without losing the float.
//
// Scores.  The matrix instruction for codes of 4 and 6 bits takes a block of 32 of them and its exponent byte from each
// lane, at 59 times the rate of the float one (9.05 PFLOP/s and 154 TFLOP/s measured), and its products and sums are
// exact to float's last bit: both factors are small whole numbers times a power of two.  So a query's block of 32 floats
// is written as a sum of six 6-bit numbers (sign, 2 bits of exponent, 3 of mantissa, largest 7.5), each piece rounded
// from what the last one left and 2^-4 of its scale.  After six, what is left is below 2^-24 of the block's largest
// value: a rounding of that one, and for smaller values of the block a coarser one than their own.
//
// Values.  A 4-bit code with its scale is a bfloat16 number; a float weight is the sum of three, to 2^-25 of it.
//
// Measured against the float instruction on converted codes: 2048 tokens over 8192 keys, head_dim 128, 2033 us and 506
// (475 TFLOP/s), 257 over 9001 380 and 116.  A step of 32 keys and 32 rows is 1150 cycles of matrix instructions and about
// 1600 of vector ones, which now bound it; the splitting of a tile's queries takes about 3000, once.
#pragma once

#include "sekv_page_row.h"

namespace sekv {
namespace page {

constexpr int kPieces = 6;
typedef uint32_t u6v __attribute__((ext_vector_type(6)));

// Values 2 i and 2 i + 1 of a block in even and odd.  True where the scales of the later pieces would end below a
// float's exponents, and where a value is infinite, whose products have a sign: such a block's products are left to
// plain arithmetic.  NaN makes every product NaN.
struct Split32 {
    u6v piece[kPieces];
    uint32_t scale[2];                                       // exponent bytes, four a word

    typedef float f16v __attribute__((ext_vector_type(16)));
    __device__ bool init(f16v even, f16v odd) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t a = __float_as_uint(even[i]) & 0x7fffffffu, b = __float_as_uint(odd[i]) & 0x7fffffffu;
            top = top > a ? top : a;
            top = top > b ? top : b;
        }
        // the smallest E that brings the largest magnitude to at most 7.5 = 1.875 * 2^2
        constexpr uint32_t kLeast = 40;
        const bool small = top < kLeast << 23, finite = top < 0x7f800000u;
        const uint32_t E = small ? kLeast : finite ? (top >> 23) - 2 + ((top & 0x7fffffu) > 0x700000u ? 1 : 0) : 127u;
        scale[0] = finite ? E | (E - 4) << 8 | (E - 8) << 16 | (E - 12) << 24 : ~0u;      // 255: no number
        scale[1] = finite ? (E - 16) | (E - 20) << 8 : ~0u;
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const float s = pow2_of(E - 4 * p);
            u6v r = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, s);
            // the conversion writes before it has read everything: its operands live on behind it
            asm volatile("" : "+v"(r) : "v"(even), "v"(odd));
            piece[p] = r;
            typedef float f32v __attribute__((ext_vector_type(32)));
            f32v back = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(r, s);
            asm volatile("" : "+v"(back) : "v"(r));
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                even[i] -= back[2 * i];
                odd[i] -= back[2 * i + 1];
            }
        }
        return (small && top != 0) || top == 0x7f800000u;
    }
};

// 16 keys' codes times 16 queries' piece B of word W of the scales, over blocks of 32: lane (row, block).
typedef float f4v __attribute__((ext_vector_type(4)));
template <int B>
__device__ inline f4v mma_codes(const uint32_t (&k)[4], uint32_t k_scale, const u6v &q, uint32_t q_scale, f4v c) {
    typedef int i8v __attribute__((ext_vector_type(8)));
    const i8v a = {int(k[0]), int(k[1]), int(k[2]), int(k[3]), 0, 0, 0, 0};
    const i8v b = {int(q[0]), int(q[1]), int(q[2]), int(q[3]), int(q[4]), int(q[5]), 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 4, 2, 0, int(k_scale), B, int(q_scale));
}
// The sum over all pieces, the smallest first.
__device__ inline f4v mma_split(const uint32_t (&k)[4], uint32_t k_scale, const Split32 &q, f4v c) {
    c = mma_codes<1>(k, k_scale, q.piece[5], q.scale[1], c);
    c = mma_codes<0>(k, k_scale, q.piece[4], q.scale[1], c);
    c = mma_codes<3>(k, k_scale, q.piece[3], q.scale[0], c);
    c = mma_codes<2>(k, k_scale, q.piece[2], q.scale[0], c);
    c = mma_codes<1>(k, k_scale, q.piece[1], q.scale[0], c);
    return mma_codes<0>(k, k_scale, q.piece[0], q.scale[0], c);
}

// The next bfloat16 piece of two floats, which keep what it leaves.
__device__ inline uint32_t take_bf16(float &x, float &y) {
    const uint32_t w = bf16_pack(x, y);
    x -= bf16_up(w & 0xffffu);
    y -= __uint_as_float(w & 0xffff0000u);
    return w;
}

}  // namespace page
}  // namespace sekv
