// Rows of the paged token store on the device: element conversions and the two storage forms.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sekv_page_index.h"
#include "sekv_page_internal.h"

namespace sekv {
namespace page {

// Storage forms as template arguments: bytes of a value (0: two values a byte), of a row, and a row's exponent bytes.
struct F32 {
    using elem = float;
    static constexpr int kBytes = 4;
    static constexpr int row(int d) { return 4 * d; }
    static constexpr int scales(int) { return 0; }
};
struct BF16 {
    using elem = uint16_t;
    static constexpr int kBytes = 2;
    static constexpr int row(int d) { return 2 * d; }
    static constexpr int scales(int) { return 0; }
};
struct E4M3 {
    static constexpr int kBytes = 1;
    static constexpr int row(int d) { return d; }
    static constexpr int scales(int) { return 1; }
};
struct E2M1 {
    static constexpr int kBytes = 0, kBlock = 32;      // values that share an exponent byte
    static constexpr int row(int d) { return d / 2; }
    static constexpr int scales(int d) { return d / kBlock; }
};

__device__ inline float bf16_up(uint32_t bits) { return __uint_as_float(bits << 16); }
// two floats to bfloat16, round to nearest even, the first in the low half
__device__ inline uint32_t bf16_pack(float a, float b) {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    b2 v;
    v[0] = __bf16(a);
    v[1] = __bf16(b);
    return __builtin_bit_cast(uint32_t, v);
}
// 2^(E - 127); E in 1..254
__device__ inline float pow2_of(uint32_t E) { return __uint_as_float(E << 23); }

// The exponent byte of a row whose largest finite magnitude is a: the smallest E >= 1 with
// a <= 448 * 2^(E - 127).  448 = 1.75 * 2^8, so E follows from a's exponent field and a test of
// its mantissa; a <= max float keeps E <= 247.
__device__ inline uint32_t row_exponent(float a) {
    const uint32_t u = __float_as_uint(a);
    const int E = int(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return a > 0.f ? uint32_t(E < 1 ? 1 : E) : 127u;
}
// x * 2^(127 - E) as an e4m3 code pair, nearest even; what is not finite becomes NaN
__device__ inline uint32_t codes4(const float (&x)[4], float inv) {
    uint32_t w = 0;
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = x[i] * inv;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (!(fabsf(y[i]) <= 448.f)) w |= 0x7fu << (8 * i);
    return w;
}
// four codes as floats, scaled by 2^(E - 127) (exact)
__device__ inline void codes4_up(uint32_t w, float scale, float (&x)[4]) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, false);
    const f2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, true);
    x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
}

// two or eight codes as bfloat16, scaled by 2^(E - 127) (exact but where bfloat16 itself ends)
__device__ inline uint32_t codes2_bf16(uint32_t w, float scale, int high) {
    return high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true))
                : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
}
__device__ inline uint4 codes8_bf16(uint32_t w0, uint32_t w1, float scale) {
    return make_uint4(codes2_bf16(w0, scale, 0), codes2_bf16(w0, scale, 1), codes2_bf16(w1, scale, 0),
                      codes2_bf16(w1, scale, 1));
}

// 4 bits: codes 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign, the earlier value in a byte's low half.  The conversions take the
// scale as an exponent byte at its place in a float: 0 is 2^-127, and 255 makes NaN of any code.  Down they round to
// nearest even and keep a zero's sign; up they are exact but where the type itself ends.
// The exponent byte of a block whose largest magnitude has the bits `top`: the smallest E in 2..252 that brings it to at
// most 6 = 1.5 * 2^2 (past 252 the codes stay at 6, so that what is finite stays finite; from 2 on nothing that is stored
// is subnormal); 255 for one that holds an infinity or NaN; 127 for zeros.
__device__ inline uint32_t block_exponent(uint32_t top) {
    const int E = int(top >> 23) - 2 + ((top & 0x7fffffu) > 0x400000u ? 1 : 0);
    return top >= 0x7f800000u ? 255u : top == 0 ? 127u : uint32_t(E < 2 ? 2 : E > 252 ? 252 : E);
}
// the codes of byte I of w
template <int I>
__device__ inline uint32_t pair_bf16(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, I));
}
template <int I>
__device__ inline void pair_f32(uint32_t w, float scale, float &x, float &y) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 r = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, I);
    x = r[0];
    y = r[1];
}
// byte i of a word, i a constant after unrolling
__device__ inline uint32_t word_pair(uint32_t w, float scale, int i) {
    return i == 0 ? pair_bf16<0>(w, scale) : i == 1 ? pair_bf16<1>(w, scale) : i == 2 ? pair_bf16<2>(w, scale) : pair_bf16<3>(w, scale);
}
// eight codes
__device__ inline uint4 word_bf16(uint32_t w, float scale) {
    return make_uint4(pair_bf16<0>(w, scale), pair_bf16<1>(w, scale), pair_bf16<2>(w, scale), pair_bf16<3>(w, scale));
}

// LDS accesses of one wave complete in order; this keeps the compiler from moving one across the point where another
// lane's value is needed.
__device__ inline void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

__device__ inline void flag(const PageTables &t) {
    __hip_atomic_fetch_or(t.error, kErrPageRange, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Pool row of token `pos` (0 <= pos < max_pages * page_size) of sequence b, head g; -1 when its
// page is outside the pool.
__device__ inline int pool_row(const PageTables &t, int b, int g, int pos) {
    return block_row(t.table[size_t(b) * t.max_pages + (pos >> t.page_shift)], t.n_pages, t.Hkv, g, t.page_shift, pos);
}

}  // namespace page
}  // namespace sekv
