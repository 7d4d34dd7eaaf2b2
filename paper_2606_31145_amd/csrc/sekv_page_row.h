// Rows of the paged token store on the device: element conversions and the two storage forms.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sekv_page_index.h"
#include "sekv_page_internal.h"

namespace sekv {
namespace page {

// Storage forms as template arguments.
struct F32 { using elem = float; static constexpr int kBytes = 4; };
struct BF16 { using elem = uint16_t; static constexpr int kBytes = 2; };
struct E4M3 { using elem = uint8_t; static constexpr int kBytes = 1; };

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
