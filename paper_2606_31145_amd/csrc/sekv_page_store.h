// Rows on their way into the paged token store: a lane's piece of a row and its storage forms.
#pragma once

#include "sekv_page_row.h"

namespace sekv {
namespace page {

typedef uint32_t u4v __attribute__((ext_vector_type(4)));

// The sequence of new token `tok`: the last b with start[b] <= tok (start in LDS); -1 for one that is nobody's.
__device__ inline int sequence_of(const PageTables &t, const int32_t *start, int tok) {
    if (tok >= start[t.B] || tok < start[0]) return -1;
    int lo = 0, hi = t.B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= tok) lo = mid; else hi = mid;
    }
    return tok < start[lo + 1] ? lo : -1;
}
// Position of sequence b's new token `tok`, and its pool row of head 0 (those of the other heads are a page's rows
// further on each); -1 without a place in the sequence's pages.
__device__ inline int64_t position_of(const PageTables &t, const int32_t *start, int b, int tok) {
    return int64_t(t.seq_len[b]) - start[b + 1] + tok;
}
__device__ inline int first_row(const PageTables &t, int b, int64_t pos) {
    return pos >= 0 && (pos >> t.page_shift) < t.max_pages ? pool_row(t, b, 0, int(pos)) : -1;
}

// The largest of L lanes' words, in each of them (L = 4, 8, 16, 32; a group of lanes starts at a multiple of L).
template <int L>
__device__ inline uint32_t lanes_max(uint32_t x) {
    auto with = [&](uint32_t y) { x = x > y ? x : y; };
    with(__builtin_amdgcn_mov_dpp(x, 0xB1, 0xf, 0xf, true));       // quad_perm: lane ^ 1
    with(__builtin_amdgcn_mov_dpp(x, 0x4E, 0xf, 0xf, true));       // quad_perm: lane ^ 2
    if constexpr (L >= 8) with(__builtin_amdgcn_mov_dpp(x, 0x141, 0xf, 0xf, true));    // 7 - lane of 8
    if constexpr (L >= 16) with(__builtin_amdgcn_mov_dpp(x, 0x140, 0xf, 0xf, true));   // 15 - lane of 16
    if constexpr (L >= 32) with(__shfl_xor(x, 16));
    return x;
}

// A lane's piece of a row, as new tokens hold it (16 bytes) or as kN floats: as it is stored unchanged; as floats; the bits
// of the largest magnitude as a float's (an infinity's or NaN's if there is one); four of its values as 8-bit codes, all
// of them as 4-bit codes, scaled by the power of two.
template <class T> struct Piece;
template <> struct Piece<F32> {
    static constexpr int kN = 4;
    u4v w;
    __device__ u4v raw() const { return w; }
    __device__ void up(float (&x)[4]) const {
        x[0] = __uint_as_float(w[0]); x[1] = __uint_as_float(w[1]); x[2] = __uint_as_float(w[2]); x[3] = __uint_as_float(w[3]);
    }
    __device__ uint32_t top() const {
        const uint32_t a = w[0] & 0x7fffffffu, b = w[1] & 0x7fffffffu, c = w[2] & 0x7fffffffu, d = w[3] & 0x7fffffffu;
        const uint32_t ab = a > b ? a : b, cd = c > d ? c : d;
        return ab > cd ? ab : cd;
    }
    __device__ uint32_t codes4(float scale) const {
        const uint32_t r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, __uint_as_float(w[0]), __uint_as_float(w[1]), scale, 0);
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(w[2]), __uint_as_float(w[3]), scale, 1);
    }
    __device__ uint32_t codes(int, float scale) const {
        typedef short s2v __attribute__((ext_vector_type(2)));
        s2v r = {0, 0};
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, __uint_as_float(w[0]), __uint_as_float(w[1]), scale, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, __uint_as_float(w[2]), __uint_as_float(w[3]), scale, true);
        return __builtin_bit_cast(uint32_t, r);
    }
};
template <> struct Piece<BF16> {
    static constexpr int kN = 8;
    u4v w;
    __device__ u4v raw() const { return w; }
    __device__ void up(float (&x)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bf16_up(w[i] & 0xffffu);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ uint32_t top() const {
        typedef uint16_t h2v __attribute__((ext_vector_type(2)));
        auto h = [&](int i) { return __builtin_bit_cast(h2v, w[i] & 0x7fff7fffu); };
        const h2v m = __builtin_elementwise_max(__builtin_elementwise_max(h(0), h(1)), __builtin_elementwise_max(h(2), h(3)));
        return uint32_t(m[0] > m[1] ? m[0] : m[1]) << 16;
    }
    __device__ uint32_t codes4(float scale) const {
        typedef __bf16 b2v __attribute__((ext_vector_type(2)));
        const uint32_t a = w[0], b = w[1], c = w[2], d = w[3];   // a bit cast of w[k] itself takes element 0
        uint32_t r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, __builtin_bit_cast(b2v, a), scale, 0);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(b2v, b), scale, 1);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(b2v, c), scale, 2);
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(b2v, d), scale, 3);
    }
    __device__ uint32_t codes(int i, float scale) const {
        typedef short s2v __attribute__((ext_vector_type(2)));
        typedef __bf16 b2v __attribute__((ext_vector_type(2)));
        s2v r = {0, 0};
        const uint32_t lo = w[2 * i], hi = w[2 * i + 1];     // a bit cast of w[k] itself takes element 0
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(b2v, lo), scale, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(b2v, hi), scale, true);
        return __builtin_bit_cast(uint32_t, r);
    }
};

// Values that a call has computed in float, on their way to T or fewer bits.
template <class T> struct Computed {
    static constexpr int kN = Piece<T>::kN;
    float x[kN];
    __device__ u4v raw() const {
        if constexpr (T::kBytes == 4) return u4v{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
        else return u4v{bf16_pack(x[0], x[1]), bf16_pack(x[2], x[3]), bf16_pack(x[4], x[5]), bf16_pack(x[6], x[7])};
    }
    __device__ void up(float (&y)[kN]) const {
#pragma unroll
        for (int i = 0; i < kN; ++i) y[i] = x[i];
    }
    __device__ uint32_t top() const {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const uint32_t a = __float_as_uint(x[i]) & 0x7fffffffu;
            m = m > a ? m : a;
        }
        return m;
    }
    __device__ uint32_t codes(int i, float scale) const {
        const Piece<F32> p{u4v{__float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]), __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3])}};
        return p.codes(0, scale);
    }
    __device__ uint32_t codes4(float scale) const {
        uint32_t r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], scale, 0);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], scale, 1);
        if constexpr (kN == 8) {
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], scale, 2);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], scale, 3);
        }
        return r;
    }
};

// Row `to` of a pool in storage form P, each lane its piece.
template <class Src, class P, int D>
__device__ inline void store_row(void *pool, uint8_t *scales, int to, const Src &src, int lane) {
    constexpr int N = Src::kN, L = D / N;
    if constexpr (P::kBytes >= 2) {
        __builtin_nontemporal_store(src.raw(), reinterpret_cast<u4v *>(static_cast<unsigned char *>(pool) + size_t(to) * P::row(D)) + lane);
    } else if constexpr (P::kBytes == 0) {
        constexpr int LB = P::kBlock / N;                    // lanes of a block
        const uint32_t Ex = block_exponent(lanes_max<LB>(src.top()));
        const uint32_t c = src.codes4(pow2_of(Ex));
        unsigned char *dst = static_cast<unsigned char *>(pool) + size_t(to) * P::row(D) + lane * (N / 2);
        if constexpr (N == 8) __builtin_nontemporal_store(c, reinterpret_cast<uint32_t *>(dst));
        else __builtin_nontemporal_store(uint16_t(c), reinterpret_cast<uint16_t *>(dst));
        if (lane % LB == 0) scales[size_t(to) * P::scales(D) + lane / LB] = uint8_t(Ex);
    } else {
        uint32_t c[N / 4];
        float m = __uint_as_float(lanes_max<L>(src.top()));
        uint32_t Ex = row_exponent(m);
        if (m <= 3.402823466e38f && Ex > 8) {                // the row's lanes agree
            const float scale = pow2_of(Ex);
#pragma unroll
            for (int i = 0; i < N / 4; ++i) c[i] = src.codes(i, scale);
        } else {
            // infinities or NaN, which do not count for the scale, or values so small that they may be
            // subnormal: element by element
            float x[N];
            src.up(x);
            m = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float y = fabsf(x[i]);
                m = y <= 3.402823466e38f ? fmaxf(m, y) : m;
            }
            m = __uint_as_float(lanes_max<L>(__float_as_uint(m)));
            Ex = row_exponent(m);
            const float inv = pow2_of(254u - Ex);
#pragma unroll
            for (int i = 0; i < N / 4; ++i) {
                const float y[4] = {x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
                c[i] = codes4(y, inv);
            }
        }
        unsigned char *dst = static_cast<unsigned char *>(pool) + size_t(to) * D + lane * N;
        typedef uint32_t u2v __attribute__((ext_vector_type(2)));
        if constexpr (N == 8) __builtin_nontemporal_store((u2v{c[0], c[1]}), reinterpret_cast<u2v *>(dst));
        else __builtin_nontemporal_store(c[0], reinterpret_cast<uint32_t *>(dst));
        if (lane == 0) scales[to] = uint8_t(Ex);
    }
}

}  // namespace page
}  // namespace sekv
