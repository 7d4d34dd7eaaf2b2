// 128 query rows of a workgroup against tiles of 64 keys in LDS: the bfloat16 form of
// sekv_page_attend for chunks.
//
// What bounds it: the matrix cores and the softmax's vector instructions together.  A wave takes 32
// rows; per tile it issues 32 matrix instructions (32x32x16, half scores, half values), and 2048 scores
// cost it about 4 vector instructions and one exponential each for 64 lanes (177 in all over bfloat16 pages; 254 in
// 4 bits, with the conversions and the order in which LDS is filled), so the two units are about equally busy and two
// workgroups share a compute unit to keep both fed.  Keys and values are fetched
// once per workgroup (each wave one block of 16 keys, which lies in one page), a tile ahead: bfloat16
// straight into LDS, codes of 8 and 4 bits through registers, where they become scaled bfloat16, so that the rest
// knows one type only.
//
// Measured, 2048 tokens over 32768 keys, head_dim 128, bfloat16 (1065 GFLOP): 1060 to 1150 us by the card, 925 to
// 1005 TFLOP/s, where a 16384^3 matrix product reaches 1364; in 8 bits 1081 us, in 4 bits 1063 to 1097;
// head_dim 64 665 us.
// The matrix cores are busy for 48 % of the cycles, at a clock that the load brings down to 1.95 GHz.
// The way there: 1211 us with the blocks of a tile looked up by one lane each instead of by all, 1166; the LDS reads placed among the products
// (sched_group_barrier) 1146; bfloat16 straight into LDS 1067.  No gain came from a priority for half of
// the waves (1109 against 1101), nor from starting a tile's scores before the last one's values (1126 to
// 1172 against 1124).  In copies that leave work out, the products alone take 688 us; without the exponentials it
// is 11 % faster, without the loads 10 %.
//
// LDS: rows of D values in 16-byte pieces, two buffers.  A piece sits at its index XOR a function of
// its row, so that what 64 lanes read together falls into different banks: for keys 16 rows at one
// piece, for values (turned on reading: 4 rows by 16 columns) 8 rows at 4 pieces.
#pragma once

#include "sekv_page_tile.h"

namespace sekv {
namespace page {

// Four rows of one column of a bf16 tile in LDS: within 16 lanes, lane i names 4 columns
// 4 (i % 4) of row i / 4 and receives column i of the four rows.
__device__ inline uint2 turn4(lds_bytes p) {
    typedef short s4v __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s4v *lds_p;
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)p));
}
template <int D> struct Swizzle {
    static constexpr int CH = D / 8;                   // 16-byte pieces a row
    static __device__ int key(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
    static __device__ int value(int row) {
        return D == 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
    }
};

// A wave's 16 rows of 8-bit keys and values on their way from a page into LDS, where they are bfloat16.
template <class P, int D>
struct Stage {
    static constexpr int N = D / 64;                   // 16-byte pieces a lane, keys or values
    static constexpr int PC = D / 16;                  // pieces a row
    typedef uint32_t u4v __attribute__((ext_vector_type(4)));
    u4v k[N], v[N];
    uint32_t ks[N], vs[N];

    __device__ void load(const PageAttendArgs &a, int row0, int lane) {
        const size_t r0 = row0 >= 0 ? row0 : 0;        // any row: its keys are masked
        const unsigned char *kp = static_cast<const unsigned char *>(a.k) + r0 * D;
        const unsigned char *vp = static_cast<const unsigned char *>(a.v) + r0 * D;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            k[i] = reinterpret_cast<const u4v *>(kp)[i * 64 + lane];
            v[i] = reinterpret_cast<const u4v *>(vp)[i * 64 + lane];
            ks[i] = a.k_scale[r0 + i * (64 / PC) + lane / PC];
            vs[i] = a.v_scale[r0 + i * (64 / PC) + lane / PC];
        }
    }
    // For a tile that not every row sees: values before row `from` and from row `end` on, which none sees, become
    // zeros, their exponent bytes those of one (255 makes no number of any code).  True when another holds a NaN,
    // or values that may decode to infinity: the product with its masked weight, zero, would be no number.
    __device__ bool mend(int row0, int from, int end, int lane) {
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = row0 + i * (64 / PC) + lane / PC;
            const uint32_t keep = row >= from && row < end ? ~0u : 0u;
            v[i] &= keep;
            vs[i] = keep ? vs[i] : 127u;
            bad |= uint32_t(vs[i] >= kOverExponent) | nan4(v[i].x) | nan4(v[i].y) | nan4(v[i].z) | nan4(v[i].w);
        }
        return bad != 0;
    }
    // into a tile's keys and values, rows row0 ..
    __device__ void store(unsigned char *kt, unsigned char *vt, int row0, int lane) const {
        using Z = Swizzle<D>;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = row0 + i * (64 / PC) + lane / PC, c = lane % PC;
            unsigned char *kr = kt + row * (D * 2), *vr = vt + row * (D * 2);
            const float fk = pow2_of(ks[i]), fv = pow2_of(vs[i]);
            *reinterpret_cast<uint4 *>(kr + (((2 * c) ^ Z::key(row)) << 4)) = codes8_bf16(k[i].x, k[i].y, fk);
            *reinterpret_cast<uint4 *>(kr + (((2 * c + 1) ^ Z::key(row)) << 4)) = codes8_bf16(k[i].z, k[i].w, fk);
            *reinterpret_cast<uint4 *>(vr + (((2 * c) ^ Z::value(row)) << 4)) = codes8_bf16(v[i].x, v[i].y, fv);
            *reinterpret_cast<uint4 *>(vr + (((2 * c + 1) ^ Z::value(row)) << 4)) = codes8_bf16(v[i].z, v[i].w, fv);
        }
    }
};

// The same in 4 bits: a lane holds a quarter of a row, which at head_dim 128 is a block with its own exponent byte.
template <int D>
struct Stage<E2M1, D> {
    static constexpr int W = D / 32;                   // words a lane, of eight codes each
    typedef uint32_t wv __attribute__((ext_vector_type(W)));
    wv k, v;
    uint32_t ks, vs;

    __device__ void load(const PageAttendArgs &a, int row0, int lane) {
        const size_t r0 = row0 >= 0 ? row0 : 0;        // any row: its keys are masked
        k = reinterpret_cast<const wv *>(static_cast<const unsigned char *>(a.k) + r0 * E2M1::row(D))[lane];
        v = reinterpret_cast<const wv *>(static_cast<const unsigned char *>(a.v) + r0 * E2M1::row(D))[lane];
        ks = a.k_scale[r0 * E2M1::scales(D) + lane * E2M1::scales(D) / 4];
        vs = a.v_scale[r0 * E2M1::scales(D) + lane * E2M1::scales(D) / 4];
    }
    // as above
    __device__ bool mend(int row0, int from, int end, int lane) {
        const int row = row0 + lane / 4;
        const uint32_t keep = row >= from && row < end ? ~0u : 0u;
        v &= keep;
        vs = keep ? vs : 127u;
        return vs >= kOverExponent4;
    }
    // Eight lanes, of two rows, write at a time, 16 bytes each, and the 128 bytes that they fill should not share banks.
    // So a lane takes its pieces in an order of its own: number u ^ turn in step u.  All in the order of u, with two lanes
    // (keys) or four (values) in the same banks, 2048 tokens over 32768 take 1121 us instead of 1097.  The order costs
    // 32 vector instructions a tile: the selections, and the places, which depend on the lane alone.
    __device__ static wv turned(wv x, int turn) {
        wv y;
#pragma unroll
        for (int u = 0; u < W; ++u) y[u] = turn & 1 ? x[u ^ 1] : x[u];
        if constexpr (W == 4) {
            x = y;
#pragma unroll
            for (int u = 0; u < W; ++u) y[u] = turn & 2 ? x[u ^ 2] : x[u];
        }
        return y;
    }
    __device__ void store(unsigned char *kt, unsigned char *vt, int row0, int lane) const {
        using Z = Swizzle<D>;
        const int row = row0 + lane / 4, c = lane % 4 * W;
        const int second = lane >> 2 & 1, turn_k = D == 128 ? lane & 2 : second, turn_v = D == 128 ? turn_k | second : second;
        unsigned char *kr = kt + row * (D * 2), *vr = vt + row * (D * 2);
        const float fk = pow2_of(ks), fv = pow2_of(vs);
        const wv kx = turned(k, turn_k), vx = turned(v, turn_v);
#pragma unroll
        for (int u = 0; u < W; ++u) {
            *reinterpret_cast<uint4 *>(kr + (((c + (u ^ turn_k)) ^ Z::key(row)) << 4)) = word_bf16(kx[u], fk);
            *reinterpret_cast<uint4 *>(vr + (((c + (u ^ turn_v)) ^ Z::value(row)) << 4)) = word_bf16(vx[u], fv);
        }
    }
};

// The same for bfloat16 storage without a way through registers: each lane names the 16 bytes that belong
// at its place in the tile, and the memory system writes them there.  Values are mended in the tile.
template <int D>
struct Direct {
    static constexpr int N = D / 32, PC = D / 8;       // pieces a lane; pieces a row
    int koff[N], voff[N];                              // bytes from the block's first row

    __device__ void init(int lane) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = i * (64 / PC) + lane / PC, c = lane % PC;
            koff[i] = row * (D * 2) + ((c ^ Swizzle<D>::key(row)) << 4);
            voff[i] = row * (D * 2) + ((c ^ Swizzle<D>::value(row)) << 4);
        }
    }
    // rows of pool row row0 on into the tile's rows row .. row + 15
    __device__ void load(const PageAttendArgs &a, int row0, lds_bytes kt, lds_bytes vt, int row) const {
        typedef const __attribute__((address_space(1))) void *global;
        const size_t r0 = row0 >= 0 ? row0 : 0;        // any row: its keys are masked
        const unsigned char *kp = static_cast<const unsigned char *>(a.k) + r0 * (D * 2);
        const unsigned char *vp = static_cast<const unsigned char *>(a.v) + r0 * (D * 2);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            __builtin_amdgcn_global_load_lds((global)(kp + koff[i]), kt + row * (D * 2) + i * 1024, 16, 0, 0);
            __builtin_amdgcn_global_load_lds((global)(vp + voff[i]), vt + row * (D * 2) + i * 1024, 16, 0, 0);
        }
    }
    // as Stage::mend, for the tile's rows row .. row + 15
    __device__ bool mend(unsigned char *vt, int row, int from, int end, int lane) const {
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint4 *p = reinterpret_cast<uint4 *>(vt + row * (D * 2) + i * 1024 + lane * 16);
            const int at = row + i * (64 / PC) + lane / PC;
            const uint32_t keep = at >= from && at < end ? ~0u : 0u;
            uint4 w = *p;
            w = make_uint4(w.x & keep, w.y & keep, w.z & keep, w.w & keep);
            *p = w;
            bad |= odd(w);
        }
        return bad != 0;
    }
};

// A maximum that is too large (sekv_page_tile.h) is put where no finite score moves it, and found there at the end.
// A flag beside it cost 2048 tokens over 32768 keys 1 %.
constexpr float kTooLarge = 3e38f;

template <int D>
struct Rows32 {
    static constexpr int DB = D / 32, QS = D / 16;
    uint4 q[QS];
    f16v o[DB];
    float m, l;
    int lo, hi;                         // keys that the column's query sees
    int kaddr[QS], vaddr[2][DB];        // this lane's pieces in a tile

    __device__ void init(const PageAttendArgs &a, const Item &it, int g, int row0, int lane) {
        const int n = lane & 31, h = lane >> 5, i = lane & 15, gs = a.group_shift;
        const int64_t cap = int64_t(a.t.max_pages) << a.t.page_shift;
        int row = row0 + n;
        row = row < it.rows ? row : it.rows - 1;
        const int64_t p = it.p0 + (row >> gs), w = int64_t(a.window) - 1;
        auto cut = [&](int64_t x, int64_t top) { return int(x < -1 ? -1 : x < top ? x : top); };
        lo = cut(p - w < 0 ? 0 : p - w, cap);
        hi = cut(p, cap - 1);
        const uint16_t *src = static_cast<const uint16_t *>(a.q) + int64_t(it.tok0 + (row >> gs)) * a.q_stride +
                              ((g << gs) + (row & ((1 << gs) - 1))) * D;
#pragma unroll
        for (int s = 0; s < QS; ++s) {
            q[s] = *reinterpret_cast<const uint4 *>(src + 16 * s + 8 * h);
            kaddr[s] = n * (D * 2) + (((2 * s + h) ^ Swizzle<D>::key(n)) << 4);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const int r = 8 * u + 4 * h + (i >> 2);
                const int c = 4 * db + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
                vaddr[u][db] = r * (D * 2) + ((c ^ Swizzle<D>::value(r)) << 4) + 8 * (i & 1);
            }
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[db][r] = 0.f;
    }

    // V^T operand: 32 elements from 32 db on, the 16 keys of block kb
    __device__ uint4 v_frag(lds_bytes vt, int kb, int db) const {
        const uint2 x = turn4(vt + vaddr[0][db] + kb * (32 * D)), y = turn4(vt + vaddr[1][db] + kb * (32 * D));
        return make_uint4(x.x, x.y, y.x, y.y);
    }

    // One tile: 64 keys from pos on.  part: some column may not see some key, and `valid` says which of the
    // four blocks hold keys.  The sum takes the weights before they are rounded: lse is a float.
    // The products take them in bfloat16, beside values of that type: 2048 tokens over 32768 keys are 1.98e-3 off 64
    // bits (root mean square, relative), 1.65e-3 of it the output's own rounding.  A second product with what the
    // rounding left would add half as many matrix instructions again.
    __device__ void step(const PageAttendArgs &a, lds_bytes kt, lds_bytes vt, int pos, uint32_t valid, bool part, int lane) {
        const int h = lane >> 5;
        f16v s[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[j][r] = 0.f;
#pragma unroll
            for (int c = 0; c < QS; ++c) s[j] = mma32(take16(kt + kaddr[c] + j * (64 * D)), q[c], s[j]);
        }
        // a piece of keys asked for four products ahead
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (int i = 0; i < 2 * QS - 4; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
        if (part) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int off = 32 * j + 8 * (r >> 2) + (r & 3), key = pos + off + 4 * h;
                    s[j][r] = (valid >> (off >> 4) & 1) && key >= lo && key <= hi ? s[j][r] : -INFINITY;
                }
        }
        float mx = s[0][0];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[j][r]);
        if (__any(mx * a.scale_log2 > m + kSlack)) {
            const float x = fmaxf(mx, across32(mx)) * a.scale_log2;
            float mn = fmaxf(m, x);
            mn = too_large(mn) ? kTooLarge : mn;
            const float f = exp2_fast(m - (mn == -INFINITY ? 0.f : mn));
            m = mn;
            l *= f;
#pragma unroll
            for (int db = 0; db < DB; ++db) o[db] *= f;
        }
        const float mu = m == -INFINITY ? 0.f : m;
        uint4 pf[4];
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = 8 * u + 2 * i;
                    const float x = exp2_fast(fmaf(s[j][r], a.scale_log2, -mu)), y = exp2_fast(fmaf(s[j][r + 1], a.scale_log2, -mu));
                    sum[i & 1] += x + y;
                    w[i] = bf16_pack(x, y);
                }
                pf[2 * j + u] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        l += sum[0] + sum[1];
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
            for (int db = 0; db < DB; ++db) o[db] = mma32(v_frag(vt, kb, db), pf[kb], o[db]);
        // and the values two products ahead
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (int i = 0; i < 4 * DB - 2; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
    }
};

}  // namespace page
}  // namespace sekv
