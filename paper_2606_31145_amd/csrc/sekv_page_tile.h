// Building blocks of sekv_page_attend on the matrix cores.
//
// Scores are formed transposed, S^T = K Q^T: a lane holds the scores of one query row (column
// lane % 16 or % 32 of the result) against several keys, so the softmax's maximum and sum are per
// lane but for one exchange between the lanes of a column, and the weights already lie as the
// second operand of O^T += V^T P^T wants them: the contraction runs over keys in the order in which
// the first product leaves them, and V is read in that same order.
//
// The running maximum is moved only when a score passes it by more than kSlack (in base 2): weights
// then reach 2^8 at most instead of 1, which float sums do not mind, and most tiles need neither an
// exchange nor a rescaling of the output.  Without the slack 257 tokens over 9001 keys take 63.7 us instead of
// 61.4, 9 ragged sequences, one of 300 tokens, 430 instead of 417.
#pragma once

#include "sekv_page_index.h"
#include "sekv_page_row.h"

namespace sekv {
namespace page {

typedef float f4v __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef __bf16 b8v __attribute__((ext_vector_type(8)));

constexpr float kSlack = 8.f;

// A weight is exp2(score * scale_log2 - m) in one fused step, while m is the rounded product of the largest score: that
// one's weight is 2 to the product's rounding error instead of 1.  The error is common to all weights and does no
// harm while it is small.  Past kLargest it may be more than 4: an item that meets such a maximum is done row by row
// instead, with rounded products on both sides (plain_rows).  Infinite maxima make no number either way.
constexpr float kLargest = 67108864.f;
__device__ inline bool too_large(float m) {                  // kLargest < |m| < infinity, without branches
    return (__float_as_uint(m) & 0x7fffffffu) - 0x4c800001u < 0x7f800000u - 0x4c800001u;
}

__device__ inline f4v mma16(const uint4 &a, const uint4 &b, f4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8v, a), __builtin_bit_cast(b8v, b), c, 0, 0, 0);
}
__device__ inline f4v mma16(float a, float b, f4v c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
__device__ inline f16v mma32(const uint4 &a, const uint4 &b, f16v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8v, a), __builtin_bit_cast(b8v, b), c, 0, 0, 0);
}
__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The value of the lane 32 or 16 away.
__device__ inline float across32(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}
__device__ inline float across16(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float((threadIdx.x & 16) ? r[0] : r[1]);
}

// Is an element not finite (bfloat16 pairs; float).
__device__ inline uint32_t odd2(uint32_t w) { return uint32_t((w & 0x7f80u) == 0x7f80u) | uint32_t((w & 0x7f800000u) == 0x7f800000u); }
__device__ inline uint32_t odd(const uint4 &v) { return odd2(v.x) | odd2(v.y) | odd2(v.z) | odd2(v.w); }
__device__ inline bool odd(float x) { return !(fabsf(x) <= 3.402823466e38f); }
// The first exponent byte whose rows may decode to infinities: 256 * 2^120 is past float and bfloat16.
constexpr uint32_t kOverExponent = 247;
// Is one of four e4m3 codes a NaN.
__device__ inline uint32_t nan4(uint32_t w) {
    const uint32_t x = ~w & 0x7f7f7f7fu;               // a zero byte: NaN
    return (x - 0x01010101u) & ~x & 0x80808080u;
}

__device__ inline Seq load_seq(const PageAttendArgs &a, int b) {
    const PageTables &t = a.t;
    return make_seq(t.tok_start[b], t.tok_start[b + 1], t.seq_len[b], t.n_tokens, int64_t(t.max_pages) << t.page_shift,
                    a.window, a.group_shift);
}

// One lane's sequence in all lanes.
__device__ inline Seq of_lane(const Seq &s, int l) {
    Seq r;
    r.start = __builtin_amdgcn_readlane(s.start, l);
    r.nq = __builtin_amdgcn_readlane(s.nq, l);
    r.first = int64_t(uint32_t(__builtin_amdgcn_readlane(uint32_t(s.first), l)) |
                      uint64_t(uint32_t(__builtin_amdgcn_readlane(uint32_t(uint64_t(s.first) >> 32), l))) << 32);
    r.lo = __builtin_amdgcn_readlane(s.lo, l);
    r.len = __builtin_amdgcn_readlane(s.len, l);
    r.tiles = __builtin_amdgcn_readlane(s.tiles, l);
    return r;
}

// What a workgroup finds out about the call.  Up to 64 sequences are one a lane, and every wave does it for itself;
// of more, a thread takes B / 256 consecutive ones, twice, and the threads meet in LDS (4096 sequences of 300
// tokens 873 us, with 64 at a time in every wave 2011).
struct Plan {
    Seq mine;             // sequence `lane` of up to 64
    int chunk;            // 0 where tok_start does not ascend within the new tokens: rows could then belong to
                          // two sequences, and a tile's counter to two tiles
    int tiles, longest;   // of a KV head; keys of the longest sequence (where chunks may be cut)
};

// lds: 256 bytes, free again on return.
__device__ inline Plan make_plan(const PageAttendArgs &a, bool is_float, int lane, unsigned char *lds) {
    Plan p;
    uint64_t W = 0;
    int mx = 0, T = 0;
    bool wrong = false;
    auto count = [&](int b) {
        const int from = a.t.tok_start[b], to = a.t.tok_start[b + 1];
        const Seq s = make_seq(from, to, a.t.seq_len[b], a.t.n_tokens, int64_t(a.t.max_pages) << a.t.page_shift, a.window,
                               a.group_shift);
        wrong |= from != s.start || to != s.start + s.nq;
        W += uint64_t(s.tiles) * uint64_t(s.len);
        T += s.tiles;
        mx = mx > s.len ? mx : s.len;
        return s;
    };
    const bool many = a.t.B > 64;
    if (!many && lane < a.t.B) p.mine = count(lane);
    p.chunk = 1 << 30;
    if (a.splits == 1) return p;
    if (many) {
        const int per = (a.t.B + 255) / 256, b0 = threadIdx.x * per, b1 = b0 + per < a.t.B ? b0 + per : a.t.B;
#pragma unroll 4
        for (int b = b0; b < b1; ++b) count(b);
    }
    if (a.t.B > 1) {
#pragma unroll
        for (int k = 1; k < 64; k *= 2) {
            W += __shfl_xor((unsigned long long)W, k);
            T += __shfl_xor(T, k);
            const int y = __shfl_xor(mx, k);
            mx = mx > y ? mx : y;
        }
    }
    wrong = __any(wrong);
    if (many) {
        struct Part { uint64_t W; int T, mx, wrong, pad; };
        Part *part = reinterpret_cast<Part *>(lds);
        if (lane == 0) part[threadIdx.x >> 6] = Part{W, T, mx, wrong, 0};
        __syncthreads();
        W = 0;
        T = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            W += part[w].W;
            T += part[w].T;
            mx = mx > part[w].mx ? mx : part[w].mx;
            wrong |= part[w].wrong != 0;
        }
        __syncthreads();
    }
    p.chunk = 0;
    if (wrong) return p;
    W = __builtin_amdgcn_readfirstlane(uint32_t(W)) | uint64_t(__builtin_amdgcn_readfirstlane(uint32_t(W >> 32))) << 32;
    p.tiles = __builtin_amdgcn_readfirstlane(T);
    p.longest = __builtin_amdgcn_readfirstlane(mx);
    p.chunk = chunk_length(W, p.tiles, p.longest, a.t.Hkv, a.target, a.splits, over_of(a.join_launch, is_float),
                           join_rows_of(a.join_launch, a.t.n_tokens, a.group_shift, p.tiles));
    return p;
}

// Pair x of the call: sequences in order, chunks of a sequence in order, tiles last first (the later
// tokens of a chunk see more keys).  kTiles: tile x instead, as its first chunk's item.  x and so the result are
// the same in all threads.  lds as above.
template <bool kTiles = false>
__device__ inline bool find_item(const PageAttendArgs &a, uint32_t x, int lane, const Plan &p, unsigned char *lds, int *b_out,
                                 int *c_out, Item *it) {
    const int64_t cap = int64_t(a.t.max_pages) << a.t.page_shift;
    auto pairs = [&](const Seq &s) { return uint32_t(s.tiles) * uint32_t(kTiles ? 1 : chunks_of(s, p.chunk)); };
    const bool many = a.t.B > 64;
    const int per = (a.t.B + 255) / 256, b0 = threadIdx.x * per, b1 = b0 + per < a.t.B ? b0 + per : a.t.B;
    uint32_t n = 0;
    if (many) {
#pragma unroll 4
        for (int b = b0; b < b1; ++b) n += pairs(load_seq(a, b));
    } else if (lane < a.t.B) {
        n = pairs(p.mine);
    }
    uint32_t incl = n;
    if (a.t.B > 1) {
#pragma unroll
        for (int k = 1; k < 64; k *= 2) {
            const uint32_t y = __shfl_up(incl, k);
            incl += lane >= k ? y : 0u;
        }
    }
    Seq s;
    uint32_t in;
    if (many) {
        uint32_t *total = reinterpret_cast<uint32_t *>(lds), *found = total + 4;
        if (lane == 63) total[threadIdx.x >> 6] = incl;
        if (threadIdx.x == 0) found[0] = ~0u;
        __syncthreads();
        uint32_t from = incl - n;
#pragma unroll
        for (int w = 0; w < 3; ++w) from += w < int(threadIdx.x >> 6) ? total[w] : 0u;
        if (x >= from && x - from < n) {                     // one thread at most
            in = x - from;
            for (int b = b0; b < b1; ++b) {
                const uint32_t k = pairs(load_seq(a, b));
                if (in < k) {
                    found[0] = uint32_t(b);
                    found[1] = in;
                    break;
                }
                in -= k;
            }
        }
        __syncthreads();
        const int b = __builtin_amdgcn_readfirstlane(found[0]);
        in = __builtin_amdgcn_readfirstlane(found[1]);
        __syncthreads();
        if (b < 0) return false;
        *b_out = b;
        s = of_lane(load_seq(a, b), 0);
    } else {
        const unsigned long long past = __ballot(incl > x);
        if (!past) return false;
        const int l = __ffsll(past) - 1;
        in = x - (__builtin_amdgcn_readlane(incl, l) - __builtin_amdgcn_readlane(n, l));
        s = of_lane(p.mine, l);
        *b_out = l;
    }
    *c_out = int(in / uint32_t(s.tiles));
    *it = make_item(s, s.tiles - 1 - int(in % uint32_t(s.tiles)), *c_out, p.chunk, cap, a.window, a.group_shift);
    return !it->idle;
}

// Pool row of the 16 keys at `pos` of sequence b and head g; -1 where the item sees none of them or on a page
// outside the pool.  Uniform in the wave: read through the scalar cache.
__device__ inline int key_block(const PageAttendArgs &a, const Item &it, int b, int g, int pos, int lane) {
    if (!block_seen(it, pos)) return -1;
    typedef const __attribute__((address_space(4))) int32_t *ro;
    const int page = ((ro)(uintptr_t)a.t.table)[int64_t(b) * a.t.max_pages + (pos >> a.t.page_shift)];
    const int r = block_row(page, a.t.n_pages, a.t.Hkv, g, a.t.page_shift, pos);
    if (r < 0 && lane == 0) flag(a.t);
    return r;
}

// Partials that the last workgroup of a tile joins cross between the chip's L2 caches: written through
// and read past them.  A second kernel sees plain stores.
template <bool kThrough>
__device__ inline void put_pair(float *p, float x, float y) {
    if (!kThrough) {
        *reinterpret_cast<float2 *>(p) = make_float2(x, y);
        return;
    }
    __hip_atomic_store(reinterpret_cast<uint64_t *>(p), __float_as_uint(x) | uint64_t(__float_as_uint(y)) << 32,
                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <bool kThrough>
__device__ inline float2 get_pair(const float *p) {
    if (!kThrough) return *reinterpret_cast<const float2 *>(p);
    const uint64_t w = __hip_atomic_load(reinterpret_cast<const uint64_t *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float(uint32_t(w)), __uint_as_float(uint32_t(w >> 32)));
}

// Where a row's result goes: the output, or a partial of its chunk.  o: N consecutive values from d0
// on, weighted by exp2(s - m); l: the sum of the weights.
template <class T, int D, int N>
__device__ inline void put(const PageAttendArgs &a, const Item &it, int chunk, int tok, int h, int d0, const float (&o)[N],
                           float m, float l) {
    const int Hq = a.t.Hkv << a.group_shift;
    const size_t row = size_t(tok) * Hq + h;
    if (it.chunk0 == it.chunk1) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        float x[N];
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = l == 0.f ? 0.f : o[i] * inv;
        if constexpr (T::kBytes == 2) {
            uint16_t *p = static_cast<uint16_t *>(a.out) + row * D + d0;
            if constexpr (N == 1) *p = uint16_t(bf16_pack(x[0], 0.f));
#pragma unroll
            for (int i = 0; i < N / 2; ++i) reinterpret_cast<uint32_t *>(p)[i] = bf16_pack(x[2 * i], x[2 * i + 1]);
        } else {
            float *p = static_cast<float *>(a.out) + row * D + d0;
#pragma unroll
            for (int i = 0; i < N; ++i) p[i] = x[i];
        }
        if (a.lse && d0 == 0) a.lse[row] = l == 0.f ? -INFINITY : m * 0.69314718055994531f + logf(l);
    } else {
        const size_t at = size_t(chunk) * a.t.n_tokens * Hq + row;
        float *p = a.part_o + at * D + d0;
        if constexpr (N == 1) {
            __hip_atomic_store(p, o[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (d0 == 0) put_pair<true>(a.part_ml + 2 * at, m, l);
        } else if (a.join_launch) {
#pragma unroll
            for (int i = 0; i < N; i += 2) put_pair<false>(p + i, o[i], o[i + 1]);
            if (d0 == 0) put_pair<false>(a.part_ml + 2 * at, m, l);
        } else {
#pragma unroll
            for (int i = 0; i < N; i += 2) put_pair<true>(p + i, o[i], o[i + 1]);
            if (d0 == 0) put_pair<true>(a.part_ml + 2 * at, m, l);
        }
    }
}

// ------------------------------------------------------------------------------------------
// 16 query rows (or NB times 16) of one wave against keys straight from memory: no LDS, so many loads
// can be in flight.  Used where the rows are few and the bytes are the bound (bfloat16, narrow tiles),
// and for float, whose matrix instruction takes 32 cycles for 2048 operations: there the loads of
// four waves through the first-level cache are no bound.  Reached: one token of each of 32 sequences of up to
// 32768, bfloat16, 455 us (5.6 TB/s); of 4 of 131072 in 8 bits 190 us (5.7 TB/s), a copy of the card moving 5.1;
// 2048 float tokens over 8192 keys 2285 us (105 of the 154 TFLOP/s of a float matrix product).
//
// Registers of a 16-key block: keys: lane (key lane % 16, g = lane / 16) holds the pieces g of its
// row; values: lane (m = lane % 16, g) holds elements D/16 m .. of the rows 4 g .. 4 g + 3, that is,
// whole rows by 16 lanes, and result tile e of O^T has the elements D/16 m + e.  bfloat16 products run
// over 32 keys: two blocks, whose rows 4 g + i are what S^T leaves in lane group g.
// ------------------------------------------------------------------------------------------
template <class T, class P, int D>
struct Keys16 {
    static constexpr int kBlocks = T::kBytes == 2 ? 2 : 1, kKeys = 16 * kBlocks;
    static constexpr int KW = D * P::kBytes / 16, VW = D * P::kBytes / 64;    // words a lane
    uint32_t k[kBlocks][KW], v[kBlocks][4][VW], ks[kBlocks], vs[kBlocks];

    __device__ static size_t base(int row) { return row >= 0 ? row : 0; }     // any row: its keys are masked
    __device__ void load_keys(const PageAttendArgs &a, const int (&row)[kBlocks], int lane) {
        const int m = lane & 15, g = lane >> 4;
#pragma unroll
        for (int j = 0; j < kBlocks; ++j) {
            const size_t r0 = base(row[j]);
            const unsigned char *kp = static_cast<const unsigned char *>(a.k) + r0 * (D * P::kBytes);
#pragma unroll
            for (int i = 0; i < KW / 4; ++i) {
                const int off = P::kBytes == 4 ? 256 * (i >> 2) + 64 * g + 16 * (i & 3) : 64 * i + 16 * g;
                const uint4 w = *reinterpret_cast<const uint4 *>(kp + m * (D * P::kBytes) + off);
                k[j][4 * i] = w.x; k[j][4 * i + 1] = w.y; k[j][4 * i + 2] = w.z; k[j][4 * i + 3] = w.w;
            }
            if constexpr (P::kBytes == 1) ks[j] = a.k_scale[r0 + m];
        }
    }
    __device__ void load_values(const PageAttendArgs &a, const int (&row)[kBlocks], int lane) {
        const int m = lane & 15, g = lane >> 4;
#pragma unroll
        for (int j = 0; j < kBlocks; ++j) {
            const size_t r0 = base(row[j]);
            const unsigned char *vp = static_cast<const unsigned char *>(a.v) + r0 * (D * P::kBytes);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned char *p = vp + (4 * g + i) * (D * P::kBytes) + m * (VW * 4);
                if constexpr (VW % 4 == 0) {
#pragma unroll
                    for (int u = 0; u < VW / 4; ++u) {
                        const uint4 w = reinterpret_cast<const uint4 *>(p)[u];
                        v[j][i][4 * u] = w.x; v[j][i][4 * u + 1] = w.y; v[j][i][4 * u + 2] = w.z; v[j][i][4 * u + 3] = w.w;
                    }
                } else if constexpr (VW == 2) {
                    const uint2 w = *reinterpret_cast<const uint2 *>(p);
                    v[j][i][0] = w.x; v[j][i][1] = w.y;
                } else {
                    v[j][i][0] = *reinterpret_cast<const uint32_t *>(p);
                }
            }
            if constexpr (P::kBytes == 1) vs[j] = *reinterpret_cast<const uint32_t *>(a.v_scale + r0 + 4 * g);
        }
    }
};

template <class T, class P, int D, int NB>
struct Rows16 {
    using Tile = Keys16<T, P, D>;
    static constexpr int VE = D / 16, QW = T::kBytes == 2 ? D / 8 : D / 4;    // words of the query a lane
    static constexpr bool kBf = T::kBytes == 2;
    static constexpr int J = Tile::kBlocks;
    uint32_t q[NB][QW];
    f4v o[NB][VE];
    float m[NB], l[NB];
    int lo[NB], hi[NB];                 // keys that the column's query sees
    int lo_all, hi_all, lo_any, hi_any; // keys that every column sees, that some column sees

    // Columns: rows row0 + 16 nb + lane % 16 of the item.
    __device__ void init(const PageAttendArgs &a, const Item &it, int g, int row0, int lane) {
        const int n = lane & 15, gq = lane >> 4, gs = a.group_shift;
        const int64_t cap = int64_t(a.t.max_pages) << a.t.page_shift;
        using E = typename T::elem;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            int row = row0 + 16 * nb + n;
            row = row < it.rows ? row : it.rows - 1;                          // spare columns repeat the last row
            const int64_t p = it.p0 + (row >> gs);
            const int64_t b = p - (int64_t(a.window) - 1);
            lo[nb] = b < 0 ? 0 : int(b < cap ? b : cap);
            hi[nb] = int(p < 0 ? -1 : p < cap ? p : cap - 1);
            const E *src = static_cast<const E *>(a.q) + int64_t(it.tok0 + (row >> gs)) * a.q_stride +
                           ((g << gs) + (row & ((1 << gs) - 1))) * D;
#pragma unroll
            for (int i = 0; i < QW / 4; ++i) {
                // the dims of product i: as Keys16 lays out its pieces
                const int dim = !kBf ? 64 * (i >> 2) + 16 * gq + 4 * (i & 3)
                              : P::kBytes == 2 ? 32 * i + 8 * gq : 64 * (i >> 1) + 16 * gq + 8 * (i & 1);
                const uint4 w = *reinterpret_cast<const uint4 *>(src + dim);
                q[nb][4 * i] = w.x; q[nb][4 * i + 1] = w.y; q[nb][4 * i + 2] = w.z; q[nb][4 * i + 3] = w.w;
            }
            m[nb] = -INFINITY;
            l[nb] = 0.f;
#pragma unroll
            for (int e = 0; e < VE; ++e) o[nb][e] = f4v{0.f, 0.f, 0.f, 0.f};
        }
        const int last = row0 + 16 * NB - 1 < it.rows ? row0 + 16 * NB - 1 : it.rows - 1;
        const int64_t p_first = it.p0 + (row0 >> gs), p_last = it.p0 + (last >> gs);
        const int64_t b = p_last - (int64_t(a.window) - 1);
        lo_all = b < 0 ? 0 : int(b < cap ? b : cap);
        hi_all = int(p_first < 0 ? -1 : p_first < cap ? p_first : cap - 1);
        const int64_t f = p_first - (int64_t(a.window) - 1);
        lo_any = f < 0 ? 0 : int(f < cap ? f : cap);
        hi_any = int(p_last < 0 ? -1 : p_last < cap ? p_last : cap - 1);
    }

    __device__ static uint4 k_frag(const Tile &t, int j, int s) {             // bfloat16: product s
        if constexpr (P::kBytes == 2) {
            return make_uint4(t.k[j][4 * s], t.k[j][4 * s + 1], t.k[j][4 * s + 2], t.k[j][4 * s + 3]);
        } else {
            return codes8_bf16(t.k[j][2 * s], t.k[j][2 * s + 1], pow2_of(t.ks[j]));
        }
    }
    // Float scores in several sums, so that fewer roundings follow each other: one chain of D terms put a single
    // token's output 7.6e-7 off (root mean square over 100 inputs of 2048 keys), two chains 4.5e-7, four 3.4e-7,
    // at the same time; with two tiles of rows four cost 1 % more than two.
    static constexpr int kSums = NB == 1 ? 4 : 2;
    __device__ void scores(const Tile &t, f4v (&s)[Tile::kBlocks][NB]) const {
#pragma unroll
        for (int j = 0; j < Tile::kBlocks; ++j) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) s[j][nb] = f4v{0.f, 0.f, 0.f, 0.f};
            if constexpr (kBf) {
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    const uint4 kf = k_frag(t, j, i);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
                        s[j][nb] = mma16(kf, make_uint4(q[nb][4 * i], q[nb][4 * i + 1], q[nb][4 * i + 2], q[nb][4 * i + 3]),
                                         s[j][nb]);
                }
            } else {
                f4v w[kSums][NB];
#pragma unroll
                for (int p = 0; p < kSums; ++p)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) w[p][nb] = f4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    float kf[4];
                    if constexpr (P::kBytes == 4) {
#pragma unroll
                        for (int u = 0; u < 4; ++u) kf[u] = __uint_as_float(t.k[j][4 * i + u]);
                    } else {
                        codes4_up(t.k[j][i], pow2_of(t.ks[j]), kf);
                    }
#pragma unroll
                    for (int u = 0; u < 4; ++u)
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb)
                            w[u % kSums][nb] = mma16(kf[u], __uint_as_float(q[nb][4 * i + u]), w[u % kSums][nb]);
                }
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    s[j][nb] = w[0][nb] + w[1][nb];
                    if constexpr (kSums == 4) s[j][nb] += w[2][nb] + w[3][nb];
                }
            }
        }
    }

    // Mask, running maximum and weights of the keys from pos on; valid: a bit for each block that holds
    // keys.  True when some column does not see some key.  bad: the maximum is too large.
    __device__ bool weights(const PageAttendArgs &a, f4v (&s)[J][NB], int pos, uint32_t valid, bool *bad, int lane) {
        const int g = lane >> 4;
        const bool part = valid != (1u << J) - 1 || pos < lo_all || pos + Tile::kKeys - 1 > hi_all;
        if (part) {
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = pos + 16 * j + 4 * g + i;
                        s[j][nb][i] = (valid >> j & 1) && key >= lo[nb] && key <= hi[nb] ? s[j][nb][i] : -INFINITY;
                    }
        }
        float mx[NB];
        bool up = false;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            mx[nb] = s[0][nb][0];
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) mx[nb] = fmaxf(mx[nb], s[j][nb][i]);
            up |= mx[nb] * a.scale_log2 > m[nb] + kSlack;
        }
        if (__any(up)) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                float x = fmaxf(mx[nb], across16(mx[nb]));
                x = fmaxf(x, across32(x)) * a.scale_log2;
                const float mn = fmaxf(m[nb], x);
                const float f = exp2_fast(m[nb] - (mn == -INFINITY ? 0.f : mn));
                m[nb] = mn;
                *bad |= too_large(mn);
                l[nb] *= f;
#pragma unroll
                for (int e = 0; e < VE; ++e) o[nb][e] *= f;
            }
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const float mu = m[nb] == -INFINITY ? 0.f : m[nb];
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[j][nb][i] = exp2_fast(fmaf(s[j][nb][i], a.scale_log2, -mu));
                    l[nb] += s[j][nb][i];
                }
        }
        return part;
    }

    // o += values x weights, which for bfloat16 are rounded to it as the values are: the matrix instruction takes one
    // type.  Off by 2^-8 of a weight at most; one token of 32 sequences of up to 32768 is 1.77e-3 off 64 bits (root
    // mean square, relative), 1.65e-3 of it the output's own rounding.
    // Where `part`, rows that no column sees count as zeros, and `bad` says that one which some columns do not see
    // holds an infinity or NaN, or 8-bit values that may become one: zero times that is no number.
    __device__ void values(Tile &t, const f4v (&s)[J][NB], int pos, uint32_t valid, bool part, bool *bad, int lane) {
        const int g = lane >> 4;
        if (part) {
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = pos + 16 * j + 4 * g + i;
                    const uint32_t keep = (valid >> j & 1) && key >= lo_any && key <= hi_any ? 0xffffffffu : 0u;
                    uint32_t wrong = 0;
                    // the exponent byte as well: one of 255 makes no number of any code
                    if constexpr (P::kBytes == 1) {
                        t.vs[j] = keep ? t.vs[j] : (t.vs[j] & ~(255u << (8 * i))) | 127u << (8 * i);
                        wrong = uint32_t((t.vs[j] >> (8 * i) & 255u) >= kOverExponent);
                    }
#pragma unroll
                    for (int w = 0; w < Tile::VW; ++w) {
                        t.v[j][i][w] &= keep;
                        wrong |= P::kBytes == 1 ? nan4(t.v[j][i][w]) : P::kBytes == 2 ? odd2(t.v[j][i][w])
                                                                              : uint32_t(odd(__uint_as_float(t.v[j][i][w])));
                    }
                    *bad |= wrong != 0;
                }
        }
        if constexpr (kBf) {
            uint4 pf[NB];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
                pf[nb] = make_uint4(bf16_pack(s[0][nb][0], s[0][nb][1]), bf16_pack(s[0][nb][2], s[0][nb][3]),
                                    bf16_pack(s[J - 1][nb][0], s[J - 1][nb][1]), bf16_pack(s[J - 1][nb][2], s[J - 1][nb][3]));
#pragma unroll
            for (int w = 0; w < VE / 2; ++w) {
                uint32_t x[J][4];                             // elements 2 w and 2 w + 1 of the lane's rows
#pragma unroll
                for (int j = 0; j < J; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if constexpr (P::kBytes == 2) x[j][i] = t.v[j][i][w];
                        else x[j][i] = codes2_bf16(t.v[j][i][w / 2], pow2_of(t.vs[j] >> (8 * i) & 255u), w & 1);
                    }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint32_t sel = u ? 0x07060302u : 0x05040100u;
                    const uint4 vf = make_uint4(__builtin_amdgcn_perm(x[0][1], x[0][0], sel), __builtin_amdgcn_perm(x[0][3], x[0][2], sel),
                                                __builtin_amdgcn_perm(x[J - 1][1], x[J - 1][0], sel),
                                                __builtin_amdgcn_perm(x[J - 1][3], x[J - 1][2], sel));
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) o[nb][2 * w + u] = mma16(vf, pf[nb], o[nb][2 * w + u]);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float vf[VE];
                if constexpr (P::kBytes == 4) {
#pragma unroll
                    for (int e = 0; e < VE; ++e) vf[e] = __uint_as_float(t.v[0][i][e]);
                } else {
#pragma unroll
                    for (int w = 0; w < VE / 4; ++w) {
                        float x[4];
                        codes4_up(t.v[0][i][w], pow2_of(t.vs[0] >> (8 * i) & 255u), x);
#pragma unroll
                        for (int u = 0; u < 4; ++u) vf[4 * w + u] = x[u];
                    }
                }
#pragma unroll
                for (int e = 0; e < VE; ++e)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) o[nb][e] = mma16(vf[e], s[0][nb][i], o[nb][e]);
            }
        }
    }

    // Every step-th group of keys from pos on.  bad: the item has to be done row by row.
    // A group's keys and values are asked for as soon as the registers of an earlier one are free, kAhead groups
    // ahead; its row blocks one group before that.  Two groups where they fit: 32 ragged sequences in bfloat16 462 us
    // against 469 with one, 4 of 131072 in 8 bits 188.6 against 191.2, 13 of float and head_dim 64 577 against 599.
    static constexpr int kTileWords = J * (Tile::KW + 4 * Tile::VW), kHeld = NB * (D / 4 + QW);
    static constexpr int kAhead = 2 * kTileWords + kHeld <= 176 ? 2 : 1;      // of 256 registers
    __device__ void run(const PageAttendArgs &a, const Item &it, int b, int g, int pos, int step, bool *bad, int lane) {
        if (pos >= it.end) return;
        Tile t[kAhead];
        uint32_t valid[kAhead];
        int row[J];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            look(a, it, b, g, pos + u * step, row, lane);
            valid[u] = bits(row);
            if (pos + u * step < it.end) {
                t[u].load_keys(a, row, lane);
                t[u].load_values(a, row, lane);
            }
        }
        for (;;) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int next = pos + kAhead * step;
                const bool more = next < it.end;
                if (more) look(a, it, b, g, next, row, lane);
                f4v s[J][NB];
                scores(t[u], s);
                if (more) t[u].load_keys(a, row, lane);
                const bool part = weights(a, s, pos, valid[u], bad, lane);
                values(t[u], s, pos, valid[u], part, bad, lane);
                if (more) {
                    t[u].load_values(a, row, lane);
                    valid[u] = bits(row);
                }
                pos += step;
                if (pos >= it.end) return;
            }
        }
    }
    __device__ static uint32_t bits(const int (&row)[J]) {
        uint32_t v = 0;
#pragma unroll
        for (int j = 0; j < J; ++j) v |= row[j] >= 0 ? 1u << j : 0u;
        return v;
    }
    __device__ static void look(const PageAttendArgs &a, const Item &it, int b, int g, int pos, int (&row)[J], int lane) {
#pragma unroll
        for (int j = 0; j < J; ++j) row[j] = key_block(a, it, b, g, pos + 16 * j, lane);
    }

    // The column's sum over its four lanes.
    __device__ float sum(int nb) const {
        float x = l[nb] + across16(l[nb]);
        return x + across32(x);
    }
};

// An item whose masked keys hold infinities or NaN, or whose scores are too large, row by row: a wave a row, 64
// keys at a time, a score a lane, then the values with the lanes over d.  Only keys that the row sees are touched.
template <class T, class P, int D>
__device__ inline void plain_rows(const PageAttendArgs &a, const Item &it, int b, int g, int c, int lane, int wave) {
    auto element = [](const void *pool, const uint8_t *scale, int row, int i) {
        const size_t at = size_t(row) * D + i;
        if constexpr (P::kBytes == 4) return static_cast<const float *>(pool)[at];
        else if constexpr (P::kBytes == 2) return bf16_up(static_cast<const uint16_t *>(pool)[at]);
        else {
            float x[4];
            codes4_up(static_cast<const uint8_t *>(pool)[at], pow2_of(scale[row]), x);
            return x[0];
        }
    };
    const int64_t cap = int64_t(a.t.max_pages) << a.t.page_shift;
    for (int rw = wave; rw < it.rows; rw += 4) {
        const int tok = it.tok0 + (rw >> a.group_shift), h = (g << a.group_shift) + (rw & ((1 << a.group_shift) - 1));
        const int64_t p = it.p0 + (rw >> a.group_shift), w = p - (int64_t(a.window) - 1);
        const int64_t from = w > it.begin ? w : it.begin, to = p + 1 < it.end ? p + 1 : it.end;
        float m = -INFINITY, l = 0.f, o[D / 64] = {};
        for (int64_t j0 = from; j0 < to; j0 += 64) {
            const int j = int(j0) + lane;
            int row = -1;
            if (j < to && j < cap) row = pool_row(a.t, b, g, j);
            float s = -INFINITY;
            if (row >= 0) {
                float x = 0.f;
                for (int i = 0; i < D; ++i) {
                    const int64_t at = int64_t(tok) * a.q_stride + h * D + i;
                    const float q = T::kBytes == 4 ? static_cast<const float *>(a.q)[at] : bf16_up(static_cast<const uint16_t *>(a.q)[at]);
                    x = fmaf(q, element(a.k, a.k_scale, row, i), x);
                }
                s = x * a.scale_log2;
            }
            float mx = s;
            for (int k = 1; k < 64; k *= 2) mx = fmaxf(mx, __shfl_xor(mx, k));
            const float mn = fmaxf(m, mx), mu = mn == -INFINITY ? 0.f : mn;
            const float f = exp2_fast(m - mu), wt = row >= 0 ? exp2_fast(s - mu) : 0.f;
            float sum = wt;
            for (int k = 1; k < 64; k *= 2) sum += __shfl_xor(sum, k);
            m = mn;
            l = l * f + sum;
            for (int e = 0; e < D / 64; ++e) o[e] *= f;
            for (int k = 0; k < 64; ++k) {
                const int r = __builtin_amdgcn_readlane(row, k);
                const float x = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(wt), k));
                if (r >= 0)
                    for (int e = 0; e < D / 64; ++e) o[e] = fmaf(x, element(a.v, a.v_scale, r, lane * (D / 64) + e), o[e]);
            }
        }
        put<T, D>(a, it, c, tok, h, lane * (D / 64), o, m, l);
    }
}

// Joins the partials of an item's rows from first on.  D / 4 threads hold a row, so several rows, or several
// shares of one row's chunks, go side by side; shares meet in LDS in a fixed order.  Four chunks a turn keep the
// loads of a share in flight; eight were slower.
// lds: 256 float4 and 256 float2.
template <class T, int D, bool kThrough>
__device__ inline void join_rows(const PageAttendArgs &a, Item it, int g, int first, int rows, int lane, unsigned char *lds) {
    constexpr int GT = D / 4, NG = 256 / GT;                 // threads a group, groups
    const int t = threadIdx.x % GT, grp = threadIdx.x / GT, n = it.chunk1 - it.chunk0 + 1;
    int side = 1;                                            // rows side by side: a power of two
    while (side < rows && side < NG) side *= 2;
    const int shares = NG / side, share = grp % shares;
    float4 *so = reinterpret_cast<float4 *>(lds);
    float2 *sm = reinterpret_cast<float2 *>(lds + 256 * sizeof(float4));
    const int Hq = a.t.Hkv << a.group_shift;
    const size_t step = size_t(a.t.n_tokens) * Hq;
    for (int r0 = 0; r0 < rows; r0 += side) {
        const int r = r0 + grp / shares, rw = first + (r < rows ? r : rows - 1);
        const int tok = it.tok0 + (rw >> a.group_shift), h = (g << a.group_shift) + (rw & ((1 << a.group_shift) - 1));
        const size_t at = size_t(it.chunk0) * step + size_t(tok) * Hq + h;
        float m = -INFINITY, l = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        constexpr int U = 4;
        for (int c0 = share; c0 < n; c0 += U * shares) {     // chunks share, share + shares, ...
            float2 ml[U], lo[U], hi[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = c0 + u * shares < n ? c0 + u * shares : n - 1;
                ml[u] = get_pair<kThrough>(a.part_ml + 2 * (at + c * step));
                lo[u] = get_pair<kThrough>(a.part_o + (at + c * step) * D + 4 * t);
                hi[u] = get_pair<kThrough>(a.part_o + (at + c * step) * D + 4 * t + 2);
            }
            float mn = m;
#pragma unroll
            for (int u = 0; u < U; ++u) mn = fmaxf(mn, ml[u].x);
            const float mu = mn == -INFINITY ? 0.f : mn, f0 = exp2_fast(m - mu);
            m = mn;
            l *= f0;
            o.x *= f0; o.y *= f0; o.z *= f0; o.w *= f0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (c0 + u * shares < n) {
                    const float f = exp2_fast(ml[u].x - mu);
                    l += f * ml[u].y;
                    o.x += f * lo[u].x; o.y += f * lo[u].y; o.z += f * hi[u].x; o.w += f * hi[u].y;
                }
            }
        }
        if (shares > 1) {
            so[threadIdx.x] = o;
            if (t == 0) sm[grp] = make_float2(m, l);
            __syncthreads();
            if (share == 0) {
                float mx = m;
                for (int s = 1; s < shares; ++s) mx = fmaxf(mx, sm[grp + s].x);
                const float mu = mx == -INFINITY ? 0.f : mx, f0 = exp2_fast(m - mu);
                l *= f0;
                o.x *= f0; o.y *= f0; o.z *= f0; o.w *= f0;
                for (int s = 1; s < shares; ++s) {
                    const float f = exp2_fast(sm[grp + s].x - mu);
                    const float4 x = so[threadIdx.x + s * GT];
                    l += f * sm[grp + s].y;
                    o.x += f * x.x; o.y += f * x.y; o.z += f * x.z; o.w += f * x.w;
                }
                m = mx;
            }
            __syncthreads();
        }
        if (share == 0 && r < rows) {
            Item whole = it;
            whole.chunk1 = whole.chunk0;                     // the output itself
            const float x[4] = {o.x, o.y, o.z, o.w};
            put<T, D>(a, whole, 0, tok, h, 4 * t, x, m, l);
        }
    }
}

}  // namespace page
}  // namespace sekv
