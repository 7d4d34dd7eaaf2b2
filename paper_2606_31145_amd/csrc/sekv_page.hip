// Paged token store: storing new tokens and reading them back.
//
// Both move bytes and compute next to nothing (a maximum over a row, one exact scaling, one
// rounding), so what bounds them is HBM for long chunks and one chain of dependent loads
// (tables, page, row) for short ones: one token of 32 sequences takes 4 us.  A row belongs to a group of
// lanes of 16 bytes each on the wide side: 8 or 16 lanes for bfloat16, 16 or 32 for float, keys and
// values beside each other in one launch.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "sekv_page_row.h"

namespace sekv {

// defined in sekv_page_attend_inst.hip, one object per (token type, storage type, head_dim)
hipError_t launch_page_attend_BF16_BF16_128(const PageAttendArgs &a, hipStream_t s);
hipError_t launch_page_attend_BF16_BF16_64(const PageAttendArgs &a, hipStream_t s);
hipError_t launch_page_attend_BF16_E4M3_128(const PageAttendArgs &a, hipStream_t s);
hipError_t launch_page_attend_BF16_E4M3_64(const PageAttendArgs &a, hipStream_t s);
hipError_t launch_page_attend_F32_F32_128(const PageAttendArgs &a, hipStream_t s);
hipError_t launch_page_attend_F32_F32_64(const PageAttendArgs &a, hipStream_t s);
hipError_t launch_page_attend_F32_E4M3_128(const PageAttendArgs &a, hipStream_t s);
hipError_t launch_page_attend_F32_E4M3_64(const PageAttendArgs &a, hipStream_t s);

namespace {

using namespace page;

constexpr int kThreads = 256;
constexpr int64_t kMaxBlocks = 1 << 21;   // a launch stays below 2^32 threads
typedef uint32_t u4v __attribute__((ext_vector_type(4)));

// The largest of L lanes' words, in each of them (L = 8, 16, 32; a group of lanes starts at a multiple of L).
template <int L>
__device__ inline uint32_t lanes_max(uint32_t x) {
    auto with = [&](uint32_t y) { x = x > y ? x : y; };
    with(__builtin_amdgcn_mov_dpp(x, 0xB1, 0xf, 0xf, true));       // quad_perm: lane ^ 1
    with(__builtin_amdgcn_mov_dpp(x, 0x4E, 0xf, 0xf, true));       // quad_perm: lane ^ 2
    with(__builtin_amdgcn_mov_dpp(x, 0x141, 0xf, 0xf, true));      // 7 - lane of 8
    if constexpr (L >= 16) with(__builtin_amdgcn_mov_dpp(x, 0x140, 0xf, 0xf, true));   // 15 - lane of 16
    if constexpr (L >= 32) with(__shfl_xor(x, 16));
    return x;
}

// 16 bytes of a row: as floats; the bits of the largest magnitude as a float's (an infinity's or NaN's if there
// is one); four of its values as codes, scaled by the power of two.
template <class T> struct Piece;
template <> struct Piece<F32> {
    static constexpr int kN = 4;
    static __device__ void up(const u4v &w, float (&x)[4]) {
        x[0] = __uint_as_float(w[0]); x[1] = __uint_as_float(w[1]); x[2] = __uint_as_float(w[2]); x[3] = __uint_as_float(w[3]);
    }
    static __device__ uint32_t top(const u4v &w) {
        const uint32_t a = w[0] & 0x7fffffffu, b = w[1] & 0x7fffffffu, c = w[2] & 0x7fffffffu, d = w[3] & 0x7fffffffu;
        const uint32_t ab = a > b ? a : b, cd = c > d ? c : d;
        return ab > cd ? ab : cd;
    }
    static __device__ uint32_t codes(const u4v &w, int, float scale) {
        typedef short s2v __attribute__((ext_vector_type(2)));
        s2v r = {0, 0};
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, __uint_as_float(w[0]), __uint_as_float(w[1]), scale, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, __uint_as_float(w[2]), __uint_as_float(w[3]), scale, true);
        return __builtin_bit_cast(uint32_t, r);
    }
};
template <> struct Piece<BF16> {
    static constexpr int kN = 8;
    static __device__ void up(const u4v &w, float (&x)[8]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bf16_up(w[i] & 0xffffu);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ uint32_t top(const u4v &w) {
        typedef uint16_t h2v __attribute__((ext_vector_type(2)));
        auto h = [&](int i) { return __builtin_bit_cast(h2v, w[i] & 0x7fff7fffu); };
        const h2v m = __builtin_elementwise_max(__builtin_elementwise_max(h(0), h(1)), __builtin_elementwise_max(h(2), h(3)));
        return uint32_t(m[0] > m[1] ? m[0] : m[1]) << 16;
    }
    static __device__ uint32_t codes(const u4v &w, int i, float scale) {
        typedef short s2v __attribute__((ext_vector_type(2)));
        typedef __bf16 b2v __attribute__((ext_vector_type(2)));
        s2v r = {0, 0};
        const uint32_t lo = w[2 * i], hi = w[2 * i + 1];     // a bit cast of w[k] itself takes element 0
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(b2v, lo), scale, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(b2v, hi), scale, true);
        return __builtin_bit_cast(uint32_t, r);
    }
};

// The place of new token `tok`: its sequence by a search in `start` (LDS), its row in the pool, or -1 (flagged).
__device__ inline int place(const PageTables &t, const int32_t *start, int tok, int g, bool first_lane) {
    if (tok >= start[t.B] || tok < start[0]) return -1;      // nobody's
    int lo = 0, hi = t.B;                                    // the last b with start[b] <= tok
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= tok) lo = mid; else hi = mid;
    }
    const int64_t pos = int64_t(t.seq_len[lo]) - start[lo + 1] + tok;
    int to = -1;
    if (tok < start[lo + 1] && pos >= 0 && (pos >> t.page_shift) < t.max_pages) to = pool_row(t, lo, g, int(pos));
    if (to < 0 && first_lane) flag(t);
    return to;
}

template <class T, class P, int D>
__device__ inline void store_row(const PageAppendArgs &a, int side, int to, const u4v &w, int lane) {
    constexpr int N = Piece<T>::kN, L = D / N;
    if constexpr (P::kBytes == T::kBytes) {
        __builtin_nontemporal_store(w, reinterpret_cast<u4v *>(static_cast<unsigned char *>(a.pool[side]) + size_t(to) * (D * T::kBytes)) + lane);
    } else {
        uint32_t c[N / 4];
        float m = __uint_as_float(lanes_max<L>(Piece<T>::top(w)));
        uint32_t Ex = row_exponent(m);
        if (m <= 3.402823466e38f && Ex > 8) {                // the row's lanes agree
            const float scale = pow2_of(Ex);
#pragma unroll
            for (int i = 0; i < N / 4; ++i) c[i] = Piece<T>::codes(w, i, scale);
        } else {
            // infinities or NaN, which do not count for the scale, or values so small that they may be
            // subnormal: element by element
            float x[N];
            Piece<T>::up(w, x);
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
        unsigned char *dst = static_cast<unsigned char *>(a.pool[side]) + size_t(to) * D + lane * N;
        typedef uint32_t u2v __attribute__((ext_vector_type(2)));
        if constexpr (N == 8) __builtin_nontemporal_store((u2v{c[0], c[1]}), reinterpret_cast<u2v *>(dst));
        else __builtin_nontemporal_store(c[0], reinterpret_cast<uint32_t *>(dst));
        if (lane == 0) a.scale[side][to] = uint8_t(Ex);
    }
}

// A block of consecutive new tokens of one head, heads side by side as they lie in a token: consecutive
// tokens are consecutive rows of a page, so that what a workgroup writes, exponent bytes included, lies
// together.  A row belongs to L lanes of 16 bytes, keys and values side by side.  The rows are asked for
// before their places are looked up, and stored past the caches: they are read again only with everything
// stored before them.  Four 8192-token chunks of 8 heads in 8 bits (202 MB), two sets of inputs in turn, which
// the last-level cache partly holds: 51.4 us with plain stores and four tokens a thread, 42.0 with stores past the
// caches, 38.1 with one token a thread as well (two: 39.5).  With inputs from memory it is 42.0 (4.8 TB/s).
template <class T, class P, int D>
__global__ void __launch_bounds__(kThreads) append_kernel(PageAppendArgs a) {
    constexpr int L = D / Piece<T>::kN, kRows = kThreads / L;
    __shared__ int32_t start[kMaxPageBatch + 1];
    const PageTables &t = a.t;
    const int lane = threadIdx.x % L;
    const int64_t all = (int64_t(t.n_tokens) + kRows - 1) / kRows * t.Hkv;
    bool first = true;
    for (int64_t c = blockIdx.x; c < all; c += gridDim.x) {
        const int g = int(c % t.Hkv);
        const int64_t tok = c / t.Hkv * kRows + threadIdx.x / L;
        u4v w[2];
        if (tok < t.n_tokens) {                              // a row of the call's buffers, stored or not
#pragma unroll
            for (int s = 0; s < 2; ++s)
                w[s] = reinterpret_cast<const u4v *>(static_cast<const unsigned char *>(a.src[s]) +
                                                     (tok * a.stride[s] + g * D) * T::kBytes)[lane];
        }
        if (first) {
            for (int i = threadIdx.x; i <= t.B; i += kThreads) start[i] = t.tok_start[i];
            __syncthreads();
            first = false;
        }
        const int to = tok < t.n_tokens ? place(t, start, int(tok), g, lane == 0) : -1;
        if (to >= 0) {
#pragma unroll
            for (int s = 0; s < 2; ++s) store_row<T, P, D>(a, s, to, w[s], lane);
        }
    }
    if (blockIdx.x == 0) {                                   // offsets that cannot be
        bool wrong = start[0] < 0 || start[t.B] > t.n_tokens;
        for (int i = threadIdx.x; i < t.B; i += kThreads) wrong |= start[i] > start[i + 1];
        if (wrong) flag(t);
    }
}

// What 16 bytes of the tokens' type are read from, and those bytes.
template <class T, class P> struct Stored { using W = u4v; static __device__ u4v up(const W &w, float) { return w; } };
template <> struct Stored<BF16, E4M3> {
    using W = uint2;
    static __device__ u4v up(const W &w, float scale) {
        float x[4], y[4];
        codes4_up(w.x, scale, x);
        codes4_up(w.y, scale, y);
        return u4v{bf16_pack(x[0], x[1]), bf16_pack(x[2], x[3]), bf16_pack(y[0], y[1]), bf16_pack(y[2], y[3])};
    }
};
template <> struct Stored<F32, E4M3> {
    using W = uint32_t;
    static __device__ u4v up(const W &w, float scale) {
        float x[4];
        codes4_up(w, scale, x);
        return u4v{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    }
};

// 64 tokens of one sequence and head for a workgroup, 16 of them (one block, in one page) for a wave, whose
// rows are consecutive on both sides.  A lane takes what makes 16 bytes of the dense side, which is the larger:
// four sequences of 131072 in 8 bits to bfloat16 (3.2 GB) 612 us (5.3 TB/s, a copy 5.1) against 676 with 16 bytes
// of the pages a lane.
template <class T, class P, int D>
__global__ void __launch_bounds__(kThreads) read_kernel(PageReadArgs a) {
    using S = Stored<T, P>;
    constexpr int PC = D * T::kBytes / 16, N = PC / 4;       // 16-byte pieces of a row, of a block a lane
    const PageTables &t = a.t;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t chunks = (int64_t(a.max_tokens) + 63) / 64, all = chunks * t.B * t.Hkv;
    for (int64_t c = blockIdx.x; c < all; c += gridDim.x) {
        const int64_t bg = c / chunks;
        const int b = int(bg / t.Hkv), g = int(bg % t.Hkv), pos = int(c % chunks) * 64 + wave * 16;
        const int have = t.seq_len[b] < a.max_tokens ? t.seq_len[b] : a.max_tokens;
        if (have < 0 && pos == 0 && lane == 0) flag(t);      // a length that cannot be
        if (pos >= have) continue;
        const int from = (pos >> t.page_shift) < t.max_pages ? pool_row(t, b, g, pos) : -1;
        if (from < 0) {
            if (lane == 0) flag(t);
            continue;
        }
        typename S::W w[2][N];
        uint32_t E[2][N];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                w[s][i] = reinterpret_cast<const typename S::W *>(static_cast<const unsigned char *>(a.pool[s]) +
                                                                  size_t(from) * (D * P::kBytes))[i * 64 + lane];
                E[s][i] = P::kBytes == 1 ? a.scale[s][from + (i * 64 + lane) / PC] : 127u;
            }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (pos + (i * 64 + lane) / PC < have)
                    reinterpret_cast<u4v *>(static_cast<unsigned char *>(a.dst[s]) +
                                            (size_t(bg) * a.max_tokens + pos) * (D * T::kBytes))[i * 64 + lane] =
                        S::up(w[s][i], pow2_of(E[s][i]));
    }
}

__global__ void __launch_bounds__(kThreads) zero_words_kernel(uint32_t *p, size_t n) {
    for (size_t i = size_t(blockIdx.x) * kThreads + threadIdx.x; i < n; i += size_t(gridDim.x) * kThreads) p[i] = 0;
}

template <class T, class P, int D>
hipError_t append(const PageAppendArgs &a, hipStream_t s) {
    constexpr int kRows = kThreads / (D / Piece<T>::kN);
    const int64_t all = (int64_t(a.t.n_tokens) + kRows - 1) / kRows * a.t.Hkv;
    hipLaunchKernelGGL((append_kernel<T, P, D>), dim3(unsigned(all < kMaxBlocks ? all : kMaxBlocks)), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}
template <class T, class P, int D>
hipError_t read(const PageReadArgs &a, hipStream_t s) {
    const int64_t all = ((int64_t(a.max_tokens) + 63) / 64) * a.t.B * a.t.Hkv;
    hipLaunchKernelGGL((read_kernel<T, P, D>), dim3(unsigned(all < kMaxBlocks ? all : kMaxBlocks)), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

// f(storage types, head_dim) for the combinations that check_page_dims lets through
template <class F>
hipError_t dispatch(int dtype, int page_dtype, int d, F f) {
    const bool q = page_dtype == SEKV_E4M3;
    if (dtype == SEKV_BF16) {
        if (d == 128) return q ? f(BF16{}, E4M3{}, std::integral_constant<int, 128>{}) : f(BF16{}, BF16{}, std::integral_constant<int, 128>{});
        return q ? f(BF16{}, E4M3{}, std::integral_constant<int, 64>{}) : f(BF16{}, BF16{}, std::integral_constant<int, 64>{});
    }
    if (d == 128) return q ? f(F32{}, E4M3{}, std::integral_constant<int, 128>{}) : f(F32{}, F32{}, std::integral_constant<int, 128>{});
    return q ? f(F32{}, E4M3{}, std::integral_constant<int, 64>{}) : f(F32{}, F32{}, std::integral_constant<int, 64>{});
}

}  // namespace

hipError_t launch_zero_words(void *p, size_t words, hipStream_t stream) {
    const size_t blocks = (words + kThreads - 1) / kThreads;
    hipLaunchKernelGGL(zero_words_kernel, dim3(unsigned(blocks < 1024 ? blocks : 1024)), dim3(kThreads), 0, stream,
                       static_cast<uint32_t *>(p), words);
    return hipGetLastError();
}

hipError_t launch_page_append(const PageAppendArgs &a, int dtype, int page_dtype, int head_dim, hipStream_t stream) {
    return dispatch(dtype, page_dtype, head_dim, [&](auto t, auto p, auto d) { return append<decltype(t), decltype(p), decltype(d)::value>(a, stream); });
}

hipError_t launch_page_read(const PageReadArgs &a, int dtype, int page_dtype, int head_dim, hipStream_t stream) {
    return dispatch(dtype, page_dtype, head_dim, [&](auto t, auto p, auto d) { return read<decltype(t), decltype(p), decltype(d)::value>(a, stream); });
}

hipError_t launch_page_attend(const PageAttendArgs &a, int dtype, int page_dtype, int head_dim, hipStream_t s) {
    const bool q = page_dtype == SEKV_E4M3;
    if (dtype == SEKV_BF16) {
        if (head_dim == 128) return q ? launch_page_attend_BF16_E4M3_128(a, s) : launch_page_attend_BF16_BF16_128(a, s);
        return q ? launch_page_attend_BF16_E4M3_64(a, s) : launch_page_attend_BF16_BF16_64(a, s);
    }
    if (head_dim == 128) return q ? launch_page_attend_F32_E4M3_128(a, s) : launch_page_attend_F32_F32_128(a, s);
    return q ? launch_page_attend_F32_E4M3_64(a, s) : launch_page_attend_F32_F32_64(a, s);
}

}  // namespace sekv
