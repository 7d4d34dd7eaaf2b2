// Paged token store: storing new tokens and reading them back.
//
// Both move bytes and compute next to nothing (a maximum over a row, one exact scaling, one
// rounding), so what bounds them is HBM for long chunks and one chain of dependent loads
// (tables, page, row) for short ones: one token of 32 sequences takes 4 us.  A row belongs to a group of
// lanes of 16 bytes each on the wide side: 8 or 16 lanes for bfloat16, 16 or 32 for float, keys and
// values beside each other in one launch.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "sekv_page_store.h"

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
hipError_t launch_page_attend_BF16_E2M1_128(const PageAttendArgs &a, hipStream_t s);
hipError_t launch_page_attend_BF16_E2M1_64(const PageAttendArgs &a, hipStream_t s);
hipError_t launch_page_attend_F32_E2M1_128(const PageAttendArgs &a, hipStream_t s);
hipError_t launch_page_attend_F32_E2M1_64(const PageAttendArgs &a, hipStream_t s);

namespace {

using namespace page;

constexpr int kThreads = 256;
constexpr int64_t kMaxBlocks = 1 << 21;   // a launch stays below 2^32 threads

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
        const int b = tok < t.n_tokens ? sequence_of(t, start, int(tok)) : -1;
        const int to = b < 0 ? -1 : first_row(t, b, position_of(t, start, b, int(tok)));
        if (b >= 0 && to < 0 && lane == 0) flag(t);
        if (to >= 0) {
#pragma unroll
            for (int s = 0; s < 2; ++s) store_row<Piece<T>, P, D>(a.pool[s], a.scale[s], to + (g << t.page_shift), Piece<T>{w[s]}, lane);
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

template <> struct Stored<BF16, E2M1> {
    using W = uint32_t;
    static __device__ u4v up(const W &w, float scale) { return __builtin_bit_cast(u4v, word_bf16(w, scale)); }
};
template <> struct Stored<F32, E2M1> {
    using W = uint16_t;
    static __device__ u4v up(const W &w, float scale) {
        float x[4];
        pair_f32<0>(w, scale, x[0], x[1]);
        pair_f32<1>(w, scale, x[2], x[3]);
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
                                                                  size_t(from) * P::row(D))[i * 64 + lane];
                E[s][i] = P::scales(D) ? a.scale[s][size_t(from) * P::scales(D) + (i * 64 + lane) * P::scales(D) / PC] : 127u;
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
template <class T, class F>
hipError_t dispatch_storage(int page_dtype, F f) {
    if (page_dtype == SEKV_E4M3) return f(T{}, E4M3{});
    if (page_dtype == SEKV_E2M1) return f(T{}, E2M1{});
    return f(T{}, T{});
}
template <class F>
hipError_t dispatch(int dtype, int page_dtype, int d, F f) {
    auto with_d = [&](auto t, auto p) {
        return d == 128 ? f(t, p, std::integral_constant<int, 128>{}) : f(t, p, std::integral_constant<int, 64>{});
    };
    return dtype == SEKV_BF16 ? dispatch_storage<BF16>(page_dtype, with_d) : dispatch_storage<F32>(page_dtype, with_d);
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
    if (dtype == SEKV_BF16) {
        if (page_dtype == SEKV_E2M1) return head_dim == 128 ? launch_page_attend_BF16_E2M1_128(a, s) : launch_page_attend_BF16_E2M1_64(a, s);
        if (page_dtype == SEKV_E4M3) return head_dim == 128 ? launch_page_attend_BF16_E4M3_128(a, s) : launch_page_attend_BF16_E4M3_64(a, s);
        return head_dim == 128 ? launch_page_attend_BF16_BF16_128(a, s) : launch_page_attend_BF16_BF16_64(a, s);
    }
    if (page_dtype == SEKV_E2M1) return head_dim == 128 ? launch_page_attend_F32_E2M1_128(a, s) : launch_page_attend_F32_E2M1_64(a, s);
    if (page_dtype == SEKV_E4M3) return head_dim == 128 ? launch_page_attend_F32_E4M3_128(a, s) : launch_page_attend_F32_E4M3_64(a, s);
    return head_dim == 128 ? launch_page_attend_F32_F32_128(a, s) : launch_page_attend_F32_F32_64(a, s);
}

}  // namespace sekv
