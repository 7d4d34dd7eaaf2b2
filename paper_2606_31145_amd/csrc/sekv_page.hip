// Paged token store: storing new tokens and reading them back.
//
// Both move bytes and compute next to nothing (a maximum over a row, one exact scaling, one
// rounding), so what bounds them is HBM for long chunks and one chain of dependent loads
// (tables, page, row) for short ones.  A row belongs to a group of lanes of 16 bytes each on the
// wide side: 8 or 16 lanes for bfloat16, 16 or 32 for float, keys and values beside each other
// in one launch.
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
constexpr int64_t kMaxBlocks = 1 << 20;   // per side: a launch stays below 2^32 threads

// 16 bytes of a row as floats, and back.
template <class T> struct Piece;
template <> struct Piece<F32> {
    static constexpr int kN = 4;
    static __device__ void up(const uint4 &w, float (&x)[4]) {
        x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
    }
};
template <> struct Piece<BF16> {
    static constexpr int kN = 8;
    static __device__ void up(const uint4 &w, float (&x)[8]) {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bf16_up(u[i] & 0xffffu);
            x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
};

template <class T, class P, int D>
__device__ inline void append_row(const PageAppendArgs &a, const int32_t *start, int side, int lane, int tok, int g) {
    constexpr int N = Piece<T>::kN, L = D / N;
    const PageTables &t = a.t;
    if (tok >= start[t.B] || tok < start[0]) return;
    int lo = 0, hi = t.B;                       // the last b with start[b] <= tok
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= tok) lo = mid; else hi = mid;
    }
    const int64_t pos = int64_t(t.seq_len[lo]) - start[lo + 1] + tok;
    int to = -1;
    if (tok < start[lo + 1] && pos >= 0 && (pos >> t.page_shift) < t.max_pages) to = pool_row(t, lo, g, int(pos));
    if (to < 0) {
        if (lane == 0) flag(t);
        return;
    }
    using E = typename T::elem;
    const uint4 w = reinterpret_cast<const uint4 *>(static_cast<const E *>(a.src[side]) + int64_t(tok) * a.stride[side] +
                                                    g * D)[lane];
    if constexpr (P::kBytes == T::kBytes) {
        reinterpret_cast<uint4 *>(static_cast<E *>(a.pool[side]) + size_t(to) * D)[lane] = w;
    } else {
        float x[N], m = 0.f;
        Piece<T>::up(w, x);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float y = fabsf(x[i]);
            m = y <= 3.402823466e38f ? fmaxf(m, y) : m;
        }
#pragma unroll
        for (int s = 1; s < L; s *= 2) m = fmaxf(m, __shfl_xor(m, s));
        const uint32_t Ex = row_exponent(m);
        const float inv = pow2_of(254u - Ex);
        uint32_t c[N / 4];
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const float y[4] = {x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
            c[i] = codes4(y, inv);
        }
        uint32_t *dst = reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(a.pool[side]) + size_t(to) * D) + lane * (N / 4);
#pragma unroll
        for (int i = 0; i < N / 4; ++i) dst[i] = c[i];
        if (lane == 0) a.scale[side][to] = uint8_t(Ex);
    }
}

// One row (token, head) of keys (blockIdx.y 0) or values (1) for each group of lanes.
template <class T, class P, int D>
__global__ void __launch_bounds__(kThreads) append_kernel(PageAppendArgs a) {
    constexpr int L = D / Piece<T>::kN;
    __shared__ int32_t start[kMaxPageBatch + 1];
    const PageTables &t = a.t;
    for (int i = threadIdx.x; i <= t.B; i += kThreads) start[i] = t.tok_start[i];
    __syncthreads();
    const int64_t rows = int64_t(t.n_tokens) * t.Hkv;
    for (int64_t row = int64_t(blockIdx.x) * (kThreads / L) + threadIdx.x / L; row < rows;
         row += int64_t(gridDim.x) * (kThreads / L))
        append_row<T, P, D>(a, start, blockIdx.y, threadIdx.x % L, int(row / t.Hkv), int(row % t.Hkv));
}

template <class T, class P, int D>
__device__ inline void read_row(const PageReadArgs &a, int side, int lane, int from, size_t to) {
    constexpr int N = Piece<T>::kN;
    using E = typename T::elem;
    uint4 w;
    if constexpr (P::kBytes == T::kBytes) {
        w = reinterpret_cast<const uint4 *>(static_cast<const E *>(a.pool[side]) + size_t(from) * D)[lane];
    } else {
        const uint32_t *c = reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(a.pool[side]) + size_t(from) * D) + lane * (N / 4);
        const float s = pow2_of(a.scale[side][from]);
        float x[N / 4][4];
#pragma unroll
        for (int i = 0; i < N / 4; ++i) codes4_up(c[i], s, x[i]);
        if constexpr (N == 8)
            w = make_uint4(bf16_pack(x[0][0], x[0][1]), bf16_pack(x[0][2], x[0][3]), bf16_pack(x[1][0], x[1][1]),
                           bf16_pack(x[1][2], x[1][3]));
        else
            w = make_uint4(__float_as_uint(x[0][0]), __float_as_uint(x[0][1]), __float_as_uint(x[0][2]), __float_as_uint(x[0][3]));
    }
    reinterpret_cast<uint4 *>(static_cast<E *>(a.dst[side]) + to)[lane] = w;
}

// One row (sequence, head, token) for each group of lanes.
template <class T, class P, int D>
__global__ void __launch_bounds__(kThreads) read_kernel(PageReadArgs a) {
    constexpr int L = D / Piece<T>::kN;
    const PageTables &t = a.t;
    const int side = blockIdx.y, lane = threadIdx.x % L;
    const int64_t chunks = (int64_t(a.max_tokens) + kThreads / L - 1) / (kThreads / L), all = chunks * t.B * t.Hkv;
    for (int64_t c = blockIdx.x; c < all; c += gridDim.x) {
        const int64_t bg = c / chunks;
        const int b = int(bg / t.Hkv), g = int(bg % t.Hkv);
        const int64_t pos = (c % chunks) * (kThreads / L) + threadIdx.x / L;
        if (pos >= a.max_tokens || pos >= t.seq_len[b]) continue;
        const int from = (pos >> t.page_shift) < t.max_pages ? pool_row(t, b, g, int(pos)) : -1;
        if (from < 0) {
            if (lane == 0) flag(t);
            continue;
        }
        read_row<T, P, D>(a, side, lane, from, (size_t(bg) * a.max_tokens + pos) * D);
    }
}

__global__ void __launch_bounds__(kThreads) zero_words_kernel(uint32_t *p, size_t n) {
    for (size_t i = size_t(blockIdx.x) * kThreads + threadIdx.x; i < n; i += size_t(gridDim.x) * kThreads) p[i] = 0;
}

template <class T, class P, int D>
hipError_t append(const PageAppendArgs &a, hipStream_t s) {
    constexpr int kRows = kThreads / (D / Piece<T>::kN);
    const int64_t rows = int64_t(a.t.n_tokens) * a.t.Hkv;
    const int64_t all = (rows + kRows - 1) / kRows;
    hipLaunchKernelGGL((append_kernel<T, P, D>), dim3(unsigned(all < kMaxBlocks ? all : kMaxBlocks), 2), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}
template <class T, class P, int D>
hipError_t read(const PageReadArgs &a, hipStream_t s) {
    constexpr int kRows = kThreads / (D / Piece<T>::kN);
    const int64_t all = ((int64_t(a.max_tokens) + kRows - 1) / kRows) * a.t.B * a.t.Hkv;
    hipLaunchKernelGGL((read_kernel<T, P, D>), dim3(unsigned(all < kMaxBlocks ? all : kMaxBlocks), 2), dim3(kThreads), 0, s, a);
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
