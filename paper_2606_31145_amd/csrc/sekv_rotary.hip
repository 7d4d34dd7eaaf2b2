// Rotary positions over rows of heads: queries by themselves, or beside keys on their way into the paged store.
//
// A workgroup takes as many consecutive tokens as it holds rows side by side, and a chunk of their heads.  It forms the
// tokens' angles once in LDS, one (token, pair) a thread at a time, takes them into registers, and passes over the heads:
// a row is read once and written once, which is what bounds long calls.  Short ones are a chain of dependent reads.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "sekv_rotary.h"

namespace sekv {
namespace {

using namespace page;

constexpr int kThreads = 256;
constexpr int64_t kMaxBlocks = 1 << 21;   // a launch stays below 2^32 threads
struct NoPages {};

template <class T, class P, int D, bool kHalf>
__global__ void __launch_bounds__(kThreads) rotary_kernel(RotaryArgs a) {
    constexpr bool kPages = !std::is_same_v<P, NoPages>;
    constexpr int N = Piece<T>::kN, L = D / N, kRows = kThreads / L;
    __shared__ double2 pairs[kRows * (D / 2)];
    __shared__ double where[kRows];
    __shared__ int32_t first[kRows];                         // a token's pool row of head 0; -1: none, -2: nobody's token
    __shared__ int32_t start[kPages ? kMaxPageBatch + 1 : 1];
    const PageTables &t = a.t;
    const int lane = threadIdx.x % L, row = threadIdx.x / L, R2 = a.rot_dim / 2;
    const int units = a.Hq + (kPages ? t.Hkv : 0);
    const int64_t all = (int64_t(t.n_tokens) + kRows - 1) / kRows * a.chunks;
    if constexpr (kPages)
        for (int i = threadIdx.x; i <= t.B; i += kThreads) start[i] = t.tok_start[i];
    for (int64_t c = blockIdx.x; c < all; c += gridDim.x) {
        const int64_t tok0 = c / a.chunks * kRows;
        const int u0 = int(c % a.chunks) * a.per, u1 = u0 + a.per < units ? u0 + a.per : units;
        __syncthreads();
        if (threadIdx.x < kRows) {
            const int64_t tok = tok0 + threadIdx.x;
            double p = 0.0;
            int to = -2;
            if (tok < t.n_tokens) {
                if constexpr (kPages) {
                    const int b = sequence_of(t, start, int(tok));
                    if (b >= 0) {
                        const int64_t pos = position_of(t, start, b, int(tok));
                        p = double(a.positions ? a.positions[tok] : pos);
                        to = first_row(t, b, pos);
                        if (to < 0 && u0 == 0) flag(t);
                    }
                } else {
                    p = double(a.positions[tok]);
                    to = -1;
                }
            }
            where[threadIdx.x] = p;
            first[threadIdx.x] = to;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < kRows * R2; i += kThreads) {
            const int r = i / R2;
            const double2 p = cos_sin(where[r] * a.freq[i - r * R2]);
            pairs[i] = make_double2(a.scale * p.x, a.transpose ? -a.scale * p.y : a.scale * p.y);
        }
        __syncthreads();
        Turn<T, D, kHalf> turn;
        turn.init(pairs + row * R2, a.rot_dim, lane);
        const int64_t tok = tok0 + row;
        const int to = first[row];
        for (int u = u0; u < u1; ++u) {
            if (u < a.Hq) {
                u4v w = {0, 0, 0, 0};
                if (to != -2) w = reinterpret_cast<const u4v *>(static_cast<const unsigned char *>(a.q) + (tok * a.q_stride + int64_t(u) * D) * T::kBytes)[lane];
                const u4v r = turn.apply(w).raw();
                if (to != -2) reinterpret_cast<u4v *>(static_cast<unsigned char *>(a.q_out) + (tok * a.out_stride + int64_t(u) * D) * T::kBytes)[lane] = r;
            } else if constexpr (kPages) {
                const int g = u - a.Hq;
                u4v w[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
                if (to >= 0) {
#pragma unroll
                    for (int s = 0; s < 2; ++s)
                        w[s] = reinterpret_cast<const u4v *>(static_cast<const unsigned char *>(a.kv.src[s]) + (tok * a.kv.stride[s] + int64_t(g) * D) * T::kBytes)[lane];
                }
                const Computed<T> k = turn.apply(w[0]);
                if (to >= 0) {
                    const int at = to + (g << t.page_shift);
                    store_row<Computed<T>, P, D>(a.kv.pool[0], a.kv.scale[0], at, k, lane);
                    store_row<Piece<T>, P, D>(a.kv.pool[1], a.kv.scale[1], at, Piece<T>{w[1]}, lane);
                }
            }
        }
    }
    if constexpr (kPages) {
        if (blockIdx.x == 0) {                               // offsets that cannot be
            __syncthreads();
            bool wrong = start[0] < 0 || start[t.B] > t.n_tokens;
            for (int i = threadIdx.x; i < t.B; i += kThreads) wrong |= start[i] > start[i + 1];
            if (wrong) flag(t);
        }
    }
}

// Workgroups aimed at: a call of few tokens is spread over its heads.
constexpr int64_t kBlocks = 2048;

template <class T, class P, int D, bool kHalf>
hipError_t launch(RotaryArgs a, hipStream_t s) {
    constexpr int kRows = kThreads / (D / Piece<T>::kN);
    const int units = a.Hq + (std::is_same_v<P, NoPages> ? 0 : a.t.Hkv);
    const int64_t blocks = (int64_t(a.t.n_tokens) + kRows - 1) / kRows;
    const int64_t want = (kBlocks + blocks - 1) / blocks;
    a.chunks = int(want < units ? want : units);
    a.per = (units + a.chunks - 1) / a.chunks;
    a.chunks = (units + a.per - 1) / a.per;
    const int64_t all = blocks * a.chunks;
    hipLaunchKernelGGL((rotary_kernel<T, P, D, kHalf>), dim3(unsigned(all < kMaxBlocks ? all : kMaxBlocks)), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

template <class T, class P>
hipError_t with_shape(const RotaryArgs &a, int layout, int d, hipStream_t s) {
    const bool half = layout == SEKV_ROTARY_HALF;
    if (d == 128) return half ? launch<T, P, 128, true>(a, s) : launch<T, P, 128, false>(a, s);
    return half ? launch<T, P, 64, true>(a, s) : launch<T, P, 64, false>(a, s);
}
template <class T>
hipError_t with_storage(const RotaryArgs &a, int layout, int page_dtype, int d, hipStream_t s) {
    if (page_dtype < 0) return with_shape<T, NoPages>(a, layout, d, s);
    if (page_dtype == SEKV_E2M1) return with_shape<T, E2M1>(a, layout, d, s);
    if (page_dtype == SEKV_E4M3) return with_shape<T, E4M3>(a, layout, d, s);
    return with_shape<T, T>(a, layout, d, s);
}

}  // namespace

hipError_t launch_rotary(RotaryArgs a, int layout, int dtype, int page_dtype, int head_dim, hipStream_t s) {
    return dtype == SEKV_BF16 ? with_storage<BF16>(a, layout, page_dtype, head_dim, s)
                              : with_storage<F32>(a, layout, page_dtype, head_dim, s);
}

}  // namespace sekv
