// Attention of new tokens over the paged store.
//
// softmax in one pass: with m the largest score so far, l = sum exp(s - m) and o = sum exp(s - m) v;
// a larger m scales l and o by exp(old - new).  First form: one wave per (token, query head), 64
// keys at a time, a score per lane, then the values row by row with the lanes over d.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "sekv_page_row.h"

namespace sekv {
namespace {

using namespace page;

template <class P>
__device__ inline float value_at(const void *pool, const uint8_t *scale, size_t row, int D, int i) {
    if constexpr (P::kBytes == 4) return static_cast<const float *>(pool)[row * D + i];
    if constexpr (P::kBytes == 2) return bf16_up(static_cast<const uint16_t *>(pool)[row * D + i]);
    if constexpr (P::kBytes == 1) {
        float x[4];
        codes4_up(static_cast<const uint8_t *>(pool)[row * D + i], pow2_of(scale[row]), x);
        return x[0];
    }
}

template <class T, class P, int D>
__global__ void __launch_bounds__(64) attend_kernel(PageAttendArgs a) {
    const PageTables &t = a.t;
    const int Hq = t.Hkv << a.group_shift, lane = threadIdx.x;
    const int tok = blockIdx.x / Hq, h = blockIdx.x % Hq, g = h >> a.group_shift;
    if (tok >= t.tok_start[t.B]) return;
    int lo = 0, hi = t.B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.tok_start[mid] <= tok) lo = mid; else hi = mid;
    }
    const int b = lo, n = t.seq_len[b];
    const int64_t p64 = int64_t(n) - t.tok_start[b + 1] + tok;
    const int cap = t.max_pages << t.page_shift;
    const int pos = p64 < 0 ? -1 : int(p64);
    if (pos >= cap && lane == 0) flag(t);
    const int end = pos + 1 < cap ? pos + 1 : cap;
    const int begin = pos - (a.window - 1) > 0 ? pos - (a.window - 1) : 0;
    __shared__ float q[D], pr[64];
    __shared__ int rows[64];
    using E = typename T::elem;
    for (int i = lane; i < D; i += 64) {
        const E x = static_cast<const E *>(a.q)[int64_t(tok) * a.q_stride + h * D + i];
        if constexpr (T::kBytes == 4) q[i] = x; else q[i] = bf16_up(x);
    }
    float m = -INFINITY, l = 0.f, o[D / 64] = {};
    for (int j0 = begin; j0 < end; j0 += 64) {
        __syncthreads();
        const int j = j0 + lane;
        const int row = j < end ? pool_row(t, b, g, j) : -1;
        if (j < end && row < 0) flag(t);
        float s = -INFINITY;
        if (row >= 0) {
            float x = 0.f;
            for (int i = 0; i < D; ++i) x = fmaf(q[i], value_at<P>(a.k, a.k_scale, row, D, i), x);
            s = x * a.scale;
        }
        float mx = s;
        for (int k = 1; k < 64; k *= 2) { const float y = __shfl_xor(mx, k); mx = mx >= y || mx != mx ? mx : y; }
        const float mn = m >= mx || m != m ? m : mx;
        const float base = mn == -INFINITY ? 0.f : mn;
        const float alpha = expf(m - base), w = row >= 0 ? expf(s - base) : 0.f;
        m = mn;
        float sum = w;
        for (int k = 1; k < 64; k *= 2) sum += __shfl_xor(sum, k);
        l = l * alpha + sum;
        pr[lane] = w;
        rows[lane] = row;
        __syncthreads();
        for (int c = 0; c < D / 64; ++c) {
            o[c] *= alpha;
            for (int k = 0; k < 64; ++k)
                if (rows[k] >= 0) o[c] = fmaf(pr[k], value_at<P>(a.v, a.v_scale, rows[k], D, c * 64 + lane), o[c]);
        }
    }
    const bool none = l == 0.f;
    for (int c = 0; c < D / 64; ++c) {
        const float x = none ? 0.f : o[c] / l;
        const size_t at = (size_t(tok) * Hq + h) * D + c * 64 + lane;
        if constexpr (T::kBytes == 4) static_cast<float *>(a.out)[at] = x;
        else static_cast<uint16_t *>(a.out)[at] = uint16_t(bf16_pack(x, 0.f));
    }
    if (a.lse && lane == 0) a.lse[size_t(tok) * Hq + h] = none ? -INFINITY : m + logf(l);
}

template <class T, class P, int D>
hipError_t attend(const PageAttendArgs &a, hipStream_t s) {
    const int Hq = a.t.Hkv << a.group_shift;
    hipLaunchKernelGGL((attend_kernel<T, P, D>), dim3(unsigned(a.t.n_tokens) * Hq), dim3(64), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_page_attend(const PageAttendArgs &a, int dtype, int page_dtype, int head_dim, hipStream_t stream) {
    const bool q = page_dtype == SEKV_E4M3;
    if (dtype == SEKV_BF16) {
        if (head_dim == 128) return q ? attend<BF16, E4M3, 128>(a, stream) : attend<BF16, BF16, 128>(a, stream);
        return q ? attend<BF16, E4M3, 64>(a, stream) : attend<BF16, BF16, 64>(a, stream);
    }
    if (head_dim == 128) return q ? attend<F32, E4M3, 128>(a, stream) : attend<F32, F32, 128>(a, stream);
    return q ? attend<F32, E4M3, 64>(a, stream) : attend<F32, F32, 64>(a, stream);
}

}  // namespace sekv
