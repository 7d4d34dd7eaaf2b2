// Rotary positions over rows of heads: queries by themselves, or beside keys on their way into the paged store.
//
// A row is read once and written once, which is what bounds long calls: 32768 tokens of 32 heads of 128 in bfloat16
// (537 MB) take 99 us (5.4 TB/s, a copy 5.1), those of four 8192-token chunks with 8 heads of keys and values into 4 bits
// (707 MB) 138 us (5.1 TB/s).  Short ones are a chain of dependent reads: 32 tokens of 32 heads 3 us, with their keys 6.1,
// of which a wave spends most on looking up its tokens one after another.
// The unit of work is a wave, so that nothing waits for a workgroup (workgroups of 16 tokens, one row a lane in flight: 132
// and 185 us, but 5.2 for the 32 tokens with their keys):
//   - queries: one token and a range of its heads, which lie together.  A lane forms one pair's cos and sin, the wave
//     meets in LDS, and each lane takes those of its piece for all the heads.
//   - keys and values: as many consecutive tokens as a wave holds rows side by side, head by head, for consecutive tokens
//     are consecutive rows of a page.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "sekv_rotary.h"

namespace sekv {
namespace {

using namespace page;

constexpr int kThreads = 256, kWaves = 4;
constexpr int64_t kMaxBlocks = 1 << 21;   // a launch stays below 2^32 threads
constexpr int kSteps = 4;                 // query rows of a lane in flight
struct NoPages {};

// Which sequence a new token belongs to and its position there, for tokens that are the same in all lanes.  Up to 64
// sequences are one a lane, read once; of more, one in 64 is looked at first.
struct Places {
    int from, to, len;

    __device__ void init(const PageTables &t, int lane) {
        if (t.B > 64) return;
        const int b = lane < t.B ? lane : t.B - 1;
        from = t.tok_start[b];
        to = t.tok_start[b + 1];
        len = t.seq_len[b];
    }
    // False for a token that is nobody's.
    __device__ bool find(const PageTables &t, int tok, int lane, int *b, int64_t *pos) const {
        int first = 0, end, n;
        if (t.B <= 64) {
            const unsigned long long in = __ballot(lane < t.B && from <= tok);
            if (!(in & 1)) return false;                     // before the first
            first = 63 - __builtin_clzll(in);
            end = __builtin_amdgcn_readlane(to, first);
            n = __builtin_amdgcn_readlane(len, first);
        } else {
            for (int left = t.B;;) {                         // among tok_start[first .. first + left - 1]
                const int step = (left + 63) / 64, at = lane * step;
                const unsigned long long in = __ballot(at < left && t.tok_start[first + (at < left ? at : 0)] <= tok);
                if (!(in & 1)) return false;
                const int l = 63 - __builtin_clzll(in);
                first += l * step;
                if (step == 1) break;
                left = left - l * step < step ? left - l * step : step;
            }
            end = t.tok_start[first + 1];
            n = t.seq_len[first];
        }
        *b = first;
        *pos = int64_t(n) - end + tok;
        return tok < end;
    }
};

// (cos, sin) of a pair, as the call wants them.
__device__ inline double2 pair_of(const RotaryArgs &a, double position, double freq) {
    const double2 p = cos_sin(position * freq);
    return make_double2(a.scale * p.x, a.transpose ? -a.scale * p.y : a.scale * p.y);
}

template <class T, int D, bool kHalf, bool kPages>
__device__ inline void turn_queries(const RotaryArgs &a, uint32_t item, double2 *pairs, int lane) {
    constexpr int N = Piece<T>::kN, L = D / N, kSide = 64 / L;       // heads side by side
    const int tok = int(item / uint32_t(a.q_chunks)), h0 = int(item % uint32_t(a.q_chunks)) * a.q_per * kSide;
    const int h1 = h0 + a.q_per * kSide < a.Hq ? h0 + a.q_per * kSide : a.Hq;
    const unsigned char *src = static_cast<const unsigned char *>(a.q) + int64_t(tok) * a.q_stride * T::kBytes;
    unsigned char *dst = static_cast<unsigned char *>(a.q_out) + int64_t(tok) * a.out_stride * T::kBytes;
    const int mine = lane / L, piece = lane % L;
    u4v w[kSteps];
    auto load = [&](int h) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int u = h + i * kSide + mine;
            w[i] = u4v{0, 0, 0, 0};
            if (u < h1) w[i] = reinterpret_cast<const u4v *>(src + u * (D * T::kBytes))[piece];
        }
    };
    load(h0);                                                // rows of the call's buffers, turned or not
    const double freq = lane < a.rot_dim / 2 ? a.freq[lane] : 0.0;
    int64_t p = 0;
    if constexpr (kPages) {
        Places places;
        places.init(a.t, lane);
        int b;
        if (!places.find(a.t, tok, lane, &b, &p)) return;
    }
    if (a.positions) p = a.positions[tok];
    if (lane < a.rot_dim / 2) pairs[lane] = pair_of(a, double(p), freq);
    wave_fence();
    Turn<T, D, kHalf> turn;
    turn.init(pairs, a.rot_dim, piece);
    for (int h = h0; h < h1; h += kSteps * kSide) {
        if (h != h0) load(h);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const u4v r = turn.apply(w[i]).raw();
            const int u = h + i * kSide + mine;
            if (u < h1) reinterpret_cast<u4v *>(dst + u * (D * T::kBytes))[piece] = r;
        }
    }
}

template <class T, class P, int D, bool kHalf>
__device__ inline void store_keys(const RotaryArgs &a, uint32_t item, double2 *pairs, int lane) {
    constexpr int N = Piece<T>::kN, L = D / N, kRows = 64 / L;
    const PageTables &t = a.t;
    const int R2 = a.rot_dim / 2, row = lane / L, piece = lane % L;
    const int64_t tok0 = int64_t(item / uint32_t(a.kv_chunks)) * kRows, tok = tok0 + row;
    const int g0 = int(item % uint32_t(a.kv_chunks)) * a.kv_per, g1 = g0 + a.kv_per < t.Hkv ? g0 + a.kv_per : t.Hkv;
    u4v w[2];
    auto load = [&](int g) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            w[s] = u4v{0, 0, 0, 0};
            if (tok < t.n_tokens)
                w[s] = reinterpret_cast<const u4v *>(static_cast<const unsigned char *>(a.kv.src[s]) +
                                                     (tok * a.kv.stride[s] + int64_t(g) * D) * T::kBytes)[piece];
        }
    };
    load(g0);                                                // rows of the call's buffers, stored or not
    const double freq = lane < R2 ? a.freq[lane] : 0.0;      // asked for before the tables, too
    Places places;
    places.init(t, lane);
    int to = -1;                                             // the lane's token's pool row of head 0
    double p = 0.0;                                          // and position
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int64_t x = tok0 + r;
        int b;
        int64_t pos;
        if (x >= t.n_tokens || !places.find(t, int(x), lane, &b, &pos)) continue;
        const int at = first_row(t, b, pos);
        if (at < 0 && lane == 0) flag(t);
        to = row == r ? at : to;
        p = row == r ? double(a.positions ? a.positions[x] : pos) : p;
    }
    double *where = reinterpret_cast<double *>(pairs + kRows * (D / 2));
    if (piece == 0) where[row] = p;
    wave_fence();
    for (int i = lane; i - lane < kRows * R2; i += 64) {     // all lanes, for the frequencies are in them
        const int r = int(uint32_t(i) / uint32_t(R2));
        const double f = __shfl(freq, i - r * R2);
        if (i < kRows * R2) pairs[i] = pair_of(a, where[r], f);
    }
    wave_fence();
    Turn<T, D, kHalf> turn;
    turn.init(pairs + row * R2, a.rot_dim, piece);
    for (int g = g0; g < g1; ++g) {
        const u4v k = w[0], v = w[1];
        if (g + 1 < g1) load(g + 1);
        const Computed<T> x = turn.apply(k);
        if (to >= 0) {
            const int at = to + (g << t.page_shift);
            store_row<Computed<T>, P, D>(a.kv.pool[0], a.kv.scale[0], at, x, piece);
            store_row<Piece<T>, P, D>(a.kv.pool[1], a.kv.scale[1], at, Piece<T>{v}, piece);
        }
    }
}

template <class T, class P, int D, bool kHalf>
__global__ void __launch_bounds__(kThreads) rotary_kernel(RotaryArgs a) {
    constexpr bool kPages = !std::is_same_v<P, NoPages>;
    constexpr int kRows = 64 / (D / Piece<T>::kN), kPairs = kPages ? kRows * (D / 2) + kRows / 2 : D / 2;   // positions behind
    __shared__ double2 pairs[kWaves][kPairs];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int64_t c = int64_t(blockIdx.x) * kWaves + wave; c < a.kv_items + a.q_items; c += int64_t(gridDim.x) * kWaves) {
        wave_fence();
        if constexpr (kPages) {
            if (c < a.kv_items) {
                store_keys<T, P, D, kHalf>(a, uint32_t(c), pairs[wave], lane);
                continue;
            }
        }
        turn_queries<T, D, kHalf, kPages>(a, uint32_t(c - a.kv_items), pairs[wave], lane);
    }
    if constexpr (kPages) {
        if (blockIdx.x == 0) {                               // offsets that cannot be
            const PageTables &t = a.t;
            bool wrong = t.tok_start[0] < 0 || t.tok_start[t.B] > t.n_tokens;
            for (int i = threadIdx.x; i < t.B; i += kThreads) wrong |= t.tok_start[i] > t.tok_start[i + 1];
            if (wrong) flag(t);
        }
    }
}

// Waves aimed at: a call of few tokens is spread over its heads, so that there are about so many, or one a token (keys:
// one for its tokens).  Each finds its tokens and forms their angles anew.  With 8192 and 2048, 8192 and 1024, 4096 and
// 1024, 2048 and 1024, 2048 and 512 (us): 2048 tokens of 32 and 8 heads into 4 bits 16.5, 14.9, 12.7, 11.9, 13.0, about
// 10 000 ragged float tokens of 12 and 12 into 8 bits 21.9, 19.8, 18.8, 18.8, 18.9.
constexpr int64_t kQueryItems = 2048, kKeyItems = 1024;

// Heads in chunks of `per` steps, so that there are about so many items.
int chunks_of(int64_t items, int64_t tokens, int steps, int *per) {
    const int64_t want = (items + tokens - 1) / tokens;
    int n = int(want < steps ? want : steps);
    *per = (steps + n - 1) / n;
    return (steps + *per - 1) / *per;
}

template <class T, class P, int D, bool kHalf>
hipError_t launch(RotaryArgs a, hipStream_t s) {
    constexpr int kSide = 64 / (D / Piece<T>::kN);
    if (!std::is_same_v<P, NoPages>) {
        const int64_t groups = (int64_t(a.t.n_tokens) + kSide - 1) / kSide;
        a.kv_chunks = chunks_of(kKeyItems, groups, a.t.Hkv, &a.kv_per);
        a.kv_items = groups * a.kv_chunks;
    }
    if (a.Hq) {
        a.q_chunks = chunks_of(kQueryItems, a.t.n_tokens, (a.Hq + kSide - 1) / kSide, &a.q_per);
        a.q_items = int64_t(a.t.n_tokens) * a.q_chunks;
    }
    const int64_t blocks = (a.kv_items + a.q_items + kWaves - 1) / kWaves;
    hipLaunchKernelGGL((rotary_kernel<T, P, D, kHalf>), dim3(unsigned(blocks < kMaxBlocks ? blocks : kMaxBlocks)), dim3(kThreads), 0, s, a);
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
