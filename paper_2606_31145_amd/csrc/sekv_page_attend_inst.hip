// Attention of new tokens over the paged store, one pair of storage types and head_dim an object.
//
// softmax in one pass: with m a bound of the scores so far, l = sum exp(s - m) and o = sum exp(s - m) v,
// a larger m scales l and o by exp(old - new).  A workgroup takes one item (sekv_page_index.h): a tile
// of query rows of one sequence and KV head against a chunk of its keys.  A tile whose keys lie in more
// than one chunk leaves partials (m, l, o), which the last of its workgroups joins, or a second kernel
// (join_in_launch in sekv_page_index.h).
//
// What bounds it: few rows, the keys' and values' bytes (sekv_page_tile.h); 128 bfloat16 rows, the matrix cores
// and the softmax's vector instructions in turn (sekv_page_wide.h); float rows, the float matrix instruction, over 4-bit
// pages the vector instructions that split weights and scale keys and values (sekv_page_split.h).
// The smallest calls are a chain of dependent reads (tables, page, rows, partials): one token over 2048 keys,
// which are 0.2 us of bytes, spends 3.0 us until its workgroups know the plan, 0.6 on finding their items, 3.4 on
// keys and values and 3.2 on the join.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "sekv_page_wide.h"

#if !defined(SEKV_T) || !defined(SEKV_P) || !defined(SEKV_D)
#error "build with -DSEKV_T=BF16|F32 -DSEKV_P=BF16|F32|E4M3|E2M1 -DSEKV_D=64|128"
#endif

namespace sekv {
namespace {

using namespace page;

constexpr int kThreads = 256, kWaves = 4;
constexpr int64_t kJoinBlocks = 2048;      // eight on each compute unit

// __syncthreads_or for a workgroup's one question, over 4-bit pages, whose items are the shortest: one token over 2048 keys
// takes 8.95 us with this and 9.1 with the library's.
__device__ inline bool any_thread(bool x, int lane, int wave) {
    __shared__ uint32_t told[kWaves];
    const bool here = __any(x);
    if (lane == 0) told[wave] = here;
    __syncthreads();
    return told[0] | told[1] | told[2] | told[3];
}
template <class P>
__device__ inline bool any_of(bool x, int lane, int wave) {
    if constexpr (P::kBytes == 0) return any_thread(x, lane, wave);
    else return __syncthreads_or(x);
}

// LDS of a workgroup's 16 NB rows: four waves' maxima and sums, then each wave's rows, where its queries pass before: what a
// wave writes early reaches no other's.
template <int D, int NB> constexpr int kRowBytes = 16 * NB * (D + 4) * 4;
template <int D, int NB>
__device__ inline unsigned char *own_rows(unsigned char *lds, int wave) {
    return lds + kWaves * 2 * 16 * NB * 4 + wave * kRowBytes<D, NB>;
}

// The four waves' parts of the same rows of an item, joined through LDS.  True when the item has to be done again by
// plain_rows.
template <class T, class P, int D, int NB>
__device__ inline bool join_waves(const PageAttendArgs &a, const Item &it, const Rows16<T, P, D, NB> &r, bool bad, int g, int c,
                                  int lane, int wave, unsigned char *lds) {
    constexpr int VE = D / 16, RS = D + 4, N = 16 * NB;
    float *ml = reinterpret_cast<float *>(lds), *so = ml + kWaves * 2 * N;
    const int n = lane & 15, gq = lane >> 4;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const float l = r.sum(nb);
        if (gq == 0) {
            ml[wave * 2 * N + 16 * nb + n] = r.m[nb];
            ml[wave * 2 * N + N + 16 * nb + n] = l;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < VE; ++e) so[(wave * N + 16 * nb + n) * RS + VE * (4 * gq + i) + e] = r.o[nb][e][i];
    }
    if (any_of<P>(bad, lane, wave)) return true;
    const int d0 = (threadIdx.x & 15) * 2;                   // and 32, 64, .. on: what 16 threads store lies together
    for (int rw = threadIdx.x >> 4; rw < it.rows; rw += 16) {
        float m = -INFINITY, sum = 0.f, o[VE / 2][2] = {};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) m = fmaxf(m, ml[w * 2 * N + rw]);
        const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = exp2_fast(ml[w * 2 * N + rw] - mu);
            sum += f * ml[w * 2 * N + N + rw];
#pragma unroll
            for (int e = 0; e < VE / 2; ++e) {
                const float *p = so + (w * N + rw) * RS + d0 + 32 * e;
                o[e][0] += f * p[0];
                o[e][1] += f * p[1];
            }
        }
#pragma unroll
        for (int e = 0; e < VE / 2; ++e)
            put<T, D>(a, it, c, it.tok0 + (rw >> a.group_shift), (g << a.group_shift) + (rw & ((1 << a.group_shift) - 1)),
                      d0 + 32 * e, o[e], m, sum);
    }
    return false;
}

// At most 16 NB rows: every wave takes all of them, and every fourth step of the keys.
template <class T, class P, int D, int NB>
__device__ inline bool narrow(const PageAttendArgs &a, const Item &it, int b, int g, int c, int lane, int wave, unsigned char *lds) {
    using R = Rows16<T, P, D, NB>;
    R r;
    bool bad = false;
    r.run(a, it, b, g, 0, it.begin + wave * R::Tile::kKeys, R::Tile::kKeys * kWaves, &bad, lane, own_rows<D, NB>(lds, wave));
    return join_waves<T, P, D, NB>(a, it, r, bad, g, c, lane, wave, lds);
}

// Up to 128 float rows: 32 to a wave, which reads all the item's keys.
template <class P, int D>
__device__ inline bool float_rows(const PageAttendArgs &a, const Item &it, int b, int g, int c, int lane, int wave, unsigned char *lds) {
    using R = Rows16<F32, P, D, 2>;
    R r;
    bool bad = false;
    if (wave * 32 < it.rows) r.run(a, it, b, g, wave * 32, it.begin, R::Tile::kKeys, &bad, lane, own_rows<D, 2>(lds, wave));
    if (any_of<P>(bad, lane, wave)) return true;
    if (wave * 32 >= it.rows) return false;
    const int n = lane & 15, gq = lane >> 4;
    if constexpr (P::kBytes == 0) {
        // through LDS, so that a store covers whole rows: straight from the registers it touches 64 of them
        constexpr int RS = D + 4, GT = D / 4;
        float *so = reinterpret_cast<float *>(own_rows<D, 2>(lds, wave));
        float m[2], l[2];
#pragma unroll
        for (int nb = 0; nb < 2; ++nb) {
            m[nb] = r.m[nb];
            l[nb] = r.sum(nb);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < R::VE; ++e) so[(16 * nb + n) * RS + R::VE * (4 * gq + i) + e] = r.o[nb][e][i];
        }
        wave_fence();
#pragma unroll 2
        for (int r0 = 0; r0 < 32; r0 += 64 / GT) {
            const int row = r0 + lane / GT, rw = wave * 32 + row, d0 = lane % GT * 4;
            const float4 x = *reinterpret_cast<const float4 *>(so + row * RS + d0);
            const float o[4] = {x.x, x.y, x.z, x.w};
            const float mr = __shfl(r0 < 16 ? m[0] : m[1], row & 15), lr = __shfl(r0 < 16 ? l[0] : l[1], row & 15);
            if (rw < it.rows)
                put<F32, D>(a, it, c, it.tok0 + (rw >> a.group_shift), (g << a.group_shift) + (rw & ((1 << a.group_shift) - 1)),
                            d0, o, mr, lr);
        }
        return false;
    }
#pragma unroll
    for (int nb = 0; nb < 2; ++nb) {
        const int rw = wave * 32 + nb * 16 + n;
        const float l = r.sum(nb);
        if (rw < it.rows) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float o[R::VE];
#pragma unroll
                for (int e = 0; e < R::VE; ++e) o[e] = r.o[nb][e][i];
                put<F32, D>(a, it, c, it.tok0 + (rw >> a.group_shift), (g << a.group_shift) + (rw & ((1 << a.group_shift) - 1)),
                            R::VE * (4 * gq + i), o, r.m[nb], l);
            }
        }
    }
    return false;
}

// One tile's work while the next one's bytes arrive.  The two tiles do not overlap, and saying so keeps the
// compiler from waiting for the arrival before it reads.
template <int D>
__device__ __forceinline__ void step_beside_load(const PageAttendArgs &a, Rows32<D> &r, const Direct<D> &dr, bool more, int next_row,
                                                 int own, lds_bytes __restrict__ kt, lds_bytes __restrict__ vt,
                                                 lds_bytes __restrict__ kn, lds_bytes __restrict__ vn, bool rows, int pos,
                                                 uint32_t valid, bool part, int lane) {
    if (more) dr.load(a, next_row, kn, vn, own);
    if (rows) r.step(a, kt, vt, pos, valid, part, lane);
}

// Up to 128 bfloat16 rows: tiles of 64 keys in LDS, two buffers; a wave fetches 16 keys of each.
template <class P, int D>
__device__ inline bool wide_bf16(const PageAttendArgs &a, const Item &it, int b, int g, int c, int lane, int wave, unsigned char *lds) {
    constexpr int kTile = 64 * D * 2;                        // bytes of a tile's keys or values
    Rows32<D> r;
    r.init(a, it, g, wave * 32, lane);
    const int64_t w = it.p0 + it.n_tok - 1 - (int64_t(a.window) - 1);
    const int64_t all_lo = w, all_hi = it.p0;                // keys that every row of the item sees
    constexpr bool kDirect = P::kBytes == 2;
    Stage<P, D> st;
    Direct<D> dr;
    bool bad = false;
    // everybody's part of a tile is in LDS
    auto arrived = [&]() {
        if (kDirect) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    // the four blocks of a tile, one a lane: their page, read two tiles ahead, then mine to fetch and which of
    // them hold keys
    auto page_of = [&](int pos) {
        const int p = pos + 16 * (lane & 3);
        return block_seen(it, p) ? a.t.table[int64_t(b) * a.t.max_pages + (p >> a.t.page_shift)] : -1;
    };
    auto rows_of = [&](int pos, int page, int *mine) {
        const int p = pos + 16 * (lane & 3), row = block_row(page, a.t.n_pages, a.t.Hkv, g, a.t.page_shift, p);
        if (row < 0 && block_seen(it, p) && lane < 4) flag(a.t);
        *mine = __builtin_amdgcn_readlane(row, wave);
        return uint32_t(__ballot(row >= 0)) & 15u;
    };
    auto partial = [&](int pos, uint32_t valid) { return valid != 15u || pos < all_lo || pos + 63 > all_hi; };
    const lds_bytes tile = (lds_bytes)lds;
    const int own = wave * 16;
    // rows of a tile that hold keys which some row of the item sees
    auto from_of = [&](int pos) { return it.first - pos; };
    auto end_of = [&](int pos, uint32_t valid) { return valid >> wave & 1 ? it.end - pos : 0; };
    int pos = it.begin, mine = -1;
    uint32_t valid = rows_of(pos, page_of(pos), &mine), ahead = 0;
    int page = page_of(pos + 64);
    if constexpr (kDirect) {
        dr.init(lane);
        dr.load(a, mine, tile, tile + 2 * kTile, own);
    } else {
        st.load(a, mine, lane);
        if (partial(pos, valid)) bad |= st.mend(own, from_of(pos), end_of(pos, valid), lane);
        st.store(lds, lds + 2 * kTile, own, lane);
    }
    arrived();
    // one tile from buffer kBuf, the next one into the other; false when that was the last
    auto turn = [&](auto kBuf) {
        constexpr int B = decltype(kBuf)::value;
        const bool more = pos + 64 < it.end;
        if (kDirect && partial(pos, valid)) {
            bad |= dr.mend(lds + (2 + B) * kTile, own, from_of(pos), end_of(pos, valid), lane);
            __syncthreads();
        }
        const bool part = partial(pos, valid), rows = wave * 32 < it.rows;
        if (more) {
            ahead = rows_of(pos + 64, page, &mine);
            page = page_of(pos + 128);
        }
        if constexpr (kDirect) {
            step_beside_load<D>(a, r, dr, more, mine, own, tile + B * kTile, tile + (2 + B) * kTile, tile + (1 - B) * kTile,
                                tile + (3 - B) * kTile, rows, pos, valid, part, lane);
        } else {
            if (more) st.load(a, mine, lane);
            if (rows) r.step(a, tile + B * kTile, tile + (2 + B) * kTile, pos, valid, part, lane);
            if (more) {
                if (partial(pos + 64, ahead)) bad |= st.mend(own, from_of(pos + 64), end_of(pos + 64, ahead), lane);
                st.store(lds + (1 - B) * kTile, lds + (3 - B) * kTile, own, lane);
            }
        }
        arrived();
        pos += 64;
        valid = ahead;
        return more;
    };
    if (it.begin < it.end)
        while (turn(std::integral_constant<int, 0>{}) && turn(std::integral_constant<int, 1>{})) {}
    if (__syncthreads_or(int(bad) | int(too_large(r.m)))) return true;
    const int n = lane & 31, h = lane >> 5, rw = wave * 32 + n;
    const float l = r.l + across32(r.l);
    if (rw < it.rows) {
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float o[4] = {r.o[db][4 * i], r.o[db][4 * i + 1], r.o[db][4 * i + 2], r.o[db][4 * i + 3]};
                put<BF16, D>(a, it, c, it.tok0 + (rw >> a.group_shift), (g << a.group_shift) + (rw & ((1 << a.group_shift) - 1)),
                             32 * db + 8 * i + 4 * h, o, r.m, l);
            }
    }
    return false;
}

template <class T, class P, int D>
__global__ void __launch_bounds__(kThreads, 2) attend_kernel(PageAttendArgs a) {
    constexpr int kNarrowLds = kWaves * kNarrowRows * (2 + D + 4) * 4, kWideLds = T::kBytes == 2 ? 4 * 64 * D * 2 : 0;
    __shared__ __attribute__((aligned(16))) unsigned char lds[kNarrowLds > kWideLds ? kNarrowLds : kWideLds];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (blockIdx.x == 0)                                     // tables that cannot be
        for (int b = threadIdx.x; b < a.t.B; b += kThreads) {
            const Seq s = load_seq(a, b);
            const int64_t cap = int64_t(a.t.max_pages) << a.t.page_shift;
            if (a.t.tok_start[b] != s.start || a.t.tok_start[b + 1] != s.start + s.nq || a.t.seq_len[b] < 0 ||
                (s.nq && a.t.seq_len[b] > cap))
                flag(a.t);
        }
    const Plan plan = make_plan<T, P>(a, lane, lds);
    int b = 0, c = 0, g = 0;
    const uint32_t x = place_of(blockIdx.x, a.t.Hkv, &g);
    Item it;
    if (!plan.chunk || !find_item<false, P::kBytes == 0>(a, x, lane, plan, lds, &b, &c, &it)) return;
    bool again;
    if (it.narrow && it.rows <= 16) again = narrow<T, P, D, 1>(a, it, b, g, c, lane, wave, lds);
    else if (it.narrow) again = narrow<T, P, D, 2>(a, it, b, g, c, lane, wave, lds);
    else if constexpr (T::kBytes == 2) again = wide_bf16<P, D>(a, it, b, g, c, lane, wave, lds);
    else again = float_rows<P, D>(a, it, b, g, c, lane, wave, lds);
    if (again) plain_rows<T, P, D>(a, it, b, g, c, lane, wave);
    if (it.chunk0 == it.chunk1 || a.join_launch) return;
    // the last of a tile's workgroups joins their partials: all stores of this one have to be out before it
    // counts itself, and the last one sets the counter back
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    __shared__ uint32_t before;
    uint32_t *cnt = a.arrived + size_t(it.tok0) * a.t.Hkv + g;
    if (threadIdx.x == 0) before = __hip_atomic_fetch_add(cnt, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (before != uint32_t(it.chunk1 - it.chunk0)) return;
    if (threadIdx.x == 0) __hip_atomic_store(cnt, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    join_rows<T, D, true>(a, it, g, 0, it.rows, lane, lds);
}

// Joins the partials of as many rows of a tile at a time as a workgroup holds side by side.
constexpr int join_parts(int D) { return kTileRows / (kThreads / (D / 4)); }
template <class T, class P, int D>
__global__ void __launch_bounds__(kThreads) join_kernel(PageAttendArgs a) {
    constexpr int kParts = join_parts(D), kRows = kTileRows / kParts;
    __shared__ __attribute__((aligned(16))) unsigned char lds[256 * (sizeof(float4) + sizeof(float2))];
    const int lane = threadIdx.x & 63;
    const Plan plan = make_plan<T, P>(a, lane, lds);
    if (!plan.chunk || plan.longest <= plan.chunk) return;   // nothing was cut
    const int64_t all = int64_t(plan.tiles) * a.t.Hkv * kParts;
    for (int64_t u = blockIdx.x; u < all; u += gridDim.x) {
        const int g = int(u % a.t.Hkv), part = int(u / a.t.Hkv % kParts);
        int b = 0, c = 0;
        Item it;
        find_item<true>(a, uint32_t(u / a.t.Hkv / kParts), lane, plan, lds, &b, &c, &it);
        const int left = it.rows - part * kRows;
        if (it.chunk0 == it.chunk1 || left <= 0) continue;
        join_rows<T, D, false>(a, it, g, part * kRows, left < kRows ? left : kRows, lane, lds);
    }
}

}  // namespace

#define SEKV_NAME2(t, p, d) launch_page_attend_##t##_##p##_##d
#define SEKV_NAME(t, p, d) SEKV_NAME2(t, p, d)

hipError_t SEKV_NAME(SEKV_T, SEKV_P, SEKV_D)(const PageAttendArgs &a, hipStream_t s) {
    using T = page::SEKV_T;
    using P = page::SEKV_P;
    hipLaunchKernelGGL((attend_kernel<T, P, SEKV_D>), dim3(unsigned(page::blocks_of(a.pairs, a.t.Hkv))), dim3(kThreads), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1 || !a.join_launch) return e;
    const int64_t parts = a.tiles * a.t.Hkv * join_parts(SEKV_D);
    hipLaunchKernelGGL((join_kernel<T, P, SEKV_D>), dim3(unsigned(parts < kJoinBlocks ? parts : kJoinBlocks)), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace sekv
