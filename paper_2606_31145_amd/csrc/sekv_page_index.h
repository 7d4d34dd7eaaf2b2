// Where a row of the paged store lies, and which workgroup of sekv_page_attend does what: integer
// arithmetic only, also compiled for the host, where a test walks through it.
//
// Work items.  The query rows of a sequence and KV head (its new tokens x its query heads) are cut
// into tiles: of kTileRows, or, when there are at most kFewRows, into narrow tiles of kNarrowRows.  A tile's keys
// are cut into chunks so that few rows over many keys still fill the device.  The chunk length is
// found from the device's tables, the same for the whole call: with T_b tiles and L_b keys of
// sequence b, W = sum T_b L_b and T = sum T_b, chunk >= max(W / target, max L_b / splits) in steps of
// kChunkStep keys.  Then there are at most sum T_b + target (tile, chunk) pairs, whatever the lengths: the grid
// can be sized before they are known, and no sequence gets more than `splits` chunks.
//
// Above that bound the length follows a model of the time, in keys: an item costs its keys and
// `over` more (its start, and the join of its partial), and `slots` items run at once.  Where
// the lengths are alike, k full rounds of items cost k (L / n + over) with n = k slots / T chunks a
// tile; the best of a few k is taken, or no cut at all.  Where they differ, the time is at most
// (W + (W / chunk) over) / slots + chunk, the last term being the item that ends last; that is least
// at chunk = sqrt(W over / slots).  Where a tile's last workgroup joins its partials, each chunk costs it about one
// key's time a row as well: a longest sequence of L keys then asks for no more than sqrt(L / rows) chunks.
// With and without that term: nine tokens of 2 heads over 35714 keys of one KV head 40 and 112 us, two of 4 over
// 14199 of two 16 and 32, four of 11 ragged sequences of up to 22057 30 and 42, one over 2048 10.4 and 12.5.
// Measured (us): `over` of 64, 128 and 256 keys where partials are joined
// in the last workgroup: one token of 8 users at 9000 in 8 bits 34.6, 34.7, 34.7; of 256, 512 and 1024 where
// a second kernel joins them: 13 ragged sequences, one of 257 tokens, 97.3, 96.4, 90.9, one of 257 alone 65.0,
// 65.0, 64.6.  Steps of 64 and 128 keys: 333 float tokens at 3000 86.4 and 94.5, one token at 2048 9.9 and 10.6.
//
// kFewRows: 48 rows of 16 sequences under a window of 4096, 8 bits: 33.8 as two narrow tiles each, 41 as one
// tile of 128; 60 rows of 8 at 9000: 51.6 and 58.8 in 8 bits, 76.9 and 76.4 in bfloat16.
#pragma once

#include <math.h>
#include <stdint.h>

#ifdef __HIPCC__
#define SEKV_HD __host__ __device__ inline
#else
#define SEKV_HD inline
#endif

namespace sekv {
namespace page {

constexpr int kNarrowRows = 32;    // one or two 16-wide matrix tiles
constexpr int kFewRows = 64;       // rows of two narrow tiles, which read the keys twice, the second time from cache
constexpr int kTileRows = 128;     // 32 rows for each of four waves
constexpr int kChunkStep = 64;     // keys: a tile of the wide form, one or two steps of four waves in the narrow one
constexpr int kSlots = 512;        // workgroups that run at once: two on each of 256 compute units
constexpr int kOver = 128, kOverWide = 1024;     // keys that an item costs beside its own; of the wide bfloat16 form
SEKV_HD int over_of(bool wide, bool is_float) { return wide && !is_float ? kOverWide : kOver; }
// What the join of a chunk costs the last workgroup of a tile, in keys; a second kernel spreads it.
SEKV_HD float join_rows_of(bool wide, int n_tokens, int group_shift, int T) {
    return wide || T < 1 ? 0.f : float(int64_t(n_tokens) << group_shift) / float(T);
}
constexpr int kBlock = 16;         // keys that lie in one page: the smallest page

// Pool row of position `pos` (below max_pages * page_size) from its table entry; -1 when the page is
// outside the pool.  The kBlock positions from a multiple of kBlock on are consecutive rows.
SEKV_HD int block_row(int page, int n_pages, int Hkv, int g, int page_shift, int pos) {
    if (uint32_t(page) >= uint32_t(n_pages)) return -1;
    return ((page * Hkv + g) << page_shift) | (pos & ((1 << page_shift) - 1));
}

// One sequence of a call.  Positions stay what seq_len says; only keys are cut off at the capacity.
struct Seq {
    int start, nq;        // its rows of the new tokens
    int64_t first;        // position of the first new token (may be negative)
    int lo, len;          // keys lo .. lo + len - 1 are seen by some query; lo a multiple of kChunkStep
    int tiles;
};

SEKV_HD Seq make_seq(int start, int end, int seq_len, int n_tokens, int64_t cap, int window, int group_shift) {
    Seq s;
    start = start < 0 ? 0 : start > n_tokens ? n_tokens : start;
    end = end < start ? start : end > n_tokens ? n_tokens : end;
    s.start = start;
    s.nq = end - start;
    const int n = seq_len < 0 ? 0 : seq_len;
    s.first = int64_t(n) - s.nq;
    int64_t lo = s.first - (int64_t(window) - 1), hi = n < cap ? n : cap;
    lo = lo < 0 ? 0 : lo / kChunkStep * kChunkStep;
    s.lo = int(lo < hi ? lo : 0);
    s.len = s.nq && lo < hi ? int(hi - lo) : 0;
    const int rows = s.nq << group_shift;
    const int per = rows <= kFewRows ? kNarrowRows : kTileRows;
    s.tiles = (rows + per - 1) / per;
    return s;
}

// A 64-bit quotient costs a wave some 150 instructions, a 32-bit one a fifth: every workgroup starts with
// these.
SEKV_HD uint64_t quotient(uint64_t a, uint32_t b) { return a >> 32 ? a / b : uint64_t(uint32_t(a) / b); }

// W, T: of one KV head
SEKV_HD int chunk_length(uint64_t W, int T, int max_len, int Hkv, int target, int splits, int over, float rows) {
    if (T < 1) return kChunkStep;
    uint64_t c = quotient(W + target - 1, uint32_t(target));
    const uint32_t d = (uint32_t(max_len) + uint32_t(splits) - 1) / uint32_t(splits);
    c = c > d ? c : d;
    const float mean = float(W) / float(T), all = float(T) * float(Hkv), len = float(max_len);
    float best = float(max_len);                             // no cut
    if (float(max_len) <= 1.1f * mean) {
        const int rounds = int((all + float(kSlots - 1)) / float(kSlots));
        float cost = float(rounds) * float(max_len);
        for (int k = 0; k <= 4; ++k) {
            float n = float(int(float((k ? k : 1) * kSlots) / all));
            if (k == 0) {                                    // fewer chunks than fill the device
                const float few = sqrtf(len / (rows + 1e-3f));
                n = n < few ? n : few;
            }
            const float x = n > 1.f ? float(k ? k : 1) * (len / n + float(over)) + n * rows : cost;
            best = x < cost ? len / n : best;
            cost = x < cost ? x : cost;
        }
    } else {
        const float x = sqrtf(mean * all * float(over) / float(kSlots) + len * rows);
        best = x < best ? x : best;
    }
    const uint32_t m = uint32_t(best) + 1;
    c = c > m ? c : m;
    const uint32_t r = uint32_t(c > (1u << 30) ? (1u << 30) : c);
    return int((r + kChunkStep - 1) / kChunkStep * kChunkStep);
}
SEKV_HD int chunks_of(const Seq &s, int chunk) { return s.len > chunk ? (s.len + chunk - 1) / chunk : 1; }

// What one item covers.
struct Item {
    int tok0, n_tok;      // tokens of the tile
    int rows;             // n_tok << group_shift
    bool narrow;
    int64_t p0;           // position of its first token
    int first;            // first key that one of its rows sees (at most the capacity)
    int begin, end;       // keys (begin a multiple of 64); empty when begin >= end
    int chunk0, chunk1;   // first and last chunk with keys of the tile; equal: no join is needed
    bool idle;            // nothing to do
};

SEKV_HD Item make_item(const Seq &s, int tile, int c, int chunk, int64_t cap, int window, int group_shift) {
    Item it;
    const int per = ((s.nq << group_shift) <= kFewRows ? kNarrowRows : kTileRows) >> group_shift;
    const int t0 = tile * per, left = s.nq - t0;
    it.tok0 = s.start + t0;
    it.n_tok = left < per ? left : per;
    it.rows = it.n_tok << group_shift;
    // The rest behind tiles of 128 rows is narrow, too: 13 ragged sequences, one of 257 tokens, 687 us against 739
    // in float, 89.3 against 90.6 in bfloat16.
    it.narrow = it.rows <= kNarrowRows;
    it.p0 = s.first + t0;
    const int64_t b64 = it.p0 - (int64_t(window) - 1), e64 = it.p0 + it.n_tok;
    const uint32_t b = b64 < 0 ? 0u : b64 < cap ? uint32_t(b64) & ~63u : uint32_t(cap);
    const uint32_t e = e64 < 0 ? 0u : e64 < cap ? uint32_t(e64) : uint32_t(cap);
    it.first = int(b64 < 0 ? 0 : b64 < cap ? b64 : cap);
    it.begin = it.end = 0;
    it.chunk0 = it.chunk1 = 0;
    it.idle = c != 0;
    if (b >= e) return it;                         // no key: the first chunk's item says so
    it.chunk0 = int((b - uint32_t(s.lo)) / uint32_t(chunk));
    it.chunk1 = int((e - 1 - uint32_t(s.lo)) / uint32_t(chunk));
    it.idle = c < it.chunk0 || c > it.chunk1;
    if (it.idle) return it;
    const uint32_t cb = uint32_t(s.lo) + uint32_t(c) * uint32_t(chunk), ce = cb + uint32_t(chunk);    // below 2^31
    it.begin = int(b > cb ? b : cb);
    it.end = int(e < ce ? e : ce);
    return it;
}

// Whether some row of the item sees a key of the block at pos.  An item begins at a multiple of 64, so under a
// window its first blocks may lie before every row's: their page may be somebody else's by then, or none.
SEKV_HD bool block_seen(const Item &it, int pos) { return pos < it.end && pos + kBlock > it.first; }

// Host side: grid and workspace of a call.
struct Launch {
    int splits;           // chunks a tile may have
    int target;           // (tile, chunk) pairs aimed at
    int64_t tiles;        // tiles of a KV head at most
    int64_t pairs;        // (tile, chunk) pairs at most
};

// One tile a sequence that has tokens, another one for those of more than kNarrowRows and at most kFewRows
// rows, and one for every kTileRows rows.
SEKV_HD int64_t most_tiles(int batch, int n_tokens, int group_shift) {
    const int64_t rows = int64_t(n_tokens) << group_shift, n = batch < n_tokens ? batch : n_tokens;
    const int64_t second = rows / (kNarrowRows + 1);
    return n + (second < n ? second : n) + rows / kTileRows;
}

SEKV_HD int most_splits(int64_t cap) {
    const int64_t n = (cap + kChunkStep - 1) / kChunkStep;
    return int(n > 256 ? 256 : n);
}
// Counters of a workspace, [n_tokens][Hkv].  The same for all dims, so that calls of any shape, captured ones
// among them, keep them in one place that no call's partials reach.  More tokens than that are about as many tiles
// as fill the device: they are not cut, and neither is a long sequence's single token beside them.
constexpr int kCounters = 1 << 17;
// `items`: how many work items fill the device.
SEKV_HD Launch plan_launch(int batch, int n_tokens, int Hkv, int group_shift, int64_t cap, int items) {
    Launch l;
    const int64_t rows = int64_t(n_tokens) << group_shift, r = rows > kTileRows ? rows : kTileRows;
    l.target = (items + Hkv - 1) / Hkv;
    const int64_t s = (int64_t(l.target) * kTileRows + r - 1) / r;
    const int most = most_splits(cap);
    l.splits = int64_t(n_tokens) * Hkv > kCounters ? 1 : int(s < most ? s : most);
    l.tiles = most_tiles(batch, n_tokens, group_shift);
    l.pairs = l.tiles + (l.splits > 1 ? l.target : 0);
    return l;
}
// Rows of partials (of all heads) that any call of up to n_tokens tokens needs: splits * rows is at
// most target * kTileRows + rows, and at most most_splits * rows.
SEKV_HD int64_t partial_rows(int n_tokens, int Hkv, int group_shift, int64_t cap, int items) {
    const int64_t rows = int64_t(n_tokens) << group_shift, target = (items + Hkv - 1) / Hkv;
    const int64_t a = target * kTileRows + rows, b = rows * most_splits(cap);
    return (a < b ? a : b) * Hkv;
}

// Whether the partials go to a second kernel.  Joining in the last workgroup of a tile saves a launch but
// leaves a tile of 128 rows to one compute unit, so it is for tiles that are probably narrow; more rows
// than sequences of narrow tiles hold mean that some tile is not.  Fewer do not mean that none is: a chunk beside
// many single tokens is joined in the last workgroups of its 128-row tiles, too, for the whole call goes one way.
// Measured (us), joined in the last workgroup and by a second kernel: one token over 2048 float keys 10.4, 12.3,
// of 8 sequences at 9001 in 8 bits 30.5, 36.0, six of 16 under a window of 4096 30.9, 35.5; 257 over 9001 90.8, 60.6,
// 13 ragged sequences, one of 257 tokens, 117.7, 90.3, two of 333 in float 75.3, 58.0; 8 heads at 9000 keys in 8 bits, 128 ragged single tokens at
// 2000 85.9, 116.8, 31 and a chunk of 257 203.8, 190.3, 31 and one of 480 222.6, 237.7, 63 and one of 512 383.3, 376.3;
// in bfloat16 140.0, 174.0; 283.8, 275.8; 305.4, 352.6; 541.9, 539.9.
SEKV_HD bool join_in_launch(int batch, int n_tokens, int group_shift) {
    return (int64_t(n_tokens) << group_shift) > int64_t(batch) * kFewRows;
}

// Workgroup -> (pair, KV head).  Consecutive workgroups go to the chip's 8 dies in turn, each with a cache of
// its own, and neighbouring pairs read the same keys.  With 8 heads a head stays on a die by itself; with 1, 2
// or 4 a die takes kNear neighbouring pairs of a head: six tokens of 16 sequences over 4096 keys of 4 heads
// 40.2 us in bfloat16 against 56.2 with kNear 1, 30.6 against 37.6 in 8 bits.
constexpr int kDies = 8, kNear = 8;
SEKV_HD bool few_heads(int Hkv) { return Hkv == 1 || Hkv == 2 || Hkv == 4; }
SEKV_HD int64_t blocks_of(int64_t pairs, int Hkv) {
    const int64_t group = few_heads(Hkv) ? kDies / Hkv * kNear : 1;
    return (pairs + group - 1) / group * group * Hkv;
}
SEKV_HD uint32_t place_of(uint32_t block, int Hkv, int *g) {
    *g = int(block % uint32_t(Hkv));
    if (!few_heads(Hkv)) return block / uint32_t(Hkv);
    const uint32_t side = kDies / Hkv, die = block % kDies, turn = block / kDies;
    return turn / kNear * (side * kNear) + die / uint32_t(Hkv) * kNear + turn % kNear;
}

}  // namespace page
}  // namespace sekv
