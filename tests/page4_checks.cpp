// The schedule of sekv_page_attend over 4-bit pages walked through on the host (sekv_page_index.h): with that storage's
// constants every key that a query sees is in exactly one item, items fit the grid and partials the workspace, whichever
// way they are joined; and the order with wide tiles first hands every pair to one workgroup.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "sekv_page_index.h"

using namespace sekv::page;

#define REQUIRE(c)                                                              \
    do {                                                                        \
        if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); std::exit(1); } \
    } while (0)

struct Tables {
    std::vector<int> start, len;
    int n_tokens;
};

// Pairs in the order of find_item: sequences as they are, or those of wide tiles first.
static void walk_pairs(const std::vector<Seq> &seq, int chunk, int gs, int64_t pairs) {
    const int B = int(seq.size());
    for (int order = 0; order < 2; ++order) {
        uint64_t wide = 0;
        for (int b = 0; b < B && order; ++b) wide |= uint64_t((seq[b].nq << gs) > kFewRows) << b;
        int64_t n[64] = {};
        int whose[64], hit[64] = {};
        for (int lane = 0; lane < 64; ++lane) {
            const int to = order ? wide_first(wide, lane) : lane;
            REQUIRE(to >= 0 && to < 64 && !hit[to]);
            hit[to] = 1;
            whose[to] = lane;
            n[to] = lane < B ? int64_t(seq[lane].tiles) * chunks_of(seq[lane], chunk) : 0;
        }
        bool narrow = false;                                 // a wide sequence behind a narrow one
        for (int at = 0; at < 64 && order; ++at) {
            if (n[at] == 0) continue;
            REQUIRE(!(narrow && (wide >> whose[at] & 1)));
            narrow |= !(wide >> whose[at] & 1);
        }
        std::vector<std::vector<int>> got(B);
        for (int b = 0; b < B; ++b) got[b].assign(size_t(seq[b].tiles) * chunks_of(seq[b], chunk), 0);
        for (int64_t x = 0; x < pairs; ++x) {
            int64_t in = x;
            int at = 0;
            while (at < 64 && in >= n[at]) in -= n[at++];
            if (at == 64) continue;
            REQUIRE(whose[at] < B);
            got[whose[at]][size_t(in)] += 1;
        }
        for (auto &g : got)
            for (int v : g) REQUIRE(v == 1);
    }
}

static void walk(const Tables &t, int Hkv, int gs, int64_t cap, int window, bool is_float, bool join_launch) {
    const int B = int(t.len.size()), items = items_of(true);
    const Launch l = plan_launch(B, t.n_tokens, Hkv, gs, cap, items);
    REQUIRE((int64_t(t.n_tokens) << gs) * Hkv * l.splits <= partial_rows(t.n_tokens, Hkv, gs, cap, items));
    std::vector<Seq> seq;
    uint64_t W = 0;
    int mx = 0, T = 0;
    for (int b = 0; b < B; ++b) {
        seq.push_back(make_seq(t.start[b], t.start[b + 1], t.len[b], t.n_tokens, cap, window, gs));
        W += uint64_t(seq[b].tiles) * uint64_t(seq[b].len);
        T += seq[b].tiles;
        mx = mx > seq[b].len ? mx : seq[b].len;
    }
    const int chunk = l.splits == 1 ? 1 << 30
                                    : call_chunk(W, T, mx, Hkv, l.target, l.splits, t.n_tokens, gs, join_launch, is_float, true);
    REQUIRE(chunk % kChunkStep == 0 && chunk > 0);
    std::vector<std::vector<int>> seen(t.n_tokens);
    for (auto &v : seen) v.assign(size_t(cap), 0);
    int64_t pairs = 0;
    for (const Seq &s : seq) {
        const int n = chunks_of(s, chunk);
        REQUIRE(n <= l.splits);
        pairs += int64_t(s.tiles) * n;
        for (int c = 0; c < n; ++c)
            for (int tile = 0; tile < s.tiles; ++tile) {
                const Item it = make_item(s, tile, c, chunk, cap, window, gs);
                if (it.idle) continue;
                REQUIRE(it.chunk0 >= 0 && it.chunk0 <= it.chunk1 && it.chunk1 < n);
                for (int i = 0; i < it.n_tok; ++i)
                    for (int j = it.begin; j < it.end; ++j)
                        if (j <= it.p0 + i && j > it.p0 + i - int64_t(window)) seen[it.tok0 + i][j] += 1;
            }
    }
    REQUIRE(pairs <= l.pairs && T <= l.tiles);
    for (int b = 0; b < B; ++b)
        for (int i = t.start[b]; i < t.start[b + 1]; ++i) {
            const int64_t p = int64_t(t.len[b]) - t.start[b + 1] + i;
            for (int64_t j = 0; j < cap; ++j) REQUIRE(seen[i][j] == (j <= p && j > p - int64_t(window) ? 1 : 0));
        }
    walk_pairs(seq, chunk, gs, l.pairs);
}

int main() {
    std::mt19937 r(11);
    auto in = [&](int a, int b) { return int(r() % unsigned(b - a + 1)) + a; };
    for (int trial = 0; trial < 1500; ++trial) {
        const int B = in(0, 3) ? in(1, 7) : in(8, 64), gs = in(0, 3), Hkv = in(1, 9), shift = in(4, 7);
        const int max_pages = in(1, 1 + ((B > 7 ? 300 : 3000) >> shift));
        const int64_t cap = int64_t(max_pages) << shift;
        const int window = in(0, 2) ? 0x7fffffff : in(1, int(cap) + 5);
        Tables t;
        t.start = {0};
        for (int b = 0; b < B; ++b) {
            const int len = in(0, 9) ? in(0, int(cap)) : in(0, 2), kind = in(0, B > 7 ? 5 : 3);
            const int q = kind == 1 ? in(0, 5) : kind == 2 ? in(0, 150) : kind == 3 ? len + in(0, 1) * 3 : 1;
            t.len.push_back(len);
            t.start.push_back(t.start.back() + (q < 300 ? q : 300));
        }
        t.n_tokens = t.start.back() + in(0, 3);
        const bool launch = join_in_launch(B, t.n_tokens, gs);
        walk(t, Hkv, gs, cap, window, trial % 2 != 0, launch);
        walk(t, Hkv, gs, cap, window, trial % 2 != 0, !launch);
    }
    // every number of sequences, any of them wide
    for (int B = 0; B <= 64; ++B)
        for (int trial = 0; trial < 200; ++trial) {
            uint64_t wide = (uint64_t(r()) << 32 | r()) & (B == 64 ? ~uint64_t(0) : (uint64_t(1) << B) - 1);
            if (trial % 3 == 0) wide &= uint64_t(r()) << 32 | r();
            uint64_t taken = 0;
            int last[2] = {-1, -1};
            for (int lane = 0; lane < 64; ++lane) {
                const int to = wide_first(wide, lane), kind = int(wide >> lane & 1);
                REQUIRE(to >= 0 && to < 64 && !(taken >> to & 1) && to > last[kind]);
                taken |= uint64_t(1) << to;
                last[kind] = to;
            }
            REQUIRE(last[1] < 0 || last[1] + 1 == __builtin_popcountll(wide));
        }
    std::printf("all 4-bit page checks passed\n");
    return 0;
}
