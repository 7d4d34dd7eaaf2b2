// Walks through the work items of sekv_page_attend on the host (sekv_page_index.h): over random ragged
// batches, every key that a query sees is in exactly one item, items fit the grid, chunks fit the
// workspace, and rows of pages lie in the pool, also where the tables are wrong.
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

static void walk(const Tables &t, int Hkv, int gs, int64_t cap, int window, int items, bool good) {
    const int B = int(t.len.size());
    const Launch l = plan_launch(B, t.n_tokens, Hkv, gs, cap, items);
    REQUIRE(l.splits >= 1 && l.splits <= 256 && l.target >= 1);
    REQUIRE((int64_t(t.n_tokens) << gs) * Hkv * l.splits <= partial_rows(t.n_tokens, Hkv, gs, cap, items));
    REQUIRE(partial_rows(t.n_tokens, Hkv, gs, cap, items) <= partial_rows(t.n_tokens + 1, Hkv, gs, cap, items));
    if (l.splits > 1) REQUIRE(int64_t(t.n_tokens) * Hkv <= kCounters);
    if (good) {                                          // every (pair, head) is some workgroup's, once
        const int64_t n = blocks_of(l.pairs, Hkv);
        std::vector<int> got(size_t(n) , 0);
        for (int64_t i = 0; i < n; ++i) {
            int g = -1;
            const int64_t x = place_of(uint32_t(i), Hkv, &g);
            REQUIRE(g >= 0 && g < Hkv && x >= 0 && x * Hkv + g < n);
            got[size_t(x * Hkv + g)] += 1;
        }
        for (int v : got) REQUIRE(v == 1);
    }
    std::vector<Seq> seq;
    uint64_t W = 0;
    int mx = 0, T = 0;
    for (int b = 0; b < B; ++b) {
        seq.push_back(make_seq(t.start[b], t.start[b + 1], t.len[b], t.n_tokens, cap, window, gs));
        const Seq &s = seq.back();
        REQUIRE(s.start >= 0 && s.nq >= 0 && s.start + s.nq <= t.n_tokens);
        REQUIRE(s.lo >= 0 && s.lo % kChunkStep == 0 && s.len >= 0 && s.lo + int64_t(s.len) <= cap);
        W += uint64_t(s.tiles) * uint64_t(s.len);
        T += s.tiles;
        mx = mx > s.len ? mx : s.len;
    }
    const int chunk = l.splits == 1 ? 1 << 30 : chunk_length(W, T, mx, Hkv, l.target, l.splits, over_of(join_in_launch(B, t.n_tokens, gs), Hkv % 2 != 0),
                                                                  join_rows_of(join_in_launch(B, t.n_tokens, gs), t.n_tokens, gs, T));
    REQUIRE(chunk % kChunkStep == 0);
    std::vector<std::vector<int>> seen(t.n_tokens);
    for (auto &v : seen) v.assign(size_t(cap), 0);
    std::vector<int> done(t.n_tokens, 0);
    int64_t pairs = 0;
    bool wide = false;
    for (int b = 0; b < B; ++b) {
        const Seq &s = seq[b];
        const int n = chunks_of(s, chunk);
        REQUIRE(n <= l.splits);
        pairs += int64_t(s.tiles) * n;
        for (int c = 0; c < n; ++c)
            for (int tile = 0; tile < s.tiles; ++tile) {
                const Item it = make_item(s, tile, c, chunk, cap, window, gs);
                if (it.idle) continue;
                REQUIRE(it.rows >= 1 && it.rows <= (it.narrow ? kNarrowRows : kTileRows));
                REQUIRE(it.tok0 >= 0 && it.n_tok >= 1 && it.tok0 + it.n_tok <= t.n_tokens && it.rows == it.n_tok << gs);
                if (!it.narrow) wide = true;
                REQUIRE(it.chunk0 >= 0 && it.chunk0 <= it.chunk1 && it.chunk1 < n);
                REQUIRE(it.begin % 64 == 0 && it.begin >= 0 && it.end <= cap);
                for (int i = 0; i < it.n_tok; ++i) {
                    if (c == it.chunk0) done[it.tok0 + i] += 1;
                    const int64_t p = it.p0 + i;
                    for (int j = it.begin; j < it.end; ++j)
                        if (j <= p && j > p - int64_t(window)) seen[it.tok0 + i][j] += 1;
                }
            }
    }
    if (!good) return;
    REQUIRE(pairs <= l.pairs && T <= l.tiles);
    if (join_in_launch(B, t.n_tokens, gs) && t.n_tokens == t.start[B]) REQUIRE(wide);
    for (int b = 0; b < B; ++b)
        for (int i = t.start[b]; i < t.start[b + 1]; ++i) {
            REQUIRE(done[i] == 1);
            const int64_t p = int64_t(t.len[b]) - t.start[b + 1] + i;
            for (int64_t j = 0; j < cap; ++j) REQUIRE(seen[i][j] == (j <= p && j > p - int64_t(window) ? 1 : 0));
        }
}

int main() {
    std::mt19937 r(7);
    auto in = [&](int a, int b) { return int(r() % unsigned(b - a + 1)) + a; };
    for (int trial = 0; trial < 3000; ++trial) {
        const int B = in(1, 7), gs = in(0, 3), Hkv = in(1, 9), shift = in(4, 7), max_pages = in(1, 1 + (3000 >> shift));
        const int64_t cap = int64_t(max_pages) << shift;
        const int window = in(0, 2) ? 0x7fffffff : in(1, int(cap) + 5);
        Tables t;
        t.start = {0};
        for (int b = 0; b < B; ++b) {
            const int len = in(0, 9) ? in(0, int(cap)) : in(0, 2), kind = in(0, 3);
            const int q = kind == 0 ? 1 : kind == 1 ? in(0, 5) : kind == 2 ? in(0, 150) : len + in(0, 1) * 3;
            t.len.push_back(len);
            t.start.push_back(t.start.back() + (q < 300 ? q : 300));
        }
        t.n_tokens = t.start.back() + in(0, 3);
        walk(t, Hkv, gs, cap, window, in(0, 1) ? 2048 : in(1, 64), true);
        // tables that cannot be: no access outside, whatever else
        for (auto &x : t.start) x = in(0, 4) ? x : in(0, 1) ? int(r()) : -x - 1;
        for (auto &x : t.len) x = in(0, 3) ? x : int(r());
        walk(t, Hkv, gs, cap, window, 2048, false);
        // rows of pages
        const int n_pages = in(1, 50);
        for (int i = 0; i < 20; ++i) {
            const int page = in(0, 3) ? in(-2, n_pages + 2) : int(r()), g = in(0, Hkv - 1), pos = in(0, int(cap) - 1);
            const int row = block_row(page, n_pages, Hkv, g, shift, pos);
            REQUIRE(row >= -1 && row < (n_pages * Hkv) << shift);
            REQUIRE((row >= 0) == (page >= 0 && page < n_pages));
        }
    }
    std::printf("all page checks passed\n");
    return 0;
}
