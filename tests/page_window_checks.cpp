// Walks through the blocks of sekv_page_attend's items on the host (sekv_page_index.h): a block is looked up
// just where some row of the item sees one of its keys, and no page before a sequence's first visible key is.
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

static void walk(int len, int nq, int gs, int64_t cap, int window, int chunk, int page) {
    const Seq s = make_seq(0, nq, len, nq, cap, window, gs);
    const int64_t first = int64_t(len) - nq - (int64_t(window) - 1);
    for (int c = 0; c < chunks_of(s, chunk); ++c)
        for (int tile = 0; tile < s.tiles; ++tile) {
            const Item it = make_item(s, tile, c, chunk, cap, window, gs);
            if (it.idle) continue;
            for (int pos = it.begin; pos < int(cap) + 256; pos += kBlock) {
                bool any = false;                        // a key of the block, seen by a row of the item
                for (int i = 0; i < it.n_tok; ++i) {
                    const int64_t p = it.p0 + i, lo = p - (int64_t(window) - 1);
                    const int64_t from = lo > pos ? lo : pos, to = p < pos + kBlock - 1 ? p : pos + kBlock - 1;
                    any |= from <= to && from >= 0 && from < it.end;
                }
                REQUIRE(block_seen(it, pos) == any);
                if (block_seen(it, pos)) REQUIRE(pos / page >= (first < 0 ? 0 : first / page));
            }
        }
}

int main() {
    std::mt19937 rng(5);
    auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
    walk(200, 1, 2, 256, 100, 1 << 30, 16);              // first visible key 100, the item begins at 64
    for (int t = 0; t < 4000; ++t) {
        const int page = 16 << pick(0, 3), cap = page * pick(1, 40);
        const int len = pick(1, cap), nq = pick(1, t % 3 ? (len < 9 ? len : 9) : len), gs = pick(0, 3);
        const int window = t % 5 ? pick(1, len + 20) : 0x7fffffff;
        walk(len, nq, gs, cap, window, t % 2 ? 64 * pick(1, 8) : 1 << 30, page);
    }
    std::printf("all window checks passed\n");
    return 0;
}
