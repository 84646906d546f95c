// Walks, on the CPU, what a workgroup of the attention that takes a whole sequence reads
// and counts (kv_layout.h, as the kernel uses it): with the 8 waves of a short batch and
// with 4, over random lengths, windows and tables, and at the longest tables.  Every
// token attended is met by one wave, once; page ids come from the sequence's own table
// row, also those asked for ahead; keys and values lie inside their page's part.
#include <cstdint>
#include <cstdio>
#include <random>
#include <vector>

#include "kv_layout.h"

using namespace pr;

static int failures = 0;
#define CHECK(cond)                                                  \
    do {                                                             \
        if (!(cond)) {                                               \
            if (failures++ < 10) fprintf(stderr, "line %d: %s\n", __LINE__, #cond); \
        }                                                            \
    } while (0)

static void walk(const KvView &c, int window, int waves, std::vector<int> *counted) {
    const int T = kv_page_tokens(c), room = c.slot_pages * T, n = kv_length(c, 0);
    const int begin = window > 0 ? kv_first(n, window) : 0, tile0 = begin & ~(kKvTile - 1), step = kKvTile * waves;
    auto page_of = [&](int64_t tok) {
        CHECK(tok >= 0 && tok <= INT32_MAX);  // held in 32 bits
        const int at = (int)((tok < room - 1 ? tok : room - 1) >> c.page_shift);
        CHECK(at >= 0 && at < c.slot_pages);
        return c.table[at];
    };
    for (int wave = 0; wave < waves; ++wave) {
        int64_t t = tile0 + kKvTile * wave;
        for (int h = 0; h < 2; ++h) {
            page_of(t + 16 * h);
            page_of(t + step + 16 * h);
        }
        for (; t < n; t += step)
            for (int h = 0; h < 2; ++h) {
                const int tok = (int)t + 16 * h, inside = tok & (T - 1);
                page_of((int64_t)tok + 2 * step);
                const int32_t pg = page_of(tok);
                CHECK(inside + 16 <= T);  // half a tile lies in one page
                CHECK(kv_key_at(c, inside + 15, c.head_dim - 8) + 8 <= c.head_dim * T);
                CHECK(kv_value_at(c, inside + 12, c.head_dim - 1) + 4 <= c.head_dim * T);
                if (!counted || !kv_page_ok(c, pg)) continue;
                for (int i = 0; i < 16; ++i)
                    if (tok + i >= begin && tok + i < n) (*counted)[tok + i]++;
            }
    }
}

int main() {
    std::mt19937 rng(11);
    auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
    const int dims[] = {64, 96, 128, 192, 256};
    for (int i = 0; i < 2000; ++i) {
        KvView c{};
        c.head_dim = dims[pick(0, 4)];
        c.kv_heads = 1;
        c.page_shift = pick(4, 8);
        c.num_pages = pick(1, 90);
        c.num_slots = 1;
        c.slot_pages = pick(1, 80);
        const int room = c.slot_pages << c.page_shift;
        std::vector<int32_t> table(c.slot_pages);
        for (auto &p : table) p = pick(0, 9) ? pick(0, c.num_pages - 1) : (pick(0, 1) ? -1 : pick(c.num_pages, 1 << 30));
        int32_t length = pick(0, 3) ? pick(0, room) : room - pick(0, 1);
        if (pick(0, 20) == 0) length = pick(0, 1) ? -5 : room + 100;
        c.table = table.data();
        c.lengths = &length;
        const int n = kv_length(c, 0), window = pick(0, 2) ? 0 : pick(1, room + 9);
        const int begin = window > 0 ? kv_first(n, window) : 0;
        for (const int waves : {kKvWaves, kKvWideWaves}) {
            std::vector<int> counted(n);
            walk(c, window, waves, &counted);
            for (int t = 0; t < n; ++t) CHECK(counted[t] == (t >= begin && kv_page_ok(c, table[t >> c.page_shift])));
        }
    }
    // the longest table: nothing that is asked for ahead passes 32 bits
    for (int shift = 4; shift <= 8; shift += 4) {
        KvView c{};
        c.head_dim = 64;
        c.kv_heads = c.num_slots = c.num_pages = 1;
        c.page_shift = shift;
        c.slot_pages = kKvMostTokens >> shift;
        std::vector<int32_t> table(c.slot_pages, 0);
        int32_t length = kKvMostTokens;
        c.table = table.data();
        c.lengths = &length;
        for (const int waves : {kKvWaves, kKvWideWaves}) walk(c, 3000, waves, nullptr);
    }
    printf("kv_whole: %s\n", failures ? "failed" : "ok");
    return failures != 0;
}
