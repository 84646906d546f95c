// Walks, on the CPU, every address that the attention and the row writes of the KV
// cache form (kv_layout.h, as the kernels use it), for random lengths, windows,
// splits and tables with entries out of range: each lies inside its page's part of
// its head, every attended token is met once per dimension, and no token past a
// sequence's end or on a bad page counts.
#include <cstdio>
#include <cstdlib>
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

static void one(std::mt19937 &rng) {
    auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
    const int dims[] = {64, 96, 128, 192, 256};
    KvView c{};
    c.head_dim = dims[pick(0, 4)];
    c.kv_heads = pick(1, 3);
    c.page_shift = pick(4, 8);
    c.num_pages = pick(1, 40);
    c.num_slots = 1;
    c.slot_pages = pick(1, 12);
    const int T = kv_page_tokens(c), D = c.head_dim, room = c.slot_pages * T;
    std::vector<int32_t> table(c.slot_pages), length(1);
    for (auto &p : table) p = pick(0, 9) ? pick(0, c.num_pages - 1) : (pick(0, 1) ? -1 : pick(c.num_pages, 1 << 30));
    length[0] = pick(0, 3) ? pick(0, room) : room;
    if (pick(0, 20) == 0) length[0] = pick(0, 1) ? -7 : 2 * room + 3;  // held within the table's row
    c.table = table.data();
    c.lengths = length.data();
    const int n = kv_length(c, 0), window = pick(0, 2) ? 0 : pick(1, room + 9);
    CHECK(n >= 0 && n <= room);
    const int begin = kv_first(n, window), span = kv_span(n, window);
    KvSplit s{pick(1, 64), 0, pick(1, 2) * 256, pick(1, 8) * 256};
    s.most = s.fill * pick(1, 4);
    const int chunks = kv_chunks(span, kv_chunk_tokens((pick(0, 1) ? 1 : 64) * kv_blocks(span), s));
    const int chunk = kv_even_chunk(span, chunks), head = pick(0, c.kv_heads - 1);
    CHECK(chunk % kKvStep == 0);
    std::vector<int> keys((size_t)n * D), values((size_t)n * D), counted(n);
    const int part = D * T;  // elements of a head in a page
    for (int k = 0; k < chunks; ++k) {
        const int from = (begin & ~(kKvTile - 1)) + k * chunk;
        const int to = (int)std::min<int64_t>(n, (int64_t)from + chunk);
        for (int wave = 0; wave < kKvWaves; ++wave)
            for (int t = from + kKvTile * wave; t < to; t += kKvStep)
                for (int h = 0; h < 2; ++h) {
                    const int tok = t + 16 * h;
                    if (tok < to) CHECK((tok >> c.page_shift) < c.slot_pages);  // the table entry that is read
                    const int pg = tok < to ? table[tok >> c.page_shift] : -1;
                    const bool good = kv_page_ok(c, pg);
                    for (int lane = 0; lane < 64; ++lane) {
                        const int col = lane & 15, g = lane >> 4;
                        for (int j = 0; j < D / 32; ++j) {
                            const int ka = kv_key_at(c, (tok & (T - 1)) + col, 8 * g) + (32 * j << c.page_shift);
                            CHECK(ka >= 0 && ka + 8 <= part && ka == kv_key_at(c, (tok & (T - 1)) + col, 32 * j + 8 * g));
                            const int va = kv_value_at(c, (tok & (T - 1)) + 4 * g, 2 * col) + 128 * j;
                            CHECK(va >= 0 && va + 8 <= part);
                            for (int e = 0; e < 2; ++e)
                                for (int i = 0; i < 4; ++i) {
                                    CHECK(va + 4 * e + i == kv_value_at(c, (tok & (T - 1)) + 4 * g + i, 32 * j + 2 * col + e));
                                    const int u = tok + 4 * g + i;
                                    if (good && u >= begin && u < to) values[(size_t)u * D + 32 * j + 2 * col + e]++;
                                }
                            const int u = tok + col;
                            if (good && u >= begin && u < to)
                                for (int e = 0; e < 8; ++e) keys[(size_t)u * D + 32 * j + 8 * g + e]++;
                        }
                        if (lane % 16 == 0)
                            for (int i = 0; i < 4; ++i) {
                                const int u = tok + 4 * g + i;
                                if (good && u >= begin && u < to) counted[u]++;
                            }
                    }
                }
    }
    CHECK(kv_head_base(c, head) + part <= (int64_t)c.kv_heads * part);
    for (int t = 0; t < n; ++t) {
        const int want = t >= begin && kv_page_ok(c, table[t >> c.page_shift]);
        CHECK(counted[t] == want);
        for (int d = 0; d < D; ++d) CHECK(keys[(size_t)t * D + d] == want && values[(size_t)t * D + d] == want);
    }
    // a row's parts
    for (int t = 0; t < T; ++t)
        for (int d = 0; d < D; d += 8) {
            CHECK(kv_key_at(c, t, d) % 8 == 0 && kv_key_at(c, t, d) + 8 <= part);
            CHECK(kv_value_at(c, t & ~3, d) % 16 == 0 && kv_value_at(c, t & ~3, d) + 32 <= part);
            for (int i = 0; i < 8; ++i) CHECK(kv_value_at(c, t & ~3, d) + 4 * i + (t & 3) == kv_value_at(c, t, d + i));
        }
}

// The split never makes more chunks than a launch has room for.
static void split(std::mt19937 &rng) {
    auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
    const int n = pick(1, 60);
    KvSplit s{pick(1, 200), 0, 256, pick(1, 8) * 256};
    s.most = s.fill * pick(1, 4);
    std::vector<int> spans(n);
    int64_t units = 0;
    int32_t total = 0;
    for (auto &x : spans) total += kv_blocks(x = pick(0, 5) ? pick(0, 400) : pick(0, 200000));
    int chunk = kv_chunk_tokens(total, s);
    for (int tries = n < s.fill ? pick(0, 3) : 0; tries; --tries) {
        int64_t now = 0;
        for (int x : spans) now += kv_chunks(x, chunk);
        const int longer = kv_longer_chunk(chunk, (int)now, s.fill);
        CHECK(longer % kKvStep == 0 && longer >= kKvStep);
        if (now > s.fill) {
            CHECK(longer > chunk);
            chunk = longer;
        }
    }
    for (int x : spans) {
        const int k = kv_chunks(x, chunk), even = kv_even_chunk(x, k);
        CHECK(k == (x <= chunk ? 1 : (x + chunk - 1) / chunk));
        CHECK((int64_t)k * even >= x && (k == 1 || even <= chunk));
        CHECK(k <= std::max(1, (x + 255) / 256));
        units += k;
    }
    CHECK(units <= (int64_t)s.most + n);
}

int main() {
    std::mt19937 rng(7);
    for (int i = 0; i < 300; ++i) one(rng);
    for (int i = 0; i < 3000; ++i) split(rng);
    printf("kv_addresses: %s\n", failures ? "failed" : "ok");
    return failures != 0;
}
