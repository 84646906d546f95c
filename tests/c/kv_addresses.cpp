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
    const int head = pick(0, c.kv_heads - 1), waves = pick(0, 1) ? kKvWaves : 4 * kKvWaves;
    // the sequence somewhere in a batch, cut into shares
    const uint32_t steps = kv_steps(span), first = (uint32_t)pick(0, 50), size = (uint32_t)pick(1, 40);
    std::vector<int> keys((size_t)n * D), values((size_t)n * D), counted(n);
    const int part = D * T;  // elements of a head in a page
    for (uint32_t u = first / size; u * size < first + steps; ++u) {
        const KvPart kp = kv_part(u * size, (u + 1) * size, first, steps);
        const int from = (begin & ~(kKvTile - 1)) + (int)kp.from * kKvStep;
        const int to = kp.to == steps ? n : (begin & ~(kKvTile - 1)) + (int)kp.to * kKvStep;
        CHECK(kp.from < kp.to && kp.to <= steps && to <= n);
        for (int wave = 0; wave < waves; ++wave)
            for (int t = from + kKvTile * wave; t < to; t += kKvTile * waves)
                for (int h = 0; h < 2; ++h) {
                    const int tok = t + 16 * h;
                    // the table entry that is read: of a page of the row's, whatever the length
                    CHECK(tok >= room || (tok >> c.page_shift) < c.slot_pages);
                    const int pg = tok < room ? table[tok >> c.page_shift] : -1;
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

// The shares of a batch cover every sequence's steps once, are no more than a launch
// has, and number the parts of a sequence in a row that no other has.
static void split(std::mt19937 &rng) {
    auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
    const int n = pick(1, 60);
    const KvSplit s{(uint32_t)pick(1, 200), (uint32_t)pick(1, 2) * 2};
    const bool shorts = pick(0, 1);
    std::vector<int> spans(n);
    std::vector<uint32_t> first(n + 1, 0);
    uint32_t longest = 0;
    for (int i = 0; i < n; ++i) {
        spans[i] = shorts || pick(0, 5) ? pick(0, 400) : pick(0, 200000);
        first[i + 1] = first[i] + kv_steps(spans[i]);
        longest = std::max(longest, kv_steps(spans[i]));
    }
    const uint32_t c = kv_share(first[n], s);
    // what the host launches
    const int64_t units = std::min<int64_t>((int64_t)n * longest, s.fill + (n >= (int)s.fill ? n : 0));
    CHECK(c >= s.least);
    std::vector<uint32_t> covered(n), where(n), parts(n), seen(n);
    std::vector<int> used(units + n);
    if (kv_keeps(first[n], n, s)) {  // shares of each sequence's own
        int64_t u = 0;
        for (int i = 0; i < n; ++i) {
            const uint32_t steps = first[i + 1] - first[i], shares = (steps + c - 1) / c, even = kv_even(steps, shares);
            for (uint32_t k = 0; k < shares; ++k, ++u) {
                const uint32_t begin = k * even, end = std::min(begin + even, steps);
                CHECK(u < units && even <= c);
                if (begin >= end) continue;  // nothing is left: see the kernel's parts
                const KvPart p = kv_part(begin, end, 0, steps);
                CHECK(p.from == covered[i] && p.to <= steps && p.whole == (shares == 1));
                covered[i] = p.to;
                if (p.from == 0) {
                    where[i] = (uint32_t)u + i;
                    parts[i] = kv_parts(0, even, 0, steps);
                }
                CHECK((uint32_t)u + i == where[i] + seen[i]);
                seen[i]++;
                used[u + i]++;
            }
        }
    } else {
        for (int64_t u = 0; u < units; ++u) {
            const uint32_t begin = kv_share_begin((uint32_t)u, c, first[n], s), end = std::min(begin + c, first[n]);
            if (begin >= first[n]) continue;
            int i = 0;
            while (first[i + 1] <= begin) ++i;
            for (;; ++i) {
                CHECK(i < n);
                const uint32_t steps = first[i + 1] - first[i];
                const KvPart p = kv_part(begin, end, first[i], steps);
                CHECK(p.from == covered[i] && p.from < p.to && p.to <= steps && p.whole == (p.to - p.from == steps));
                covered[i] = p.to;
                if (p.from == 0) {
                    where[i] = (uint32_t)u + i;
                    parts[i] = kv_parts((uint32_t)u, c, first[i], steps);
                    CHECK((parts[i] == 1) == p.whole);
                }
                CHECK((uint32_t)u + i == where[i] + seen[i] && u + i < units + n);
                seen[i]++;
                used[u + i]++;
                if (first[i] + p.to >= end) break;
            }
        }
    }
    for (int i = 0; i < n; ++i) CHECK(covered[i] == first[i + 1] - first[i] && seen[i] == parts[i]);
    for (int x : used) CHECK(x <= 1);
}

// Shares of the most steps and the most workgroups that a batch may have: each step is
// in one share, though the last workgroups' products pass 32 bits.
static void many() {
    for (const uint32_t fill : {1u, 2u, 7u, 1280u})
        for (const uint32_t steps : {1u << 19, 1u << 27, (1u << 31) + 5})
            for (const uint32_t n : {1u, fill, 1u << 16, 1u << 23}) {
                const KvSplit s{fill, 4};
                const uint32_t c = kv_share(steps, s);
                uint32_t covered = 0;
                for (uint32_t u = 0; u < fill + n; ++u) {
                    const uint32_t begin = kv_share_begin(u, c, steps, s);
                    if (begin >= steps) continue;
                    CHECK(begin == covered && begin + c > begin);
                    covered = std::min(begin + c, steps);
                }
                CHECK(covered == steps);
            }
}

int main() {
    std::mt19937 rng(7);
    for (int i = 0; i < 300; ++i) one(rng);
    for (int i = 0; i < 3000; ++i) split(rng);
    many();
    printf("kv_addresses: %s\n", failures ? "failed" : "ok");
    return failures != 0;
}
