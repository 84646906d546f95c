// Walks, on the CPU, where the attention keeps the parts of sequences that several shares
// take (kv_layout.h, as the kernels number them), over random batches and splits: no two
// parts in one place, none past what the host gives room for, and a sequence's parts
// found again from its first one.
#include <algorithm>
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

static int kept[2], split_batches[2];

static void batch(std::mt19937 &rng) {
    auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
    const int n = pick(0, 3) ? pick(1, 40) : pick(1, 700);
    const KvSplit s{(uint32_t)(pick(0, 2) ? pick(1, 60) : pick(1, 1300)), (uint32_t)pick(1, 2) * 2};
    const int kind = pick(0, 3);
    std::vector<uint32_t> first(n + 1, 0);
    uint32_t longest = 0;
    for (int i = 0; i < n; ++i) {
        const int span = kind == 0 ? pick(0, 400) : kind == 1 ? pick(0, 3000) : pick(0, 30) ? pick(0, 500) : pick(0, 100000);
        first[i + 1] = first[i] + kv_steps(span);
        longest = std::max(longest, kv_steps(span));
    }
    const uint32_t total = first[n], size = kv_share(total, s);
    // what the host knows: the longest sequence there may be
    const int64_t room = (int64_t)longest + (pick(0, 1) ? pick(0, 200) : 0);
    const int64_t units = std::min<int64_t>(n * room, s.fill + (n >= (int)s.fill ? n : 0));
    const int64_t places = kv_parts_kept(n, units, s);
    std::vector<int> used(places);
    auto put = [&](uint32_t at) {
        CHECK((int64_t)at < places);
        if ((int64_t)at < places) CHECK(used[at]++ == 0);
    };
    const bool keeps = kv_keeps(total, n, s);
    if (keeps) {
        uint32_t u = 0, split = 0;
        for (int i = 0; i < n; ++i) {
            const uint32_t steps = first[i + 1] - first[i], shares = (steps + size - 1) / size;
            for (uint32_t k = 0; k < shares && shares > 1; ++k) {
                const uint32_t at = kv_part_at(split + k, k == 0);
                CHECK(at == kv_part_next(kv_part_at(split, true), k));
                put(at);
            }
            u += shares;
            if (shares > 1) split += shares;
        }
        CHECK(u <= units);
        split_batches[1] += split > 0;
    } else {
        std::vector<uint32_t> where(n), seen(n);
        bool some = false;
        for (uint32_t u = 0; u < units; ++u) {
            const uint32_t begin = kv_share_begin(u, size, total, s), end = std::min(begin + size, total);
            if (begin >= total) continue;
            int i = (int)(std::upper_bound(first.begin(), first.end(), begin) - first.begin()) - 1;
            for (;; ++i) {
                const uint32_t steps = first[i + 1] - first[i];
                const KvPart p = kv_part(begin, end, first[i], steps);
                if (!p.whole) {
                    const uint32_t at = kv_part_at(u, p.from == 0);
                    if (p.from == 0) where[i] = at;
                    CHECK(at == kv_part_next(where[i], seen[i]));
                    seen[i]++;
                    put(at);
                    some = true;
                }
                if (first[i] + p.to >= end) break;
            }
        }
        split_batches[0] += some;
    }
    kept[keeps]++;
}

int main() {
    std::mt19937 rng(5);
    for (int i = 0; i < 6000; ++i) batch(rng);
    CHECK(split_batches[0] > 500 && split_batches[1] > 100);
    printf("kv_kept: %s (%d and %d batches, %d and %d with parts)\n", failures ? "failed" : "ok", kept[0], kept[1],
           split_batches[0], split_batches[1]);
    return failures != 0;
}
