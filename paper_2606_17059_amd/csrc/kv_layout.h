// kv_layout.h -- the paged KV cache as the kernels see it (the contract is in
// include/prefix_router.h, pr_kv): sizes, and where numbers lie.  Plain C++, so
// that the addresses can be walked on the CPU.
#ifndef PR_KV_LAYOUT_H
#define PR_KV_LAYOUT_H

#include <stdint.h>

#ifdef __HIPCC__
#define PR_KV_FN __host__ __device__ __forceinline__
#else
#define PR_KV_FN inline
#endif

namespace pr {

// A pr_kv without its host-side fields.
struct KvView {
    void *k, *v;
    int64_t k_layer, k_page, v_layer, v_page;  // elements
    int32_t *table, *lengths, *refs;
    unsigned long long *free_pages;
    unsigned long long *skipped;
    int32_t layers, kv_heads, head_dim, page_shift, num_pages, num_slots, slot_pages;
    float k_scale, v_scale;
};

PR_KV_FN int32_t kv_page_tokens(const KvView &c) { return 1 << c.page_shift; }
PR_KV_FN int32_t kv_pages(const KvView &c, int64_t tokens) {
    return (int32_t)((tokens + kv_page_tokens(c) - 1) >> c.page_shift);
}
PR_KV_FN bool kv_page_ok(const KvView &c, int32_t page) { return (uint32_t)page < (uint32_t)c.num_pages; }
PR_KV_FN bool kv_slot_ok(const KvView &c, int32_t slot) { return (uint32_t)slot < (uint32_t)c.num_slots; }

// Tokens a sequence holds, never more than its table row has room for.
PR_KV_FN int32_t kv_length(const KvView &c, int32_t slot) {
    const int32_t n = c.lengths[slot], most = c.slot_pages << c.page_shift;
    return n < 0 ? 0 : (n < most ? n : most);
}

// Element of a page's part for one head (head_dim * page_tokens elements from
// kv_head_base): keys lie in blocks of 8 dimensions, values in blocks of 4 tokens.
PR_KV_FN int32_t kv_key_at(const KvView &c, int32_t token, int32_t dim) {
    return (((dim >> 3) << c.page_shift) + token) * 8 + (dim & 7);
}
PR_KV_FN int32_t kv_value_at(const KvView &c, int32_t token, int32_t dim) {
    return ((token >> 2) * c.head_dim + dim) * 4 + (token & 3);
}
PR_KV_FN int64_t kv_head_base(const KvView &c, int32_t head) {
    return ((int64_t)head * c.head_dim) << c.page_shift;
}

// ---- how attention splits a batch ---------------------------------------------
constexpr int32_t kKvMostTokens = 1 << 30;  // of a sequence
constexpr int kKvTile = 32;        // tokens a wave takes at a time
constexpr int kKvWaves = 4;        // waves of a workgroup that takes a share of a batch
constexpr int kKvStep = kKvTile * kKvWaves;
constexpr int kKvWideWaves = 8;    // waves of a workgroup that takes a whole short sequence

// First token attended, rounded down to a tile, and the tiles' tokens from there.
PR_KV_FN int32_t kv_first(int32_t length, int32_t window) {
    return window > 0 && length > window ? length - window : 0;
}
PR_KV_FN int32_t kv_span(int32_t length, int32_t window) {
    return length - (kv_first(length, window) & ~(kKvTile - 1));
}

// Steps of a workgroup that a span takes (one where there is nothing: its output is
// written too).
PR_KV_FN uint32_t kv_steps(int32_t span) {
    return span <= 0 ? 1 : ((uint32_t)span + kKvStep - 1) / kKvStep;
}

// How a batch's steps, one sequence's after another's, are cut into equal shares: `fill`
// of them occupy the GPU once, and none is shorter than `least`.
struct KvSplit {
    uint32_t fill, least;
};
PR_KV_FN uint32_t kv_share(uint32_t steps, const KvSplit &s) {
    const uint32_t c = (steps + s.fill - 1) / s.fill;
    return c < s.least ? s.least : c;
}
// First step of share u, `steps` where there is none.  Shares from `fill` on have
// nothing, and their product may pass 32 bits.
PR_KV_FN uint32_t kv_share_begin(uint32_t u, uint32_t size, uint32_t steps, const KvSplit &s) {
    return u < s.fill ? u * size : steps;
}

// Whether shares keep to sequences instead: one for each, or equal ones of a sequence
// longer than a share.  So it is where there are more sequences than shares and they
// are short: a share of several would begin anew with each, where workgroups beside it
// could (600 sequences of 10 to 600 tokens on 4 key heads of 128: 82 us, 87 across;
// 128 of 4,096 to 16,384 on 8: 953 us, 904 across).
constexpr uint32_t kKvShort = 8;   // steps of a short sequence, on average
PR_KV_FN bool kv_keeps(uint32_t steps, int64_t n, const KvSplit &s) { return n >= s.fill && steps < n * kKvShort; }
PR_KV_FN uint32_t kv_even(uint32_t steps, uint32_t shares) { return (steps + shares - 1) / shares; }

// A share's part [from, to) of a sequence that has the steps [first, first + steps) of
// the batch, in steps of the sequence.
struct KvPart {
    uint32_t from, to;
    bool whole;  // the sequence has no other part
};
PR_KV_FN KvPart kv_part(uint32_t begin, uint32_t end, uint32_t first, uint32_t steps) {
    KvPart p;
    p.from = begin > first ? begin - first : 0;
    p.to = end < first + steps ? end - first : steps;
    p.whole = p.from == 0 && p.to == steps;
    return p;
}
// Where parts of sequences that have several are kept until they are joined.  A share has a
// number: its own where shares go on from sequence to sequence (it then has two such parts
// at most, one that begins its sequence and one that does not), else that among the shares of
// sequences that have several.  `fill` shares of `size` steps or more are all the steps, so
// of the latter there are less than 2 fill (a sequence with x > 1 times the steps of a share
// has less than x + 1 < 2 x).
PR_KV_FN uint32_t kv_part_at(uint32_t number, bool begins) { return 2 * number - !begins; }
// ... and part k of a sequence whose first one is kept at `first`.
PR_KV_FN uint32_t kv_part_next(uint32_t first, uint32_t k) { return first + (k ? 2 * k - 1 : 0); }
PR_KV_FN int64_t kv_parts_kept(int64_t n, int64_t units, const KvSplit &s) {
    const int64_t numbers = n < s.fill ? s.fill : 2 * (int64_t)s.fill;
    return 2 * (numbers < units ? numbers : units);
}

// Parts of a sequence, the first of which is in share `share`.
PR_KV_FN uint32_t kv_parts(uint32_t share, uint32_t c, uint32_t first, uint32_t steps) {
    return (first + steps - 1) / c - share + 1;
}

}  // namespace pr

#endif
