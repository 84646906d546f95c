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
constexpr int kKvWaves = 4;        // waves of a workgroup that takes a chunk
constexpr int kKvStep = kKvTile * kKvWaves;

// First token attended, rounded down to a tile, and the tiles' tokens from there.
PR_KV_FN int32_t kv_first(int32_t length, int32_t window) {
    return window > 0 && length > window ? length - window : 0;
}
PR_KV_FN int32_t kv_span(int32_t length, int32_t window) {
    return length - (kv_first(length, window) & ~(kKvTile - 1));
}

// A span in blocks: 256 sequences' blocks can be added in 32 bits.
constexpr int kKvBlock = 256;
PR_KV_FN int32_t kv_blocks(int32_t span) { return (span + kKvBlock - 1) / kKvBlock; }

// How a batch's tokens are cut: `fill` chunks occupy the GPU once; chunks longer
// than `worth` are cut further, into `most` of them, for the sake of an even end;
// no chunk is shorter than `least`.
struct KvSplit {
    int32_t fill, most, least, worth;
};

// Tokens a chunk has at most, in whole steps of a workgroup.
PR_KV_FN int32_t kv_chunk_tokens(int32_t blocks, const KvSplit &s) {
    const uint32_t steps = (uint32_t)blocks * (kKvBlock / kKvStep), worth = (uint32_t)(s.worth / kKvStep);
    uint32_t c = (steps + (uint32_t)s.fill - 1) / (uint32_t)s.fill;
    if (c > worth) {
        const uint32_t cut = (steps + (uint32_t)s.most - 1) / (uint32_t)s.most;
        c = cut > worth ? cut : worth;
    }
    if (c >= (uint32_t)kKvMostTokens / kKvStep) return kKvMostTokens;
    return (int32_t)(c * kKvStep) < s.least ? s.least : (int32_t)(c * kKvStep);
}
// The chunk that makes about `fill` units of what `units` of length c were.
PR_KV_FN int32_t kv_longer_chunk(int32_t c, int32_t units, int32_t fill) {
    const uint64_t x = (uint64_t)((uint32_t)c / kKvStep) * (uint32_t)units / (uint32_t)fill + 1;
    return x >= (uint64_t)kKvMostTokens / kKvStep ? kKvMostTokens : (int32_t)(x * kKvStep);
}

// Chunks of one sequence (one where it has no tokens: its output is written too).
PR_KV_FN int32_t kv_chunks(int32_t span, int32_t chunk) {
    return span <= chunk ? 1 : (int32_t)(((uint32_t)span + (uint32_t)chunk - 1) / (uint32_t)chunk);
}

// A sequence's chunks made even.
PR_KV_FN int32_t kv_even_chunk(int32_t span, int32_t chunks) {
    if (chunks <= 1) return kKvMostTokens;
    const uint32_t steps = ((uint32_t)span + kKvStep - 1) / kKvStep;
    return (int32_t)((steps + (uint32_t)chunks - 1) / (uint32_t)chunks * kKvStep);
}

}  // namespace pr

#endif
