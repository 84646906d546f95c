// kv_pages.h -- the pages of the KV cache: who holds them, where new tokens go,
// and what is copied (the contract is in include/prefix_router.h, pr_kv).
//
// Decisions that depend on the order of a batch are taken by one workgroup (a
// batch is a few thousand entries and a cache's free bits a few KB to 128 KB, so
// a launch more would cost more than it saves); everything that moves keys and
// values, or touches a page per thread, is a grid.  Counts are changed by integer
// atomics only, whose result does not depend on their order.
#ifndef PR_KV_PAGES_H
#define PR_KV_PAGES_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kv_launch.h"
#include "kv_layout.h"
#include "wave_ops.h"

namespace pr {

using kv_u32x4 = __attribute__((ext_vector_type(4))) uint32_t;

constexpr int kKvPlanThreads = 1024;

// Sum of v over the threads before this one, the workgroup's sum in *all.
template <typename T>
__device__ inline T kv_block_before(T v, T *all) {
    __shared__ T part[kKvPlanThreads / 64];
    const int lane = (int)(threadIdx.x & 63), wave = (int)(threadIdx.x >> 6);
    T upto = v;
    for (int s = 1; s < 64; s <<= 1) {
        const T o = __shfl_up(upto, s);
        if (lane >= s) upto += o;
    }
    __syncthreads();
    if (lane == 63) part[wave] = upto;
    __syncthreads();
    T before = 0, sum = 0;
    for (int i = 0; i < kKvPlanThreads / 64; ++i) {
        if (i < wave) before += part[i];
        sum += part[i];
    }
    *all = sum;
    return before + upto - v;
}

__global__ void __launch_bounds__(256) kv_init_kernel(KvView c) {
    const int64_t step = (int64_t)gridDim.x * 256, first = (int64_t)blockIdx.x * 256 + threadIdx.x;
    for (int64_t i = first; i < (int64_t)c.num_slots * c.slot_pages; i += step) c.table[i] = -1;
    for (int64_t i = first; i < c.num_slots; i += step) c.lengths[i] = 0;
    for (int64_t i = first; i < c.num_pages; i += step) c.refs[i] = 0;
    for (int64_t i = first; i < ((int64_t)c.num_pages + 63) / 64; i += step) {
        const int64_t left = c.num_pages - 64 * i;
        c.free_pages[i] = left >= 64 ? ~0ull : (1ull << left) - 1;
    }
    if (first == 0) *c.skipped = 0;
}

// What kv_extend_plan_kernel decides about an entry.
struct KvGrant {
    int32_t start;   // tokens the sequence held
    int32_t source;  // the shared page it copies (its first new page takes its place), or -1
    int32_t slot;    // -1: skipped
};

struct KvExtend {
    KvView c;
    const int32_t *slots;
    const int64_t *offsets;
    int64_t n, rows;
    int32_t *place;
    int32_t *owner;   // [num_slots]: the first entry that appends to the slot
    KvGrant *grant;   // [n]
    int32_t *rank;    // [n]: pages that the entries before it ask for
    int32_t *fresh;   // the call's new pages
    int32_t *copies;  // entries that copy a page
    int32_t *count;   // new pages, copies
    int64_t most;     // pages the call can need (capacity of fresh)
};

// The free bits of a word that are pages.
__device__ __forceinline__ unsigned long long kv_free_word(const KvView &c, int32_t w) {
    const int32_t in = c.num_pages - 64 * w;
    return c.free_pages[w] & (in >= 64 ? ~0ull : (1ull << in) - 1);
}

// Tokens entry i appends, -1 if it is out of order or out of range.
__device__ __forceinline__ int64_t kv_appended(const KvExtend &x, int64_t i) {
    const int64_t a = x.offsets[i], b = x.offsets[i + 1];
    return a < 0 || b < a || b > x.rows ? -1 : b - a;
}

__global__ void __launch_bounds__(kKvPlanThreads) kv_extend_plan_kernel(KvExtend x) {
    const KvView &c = x.c;
    const int tid = (int)threadIdx.x;
    __shared__ int32_t copies, skipped, granted;
    if (tid == 0) copies = skipped = granted = 0;
    // a slot's first entry
    for (int64_t i = tid; i < x.n; i += kKvPlanThreads)
        if (kv_slot_ok(c, x.slots[i]) && kv_appended(x, i) > 0) x.owner[x.slots[i]] = INT32_MAX;
    __syncthreads();
    for (int64_t i = tid; i < x.n; i += kKvPlanThreads)
        if (kv_slot_ok(c, x.slots[i]) && kv_appended(x, i) > 0) atomicMin(&x.owner[x.slots[i]], (int32_t)i);
    // free pages
    const int32_t words = (c.num_pages + 63) / 64;
    int32_t mine = 0, available = 0;
    for (int32_t w = tid; w < words; w += kKvPlanThreads) mine += (int32_t)__popcll(kv_free_word(c, w));
    kv_block_before(mine, &available);
    if (available > x.most) available = (int32_t)x.most;
    // pages each entry needs, in the order of the batch: the first that finds too few
    // left is refused, and with it every later one that needs a page
    int64_t upto = 0;
    for (int64_t i0 = 0; i0 < x.n; i0 += kKvPlanThreads) {
        const int64_t i = i0 + tid;
        KvGrant g{0, -1, -1};
        int64_t need = 0, add = 0;
        int32_t slot = -1;
        if (i < x.n) {
            slot = x.slots[i];
            add = kv_appended(x, i);
            if (kv_slot_ok(c, slot) && add >= 0 &&
                (add == 0 || __hip_atomic_load(&x.owner[slot], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == i)) {
                g.start = kv_length(c, slot);
                if (g.start + add <= (int64_t)c.slot_pages << c.page_shift) {
                    g.slot = slot;
                    const int32_t old = kv_pages(c, g.start);
                    if (add > 0 && (g.start & (kv_page_tokens(c) - 1))) {
                        const int32_t last = c.table[(int64_t)slot * c.slot_pages + old - 1];
                        if (!kv_page_ok(c, last)) g.slot = -1;  // nothing to append to
                        else if (c.refs[last] > 1) g.source = last;
                    }
                    if (g.slot >= 0) need = kv_pages(c, g.start + add) - old + (g.source >= 0);
                }
            }
        }
        int64_t asked = 0;
        const int64_t before = upto + kv_block_before(need, &asked);
        upto += asked;
        if (need > 0) {
            if (before + need > available) g.slot = g.source = -1;
            else atomicMax(&granted, (int32_t)(before + need));
        }
        if (i < x.n) {
            if (g.slot < 0 && slot != -1) atomicAdd(&skipped, 1);
            x.grant[i] = g;
            x.rank[i] = (int32_t)(before < INT32_MAX ? before : INT32_MAX);
            if (g.source >= 0) x.copies[atomicAdd(&copies, 1)] = (int32_t)i;
            if (g.slot >= 0 && add > 0) c.lengths[g.slot] = g.start + (int32_t)add;
        }
    }
    __syncthreads();
    // the lowest free pages
    int32_t seen = 0;
    for (int32_t w0 = 0; w0 < words && seen < granted; w0 += kKvPlanThreads) {
        const int32_t w = w0 + tid;
        const unsigned long long bits = w < words ? kv_free_word(c, w) : 0;
        int32_t all = 0;
        int32_t r = seen + kv_block_before((int32_t)__popcll(bits), &all);
        unsigned long long left = bits;
        for (; left && r < granted; ++r) {
            const int32_t p = 64 * w + __builtin_ctzll(left);
            left &= left - 1;
            x.fresh[r] = p;
            c.refs[p] = 1;
        }
        if (left != bits) c.free_pages[w] = left;
        seen += all;
    }
    __syncthreads();
    // copied pages have one holder less; the last one's leaving frees them
    for (int32_t k = tid; k < copies; k += kKvPlanThreads) {
        const int32_t p = x.grant[x.copies[k]].source;
        if (atomicSub(&c.refs[p], 1) == 1) atomicOr(&c.free_pages[p >> 6], 1ull << (p & 63));
    }
    if (tid == 0) {
        x.count[0] = granted;
        x.count[1] = copies;
        if (skipped) atomicAdd(c.skipped, (unsigned long long)skipped);
    }
}

// Copies the first `tokens` tokens of page src to page dst, one (layer, head) of
// keys or values, by one wave.
template <typename T>
__device__ inline void kv_copy_tokens(const T *src, T *dst, bool keys, int32_t tokens, const KvView &c) {
    using V8 = __attribute__((ext_vector_type(8))) T;
    using V4 = __attribute__((ext_vector_type(4))) T;
    const int32_t lane = (int32_t)(threadIdx.x & 63);
    if (keys) {
        const int32_t units = c.head_dim / 8 * tokens;
        for (int32_t u = lane; u < units; u += 64) {
            const int32_t at = kv_key_at(c, u % tokens, u / tokens * 8);
            *(V8 *)(dst + at) = *(const V8 *)(src + at);
        }
    } else {
        const int32_t units = (tokens + 3) / 4 * c.head_dim;
        for (int32_t u = lane; u < units; u += 64) {
            const int32_t left = tokens - u / c.head_dim * 4;
            if (left >= 4) {
                *(V4 *)(dst + 4 * u) = *(const V4 *)(src + 4 * u);
            } else {
                for (int32_t e = 0; e < left; ++e) dst[4 * u + e] = src[4 * u + e];
            }
        }
    }
}

// The pages into the tables, each row's place, and the copies.
template <typename T>
__global__ void __launch_bounds__(256) kv_extend_place_kernel(KvExtend x) {
    const KvView &c = x.c;
    const int32_t pages = x.count[0], copies = x.count[1];
    const int64_t step = (int64_t)gridDim.x * 256, first = (int64_t)blockIdx.x * 256 + threadIdx.x;
    for (int64_t r = first; r < pages; r += step) {
        int64_t lo = 0, hi = x.n;  // the last entry with rank[lo] <= r
        while (hi - lo > 1) {
            const int64_t mid = (lo + hi) >> 1;
            if (x.rank[mid] <= r) lo = mid;
            else hi = mid;
        }
        const KvGrant g = x.grant[lo];
        const int32_t at = kv_pages(c, g.start) - (g.source >= 0) + (int32_t)(r - x.rank[lo]);
        if (g.slot >= 0 && (uint32_t)at < (uint32_t)c.slot_pages) c.table[(int64_t)g.slot * c.slot_pages + at] = x.fresh[r];
    }
    for (int64_t r = first; r < x.rows; r += step) {
        if (x.n == 0) {
            x.place[r] = -1;
            continue;
        }
        int64_t lo = 0, hi = x.n;
        if (x.rows == x.n && x.offsets[r] == r && x.offsets[r + 1] == r + 1) {
            lo = r;  // a token each
        } else {
            while (hi - lo > 1) {  // the last entry that begins at or before r
                const int64_t mid = (lo + hi) >> 1;
                if (x.offsets[mid] <= r) lo = mid;
                else hi = mid;
            }
        }
        int32_t to = -1;
        const KvGrant g = x.grant[lo];
        const int64_t a = x.offsets[lo];
        if (g.slot >= 0 && r >= a && r < x.offsets[lo + 1]) {
            const int64_t pos = g.start + (r - a);
            const int32_t col = (int32_t)(pos >> c.page_shift), old = kv_pages(c, g.start) - (g.source >= 0);
            const int32_t page = col >= old ? x.fresh[x.rank[lo] + col - old] : c.table[(int64_t)g.slot * c.slot_pages + col];
            if (kv_page_ok(c, page)) to = (page << c.page_shift) + (int32_t)(pos & (kv_page_tokens(c) - 1));
        }
        x.place[r] = to;
    }
    const int64_t items = (int64_t)copies * c.layers * c.kv_heads * 2;
    for (int64_t it = first >> 6; it < items; it += step >> 6) {
        const bool keys = it & 1;
        int64_t y = it >> 1;
        const int32_t head = (int32_t)(y % c.kv_heads);
        y /= c.kv_heads;
        const int32_t layer = (int32_t)(y % c.layers), i = x.copies[y / c.layers];
        const KvGrant g = x.grant[i];
        const int64_t at = layer * (keys ? c.k_layer : c.v_layer) + kv_head_base(c, head);
        T *pool = (T *)(keys ? c.k : c.v) + at;
        const int64_t page = keys ? c.k_page : c.v_page;
        kv_copy_tokens<T>(pool + g.source * page, pool + x.fresh[x.rank[i]] * page, keys,
                          g.start & (kv_page_tokens(c) - 1), c);
    }
}

// ---- rows ------------------------------------------------------------------------
struct KvRows {
    KvView c;
    const int32_t *place;
    const void *k, *v;
    int64_t k_stride, v_stride, rows, layer;
    bool aligned;  // rows may be read 16 bytes at a time
};

// Conversion of eight 16-bit numbers of a row to what the cache holds.
struct KvSame {
    using T = uint16_t;
    __device__ static void put(const uint16_t *in, float, T *out) {
        for (int i = 0; i < 8; ++i) out[i] = in[i];
    }
};
// Nearest e4m3 of number / scale.  The conversion instruction rounds to nearest,
// ties to even; what lies past the range is held at its end first, NaN kept.
template <bool BF16>
struct KvE4m3 {
    using T = uint8_t;
    __device__ static float one(uint16_t b, float scale) {
        float x;
        if (BF16) x = __uint_as_float((uint32_t)b << 16);
        else x = (float)__builtin_bit_cast(_Float16, b);
        x = x / scale;
        return x > 448.f ? 448.f : (x < -448.f ? -448.f : x);
    }
    __device__ static void put(const uint16_t *in, float scale, T *out) {
        for (int i = 0; i < 8; i += 4) {
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(one(in[i], scale), one(in[i + 1], scale), 0, false);
            w = __builtin_amdgcn_cvt_pk_fp8_f32(one(in[i + 2], scale), one(in[i + 3], scale), w, true);
            for (int e = 0; e < 4; ++e) out[i + e] = (uint8_t)((uint32_t)w >> (8 * e));
        }
    }
};

__device__ __forceinline__ void kv_load8(const uint16_t *src, bool aligned, uint16_t *out) {
    if (aligned) {
        const kv_u32x4 x = *(const kv_u32x4 *)src;
        for (int e = 0; e < 4; ++e) {
            out[2 * e] = (uint16_t)x[e];
            out[2 * e + 1] = (uint16_t)(x[e] >> 16);
        }
    } else {
        for (int e = 0; e < 8; ++e) out[e] = src[e];
    }
}

// Place of a row if it is one, else -1.
__device__ __forceinline__ int32_t kv_place(const KvRows &x, int64_t r) {
    if (r < 0 || r >= x.rows) return -1;
    const int32_t p = x.place[r];
    return p >= 0 && (p >> x.c.page_shift) < x.c.num_pages ? p : -1;
}

// A thread takes eight dimensions of a row: its key is 8 contiguous numbers; its
// value's numbers lie 4 tokens apart, so the thread of a block's first token
// writes all four of them where the batch has them in a row (prompts), and single
// numbers otherwise (a decode step).  Four rows' threads lie side by side, so that
// the keys of four tokens are written together.
template <typename P>
__device__ inline void kv_write_eight(const KvRows &x, int64_t r, int32_t dim) {
    using T = typename P::T;
    using V8 = __attribute__((ext_vector_type(8))) T;
    const KvView &c = x.c;
    const int32_t p = kv_place(x, r);
    if (p < 0) return;
    const int32_t head = dim / c.head_dim, d = dim % c.head_dim, t = p & (kv_page_tokens(c) - 1);
    const int64_t page = p >> c.page_shift;
    uint16_t in[8];
    union {
        T e[8];
        V8 v;
    } k;
    kv_load8((const uint16_t *)x.k + r * x.k_stride + dim, x.aligned, in);
    P::put(in, c.k_scale, k.e);
    *(V8 *)((T *)c.k + x.layer * c.k_layer + page * c.k_page + kv_head_base(c, head) + kv_key_at(c, t, d)) = k.v;

    const int64_t lead = r - (p & 3);
    const int32_t q = p & ~3;
    T *dst = (T *)c.v + x.layer * c.v_layer + page * c.v_page + kv_head_base(c, head) + kv_value_at(c, t & ~3, d);
    bool whole = true;
    for (int e = 0; e < 4; ++e) whole &= kv_place(x, lead + e) == q + e;
    if (whole) {
        if (p != q) return;
        union {
            T e[32];
            V8 v[4];
        } b;
        for (int e = 0; e < 4; ++e) {
            T one[8];
            kv_load8((const uint16_t *)x.v + (r + e) * x.v_stride + dim, x.aligned, in);
            P::put(in, c.v_scale, one);
            for (int i = 0; i < 8; ++i) b.e[4 * i + e] = one[i];
        }
        for (int i = 0; i < 4; ++i) *(V8 *)(dst + 8 * i) = b.v[i];
    } else {
        T one[8];
        kv_load8((const uint16_t *)x.v + r * x.v_stride + dim, x.aligned, in);
        P::put(in, c.v_scale, one);
        for (int i = 0; i < 8; ++i) dst[4 * i + (p & 3)] = one[i];
    }
}

template <typename P>
__global__ void __launch_bounds__(256) kv_write_kernel(KvRows x) {
    const int32_t eights = x.c.kv_heads * x.c.head_dim / 8;
    const int64_t items = (x.rows + 3) / 4 * 4 * eights;
    for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < items; id += (int64_t)gridDim.x * 256)
        kv_write_eight<P>(x, id / (4 * eights) * 4 + (id & 3), (int32_t)(id % (4 * eights) >> 2) * 8);
}

// ---- forks and trims: a workgroup an entry -----------------------------------------
__global__ void __launch_bounds__(256) kv_fork_kernel(KvView c, const int32_t *src, const int32_t *dst,
                                                      const int32_t *tokens, int64_t n) {
    const int64_t i = blockIdx.x;
    const int32_t from = src[i], to = dst[i], keep = tokens[i];
    if (to == -1) return;
    __shared__ int32_t clash;
    if (threadIdx.x == 0) clash = 0;
    __syncthreads();
    for (int64_t k = threadIdx.x; k < n; k += 256)
        if (dst[k] == from || (k < i && dst[k] == to)) clash = 1;
    __syncthreads();
    // lengths[to] is read before this workgroup, the only one that may, writes it
    const bool bad = clash || !kv_slot_ok(c, from) || !kv_slot_ok(c, to) || keep < 0 || keep > kv_length(c, from) ||
                     c.lengths[to] != 0;
    __syncthreads();
    if (bad) {
        if (threadIdx.x == 0) atomicAdd(c.skipped, 1ull);
        return;
    }
    const int32_t pages = kv_pages(c, keep);
    for (int32_t k = (int32_t)threadIdx.x; k < pages; k += 256) {
        const int32_t p = c.table[(int64_t)from * c.slot_pages + k];
        c.table[(int64_t)to * c.slot_pages + k] = p;
        if (kv_page_ok(c, p)) atomicAdd(&c.refs[p], 1);
    }
    if (threadIdx.x == 0) c.lengths[to] = keep;
}

__global__ void __launch_bounds__(256) kv_trim_kernel(KvView c, const int32_t *slots, const int32_t *keep,
                                                      int64_t keep_stride) {
    const int64_t i = blockIdx.x;
    const int32_t slot = slots[i], to = keep ? keep[i * keep_stride] : 0;
    if (slot == -1) return;
    if (!kv_slot_ok(c, slot) || to < 0) {
        if (threadIdx.x == 0) atomicAdd(c.skipped, 1ull);
        return;
    }
    // of the entries that name a slot each frees what its own minimum cuts off
    __shared__ int32_t had;
    if (threadIdx.x == 0) had = atomicMin(&c.lengths[slot], to);
    __syncthreads();
    const int32_t room = c.slot_pages << c.page_shift, was = min(had, room);
    if (was <= to) return;
    const int32_t last = kv_pages(c, was);
    for (int32_t k = kv_pages(c, to) + (int32_t)threadIdx.x; k < last; k += 256) {
        int32_t *at = &c.table[(int64_t)slot * c.slot_pages + k];
        const int32_t p = *at;
        *at = -1;
        if (kv_page_ok(c, p) && atomicSub(&c.refs[p], 1) == 1) atomicOr(&c.free_pages[p >> 6], 1ull << (p & 63));
    }
}

// ---- compaction -----------------------------------------------------------------------
struct KvCompact {
    KvView c;
    int32_t *moved;           // or nullptr
    int32_t *from, *target;   // [num_pages / 2]: pages that move and where to
    int32_t *to;              // [num_pages]: a moving page's new id
    int32_t *count;           // pages that move, pages held
};

__global__ void __launch_bounds__(kKvPlanThreads) kv_compact_plan_kernel(KvCompact x) {
    const KvView &c = x.c;
    const int tid = (int)threadIdx.x;
    const int32_t words = (c.num_pages + 63) / 64;
    int32_t mine = 0, unheld = 0;
    for (int32_t w = tid; w < words; w += kKvPlanThreads) mine += (int32_t)__popcll(kv_free_word(c, w));
    kv_block_before(mine, &unheld);
    const int32_t held = c.num_pages - unheld;
    int32_t holes = 0, movers = 0;
    for (int32_t w0 = 0; w0 < words; w0 += kKvPlanThreads) {
        const int32_t w = w0 + tid, page = 64 * w;
        unsigned long long hole = 0, move = 0;
        if (w < words) {
            const int32_t in = c.num_pages - page, low = held - page;  // pages of the word, and below `held`
            const unsigned long long valid = in >= 64 ? ~0ull : (1ull << in) - 1;
            const unsigned long long below = low >= 64 ? ~0ull : (low > 0 ? (1ull << low) - 1 : 0);
            const unsigned long long bits = kv_free_word(c, w);
            hole = bits & below;
            move = ~bits & valid & ~below;
        }
        int32_t all = 0;
        int32_t r = holes + kv_block_before((int32_t)__popcll(hole), &all);
        holes += all;
        for (; hole; hole &= hole - 1) x.target[r++] = page + __builtin_ctzll(hole);
        r = movers + kv_block_before((int32_t)__popcll(move), &all);
        movers += all;
        for (; move; move &= move - 1) x.from[r++] = page + __builtin_ctzll(move);
    }
    __syncthreads();
    const int32_t n = min(holes, movers);  // equal, unless the free bits are not the counts'
    for (int32_t k = tid; k < n; k += kKvPlanThreads) {
        const int32_t p = x.from[k], q = x.target[k];
        x.to[p] = q;
        c.refs[q] = c.refs[p];
        c.refs[p] = 0;
    }
    for (int32_t w = tid; w < words; w += kKvPlanThreads) {
        const int32_t page = 64 * w, in = c.num_pages - page, low = held - page;
        const unsigned long long valid = in >= 64 ? ~0ull : (1ull << in) - 1;
        c.free_pages[w] = valid & ~(low >= 64 ? ~0ull : (low > 0 ? (1ull << low) - 1 : 0));
    }
    if (tid == 0) {
        x.count[0] = n;
        x.count[1] = held;
        if (x.moved) {
            x.moved[0] = n;
            x.moved[1] = held;
        }
    }
}

// The moving pages' numbers, one (page, layer, keys or values) a workgroup at a
// time, and the tables.
__global__ void __launch_bounds__(256) kv_compact_move_kernel(KvCompact x, int32_t bytes) {
    const KvView &c = x.c;
    const int32_t n = x.count[0], held = x.count[1];
    if (n == 0) return;
    const int64_t step = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)c.num_slots * c.slot_pages; i += step) {
        const int32_t p = c.table[i];
        if (p >= held && kv_page_ok(c, p)) c.table[i] = x.to[p];
    }
    const int64_t items = (int64_t)n * c.layers * 2;
    const int32_t units = (int32_t)(((int64_t)c.kv_heads * c.head_dim << c.page_shift) * bytes / 16);
    for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
        const bool keys = it & 1;
        const int64_t y = it >> 1;
        const int32_t layer = (int32_t)(y % c.layers), k = (int32_t)(y / c.layers);
        char *pool = (char *)(keys ? c.k : c.v) + layer * (keys ? c.k_layer : c.v_layer) * bytes;
        const int64_t page = (keys ? c.k_page : c.v_page) * bytes;
        const kv_u32x4 *src = (const kv_u32x4 *)(pool + x.from[k] * page);
        kv_u32x4 *dst = (kv_u32x4 *)(pool + x.target[k] * page);
        for (int32_t u = (int32_t)threadIdx.x; u < units; u += 256) dst[u] = src[u];
    }
}

// ---- attention's split of large batches --------------------------------------------------
__global__ void __launch_bounds__(kKvPlanThreads) kv_plan_kernel(KvAttend a) {
    const int tid = (int)threadIdx.x;
    int64_t mine = 0, total = 0;  // blocks
    auto span = [&](int64_t i) {
        const int32_t s = a.slots[i];
        return kv_span(kv_slot_ok(a.c, s) ? kv_length(a.c, s) : 0, a.window);
    };
    for (int64_t i = tid; i < a.n; i += kKvPlanThreads) mine += kv_blocks(span(i));
    kv_block_before(mine, &total);
    const int32_t chunk = kv_chunk_tokens((int32_t)min(total, (int64_t)INT32_MAX / (kKvBlock / kKvStep)), a.split);
    int32_t before = 0;
    for (int64_t i0 = 0; i0 < a.n; i0 += kKvPlanThreads) {
        const int64_t i = i0 + tid;
        const int32_t cnt = i < a.n ? kv_chunks(span(i), chunk) : 0;
        int32_t all = 0;
        const int32_t at = before + kv_block_before(cnt, &all);
        if (i < a.n) a.plan[i] = at;
        before += all;
    }
    if (tid == 0) a.plan[a.n] = before;
}

}  // namespace pr

#endif
