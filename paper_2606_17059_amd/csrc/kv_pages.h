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

// Sums that stop at 2^32 - 1: what is compared with a count of pages may be more
// than any cache has.
__device__ __forceinline__ uint32_t kv_add(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

// Sum of v over the threads before this one, the workgroup's sum in *all.
__device__ inline uint32_t kv_block_before(uint32_t v, uint32_t *all) {
    __shared__ uint32_t part[kKvPlanThreads / 64];
    const int lane = (int)(threadIdx.x & 63), wave = (int)(threadIdx.x >> 6);
    const uint32_t upto = lanes_upto(v, kv_add);
    __syncthreads();
    if (lane == 63) part[wave] = upto;
    __syncthreads();
    uint32_t before = 0, sum = 0;
#pragma unroll
    for (int i = 0; i < kKvPlanThreads / 64; ++i) {
        if (i == wave) before = sum;
        sum = kv_add(sum, part[i]);
    }
    *all = sum;
    return kv_add(before, upto - v);  // exact in the wave unless past everything
}

// Calls put(rank, page) for the set bits of the workgroup's words, a wave a word: `bits`
// is a thread's word, 64 * first the first thread's first page, `rank` the number of
// set bits in the words before its own.  All threads call it with the same number of
// `words` that may have bits.
template <typename Put>
__device__ inline void kv_each_bit(unsigned long long bits, int32_t first, uint32_t rank, int32_t words, Put put) {
    const int lane = (int)(threadIdx.x & 63), wave = uniform((int)(threadIdx.x >> 6));
    auto one = [&](uint64_t w, int k, uint32_t r) {
        if (w >> lane & 1) put(r + (uint32_t)__popcll(w & ((1ull << lane) - 1)), 64 * (first + k) + lane);
    };
    const uint64_t some = __ballot(bits != 0);
    if (words <= 64) {
        // a wave its own words: dealing them out costs 0.8 us, one wave's 64 words 3 us
        for (uint64_t m = some; m; m &= m - 1) {
            const int src = __builtin_ctzll(m);
            one(readlane64(bits, src), 64 * wave + src, (uint32_t)__builtin_amdgcn_readlane((int)rank, src));
        }
        return;
    }
    __shared__ unsigned long long word[kKvPlanThreads];
    __shared__ uint32_t before[kKvPlanThreads];
    __shared__ uint64_t any[kKvPlanThreads / 64];
    __syncthreads();  // the arrays are the last call's until here
    word[threadIdx.x] = bits;
    before[threadIdx.x] = rank;
    if (lane == 0) any[wave] = some;
    __syncthreads();
    for (int v = 0; v < kKvPlanThreads / 64; ++v) {
        // of the words of wave v this wave takes every sixteenth
        for (uint64_t m = any[v] & (0x0001000100010001ull << wave); m; m &= m - 1) {
            const int k = 64 * v + __builtin_ctzll(m);
            one(word[k], k, before[k]);
        }
    }
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

// Takes entries that were reported from the count.
__global__ void __launch_bounds__(1) kv_reported_kernel(unsigned long long *skipped, unsigned long long reported) {
    atomicAdd(skipped, 0 - reported);
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

// An entry of an extension: its slot (-1 if it is none), and the tokens it appends (-1
// if its offsets are out of order or out of range).
struct KvEntry {
    int32_t slot;
    int64_t add;
};
__device__ __forceinline__ KvEntry kv_entry(const KvExtend &x, int64_t i) {
    if (i >= x.n) return KvEntry{-1, 0};
    const int64_t a = x.offsets[i], b = x.offsets[i + 1];
    return KvEntry{x.slots[i], a < 0 || b < a || b > x.rows ? -1 : b - a};
}

// What an entry's sequence holds: its tokens, its last page if that is partly filled
// (-1: no such page), and who holds that.
struct KvTail {
    int32_t start, last, holders;
};
__device__ __forceinline__ KvTail kv_tail(const KvView &c, const KvEntry &e) {
    KvTail t{0, -1, 0};
    if (!kv_slot_ok(c, e.slot) || e.add <= 0) return t;
    t.start = kv_length(c, e.slot);
    if (t.start & (kv_page_tokens(c) - 1)) t.last = c.table[(int64_t)e.slot * c.slot_pages + (t.start >> c.page_shift)];
    if (kv_page_ok(c, t.last)) t.holders = c.refs[t.last];
    return t;
}

// One workgroup.  The loads of the first 1,024 entries and words of free bits are
// started before the first barrier: a batch of up to that many waits for memory
// four times in a row (its slots, lengths, last pages, and their holders).  256
// sequences with a token each among 13,000 pages: 5.4 us; 256 that copy a shared page
// and get 64 tokens each: 8.5 us.
__global__ void __launch_bounds__(kKvPlanThreads) kv_extend_plan_kernel(KvExtend x) {
    const KvView &c = x.c;
    const int tid = (int)threadIdx.x;
    const int32_t words = (c.num_pages + 63) / 64;
    __shared__ int32_t copies, skipped;
    __shared__ uint32_t granted;
    if (tid == 0) copies = skipped = granted = 0;
    const KvEntry e0 = kv_entry(x, tid);
    const unsigned long long w0 = tid < words ? kv_free_word(c, tid) : 0;
    // a slot's first entry
    auto claims = [&](const KvEntry &e) { return kv_slot_ok(c, e.slot) && e.add > 0; };
    for (int64_t i = tid; i < x.n; i += kKvPlanThreads) {
        const KvEntry e = i == tid ? e0 : kv_entry(x, i);
        if (claims(e)) x.owner[e.slot] = INT32_MAX;
    }
    const KvTail t0 = kv_tail(c, e0);
    __syncthreads();
    for (int64_t i = tid; i < x.n; i += kKvPlanThreads) {
        const KvEntry e = i == tid ? e0 : kv_entry(x, i);
        if (claims(e)) atomicMin(&x.owner[e.slot], (int32_t)i);
    }
    // free pages
    uint32_t mine = (uint32_t)__popcll(w0), available = 0;
    for (int32_t w = tid + kKvPlanThreads; w < words; w += kKvPlanThreads) mine += (uint32_t)__popcll(kv_free_word(c, w));
    kv_block_before(mine, &available);
    if (available > x.most) available = (uint32_t)x.most;
    // pages each entry needs, in the order of the batch: the first that finds too few
    // left is refused, and with it every later one that needs a page
    uint32_t upto = 0;
    for (int64_t i0 = 0; i0 < x.n; i0 += kKvPlanThreads) {
        const int64_t i = i0 + tid;
        const KvEntry e = i0 == 0 ? e0 : kv_entry(x, i);
        const KvTail t = i0 == 0 ? t0 : kv_tail(c, e);
        KvGrant g{t.start, -1, -1};
        uint32_t need = 0;
        if (e.add == 0 && kv_slot_ok(c, e.slot)) {
            g.slot = e.slot;  // nothing to do, and nothing wrong
        } else if (claims(e) &&
                   __hip_atomic_load(&x.owner[e.slot], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == i &&
                   t.start + e.add <= (int64_t)c.slot_pages << c.page_shift &&
                   (kv_page_ok(c, t.last) || !(t.start & (kv_page_tokens(c) - 1)))) {
            g.slot = e.slot;
            if (t.holders > 1) g.source = t.last;
            need = (uint32_t)(kv_pages(c, t.start + e.add) - kv_pages(c, t.start) + (g.source >= 0));
        }
        uint32_t asked = 0;
        const uint32_t before = kv_add(upto, kv_block_before(need, &asked)), after = kv_add(before, need);
        upto = kv_add(upto, asked);
        if (need > 0) {
            if (after > available) g.slot = g.source = -1;
            else atomicMax(&granted, after);
        }
        if (i < x.n) {
            if (g.slot < 0 && e.slot != -1) atomicAdd(&skipped, 1);
            x.grant[i] = g;
            x.rank[i] = (int32_t)(before < INT32_MAX ? before : INT32_MAX);
            if (g.source >= 0) x.copies[atomicAdd(&copies, 1)] = (int32_t)i;
            if (g.slot >= 0 && e.add > 0) c.lengths[g.slot] = g.start + (int32_t)e.add;
        }
    }
    __syncthreads();
    // the lowest free pages
    const uint32_t wanted = granted;
    uint32_t seen = 0;
    for (int32_t f = 0; f < words && seen < wanted; f += kKvPlanThreads) {
        const int32_t w = f + tid;
        const unsigned long long bits = f == 0 ? w0 : (w < words ? kv_free_word(c, w) : 0);
        uint32_t all = 0;
        const uint32_t r = seen + kv_block_before((uint32_t)__popcll(bits), &all);
        // the word's first wanted - r free pages are taken
        unsigned long long taken = r < wanted ? bits : 0;
        if (taken && r + (uint32_t)__popcll(bits) > wanted) {
            taken = 0;
            unsigned long long left = bits;
            for (uint32_t k = r; k < wanted; ++k, left &= left - 1) taken |= left & (~left + 1);
        }
        kv_each_bit(taken, f, r, min(words, (int32_t)wanted), [&](uint32_t rank, int32_t p) {
            x.fresh[rank] = p;
            c.refs[p] = 1;
        });
        if (taken) c.free_pages[w] = bits & ~taken;
        seen += all;
    }
    if (tid == 0) {
        x.count[0] = (int32_t)wanted;
        x.count[1] = copies;
        if (skipped) atomicAdd(c.skipped, (unsigned long long)skipped);
    }
}

// Copies the first `tokens` tokens of page src to page dst, one (layer, head) of
// keys or values, by one wave, four units a lane on their way at once.
template <typename T>
__device__ inline void kv_copy_tokens(const T *src, T *dst, bool keys, int32_t tokens, const KvView &c) {
    using V8 = __attribute__((ext_vector_type(8))) T;
    using V4 = __attribute__((ext_vector_type(4))) T;
    const int32_t lane = (int32_t)(threadIdx.x & 63);
    if (keys) {
        const int32_t units = c.head_dim / 8 * tokens;
        for (int32_t u0 = lane; u0 < units; u0 += 256) {
            V8 x[4];
            int32_t at[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t u = (uint32_t)(u0 + 64 * i), block = u / (uint32_t)tokens;
                at[i] = kv_key_at(c, (int32_t)(u - block * (uint32_t)tokens), (int32_t)block * 8);
                if (u < (uint32_t)units) x[i] = *(const V8 *)(src + at[i]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (u0 + 64 * i < units) *(V8 *)(dst + at[i]) = x[i];
        }
    } else {
        const int32_t whole = tokens / 4 * c.head_dim, units = (tokens + 3) / 4 * c.head_dim;
        for (int32_t u0 = lane; u0 < whole; u0 += 256) {
            V4 x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (u0 + 64 * i < whole) x[i] = *(const V4 *)(src + 4 * (u0 + 64 * i));
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (u0 + 64 * i < whole) *(V4 *)(dst + 4 * (u0 + 64 * i)) = x[i];
        }
        for (int32_t u = whole + lane; u < units; u += 64)
            for (int32_t e = 0; e < (tokens & 3); ++e) dst[4 * u + e] = src[4 * u + e];
    }
}

// The last of the n numbers in a, which do not decrease, that is at most v (0 if none is).
template <typename N>
__device__ __forceinline__ int64_t kv_last_at_most(const N *a, int64_t n, int64_t v) {
    int64_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const int64_t mid = (lo + hi) >> 1;
        if (a[mid] <= v) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The first `row_blocks` workgroups: each row's place, the new pages into the tables,
// and the copied pages' counts.  The others: the copies, a wave for each (layer, head,
// keys or values).
template <typename T>
__global__ void __launch_bounds__(256) kv_extend_place_kernel(KvExtend x, uint32_t row_blocks) {
    const KvView &c = x.c;
    if (blockIdx.x < row_blocks) {
        const int64_t step = (int64_t)row_blocks * 256, first = (int64_t)blockIdx.x * 256 + threadIdx.x;
        for (int64_t r = first; r < x.rows; r += step) {
            int32_t to = -1;
            if (x.n > 0) {
                // a token each, or the last entry that begins at or before r
                const bool each = x.rows == x.n && x.offsets[r] == r && x.offsets[r + 1] == r + 1;
                const int64_t i = each ? r : kv_last_at_most(x.offsets, x.n, r);
                const KvGrant g = x.grant[i];
                const int64_t a = x.offsets[i];
                if (g.slot >= 0 && r >= a && r < x.offsets[i + 1]) {
                    const int64_t pos = g.start + (r - a);
                    const int32_t col = (int32_t)(pos >> c.page_shift), old = kv_pages(c, g.start) - (g.source >= 0);
                    const int32_t page = col >= old ? x.fresh[x.rank[i] + col - old]
                                                    : c.table[(int64_t)g.slot * c.slot_pages + col];
                    if (kv_page_ok(c, page)) to = (page << c.page_shift) + (int32_t)(pos & (kv_page_tokens(c) - 1));
                }
            }
            x.place[r] = to;
        }
        const int32_t pages = x.count[0];
        for (int64_t r = first; r < pages; r += step) {
            const int64_t i = kv_last_at_most(x.rank, x.n, r);
            const KvGrant g = x.grant[i];
            const int32_t at = kv_pages(c, g.start) - (g.source >= 0) + (int32_t)(r - x.rank[i]);
            if (g.slot >= 0 && (uint32_t)at < (uint32_t)c.slot_pages)
                c.table[(int64_t)g.slot * c.slot_pages + at] = x.fresh[r];
        }
        // copied pages have one holder less; the last one's leaving frees them
        for (int64_t k = first; k < x.count[1]; k += step) {
            const int32_t p = x.grant[x.copies[k]].source;
            if (atomicSub(&c.refs[p], 1) == 1) atomicOr(&c.free_pages[p >> 6], 1ull << (p & 63));
        }
        return;
    }
    const uint32_t waves = (gridDim.x - row_blocks) * 4, each = (uint32_t)c.layers * (uint32_t)c.kv_heads * 2;
    const uint64_t items = (uint64_t)(uint32_t)x.count[1] * each;
    for (uint64_t it = (blockIdx.x - row_blocks) * 4 + (threadIdx.x >> 6); it < items; it += waves) {
        const KvGrant g = x.grant[x.copies[it / each]];
        const uint32_t y = (uint32_t)(it % each), layer = (y >> 1) / (uint32_t)c.kv_heads;
        const bool keys = y & 1;
        const int64_t at = layer * (keys ? c.k_layer : c.v_layer) +
                           kv_head_base(c, (int32_t)((y >> 1) - layer * (uint32_t)c.kv_heads));
        T *pool = (T *)(keys ? c.k : c.v) + at;
        const int64_t page = keys ? c.k_page : c.v_page;
        kv_copy_tokens<T>(pool + g.source * page, pool + x.fresh[x.rank[x.copies[it / each]]] * page, keys,
                          g.start & (kv_page_tokens(c) - 1), c);
    }
}

// ---- rows ------------------------------------------------------------------------
// A scale without its power of two, so that quotients by it neither overflow nor lose
// bits: number / scale is (number * shift) / unit.
struct KvUnit {
    float shift, unit, over;  // over: 1 / unit
};

struct KvRows {
    KvView c;
    const int32_t *place;
    const void *k, *v;
    int64_t k_stride, v_stride, rows, layer;
    bool aligned;  // rows may be read 16 bytes at a time
    KvUnit k_unit, v_unit;
};

// Conversion of eight 16-bit numbers of a row to what the cache holds.
struct KvSame {
    using T = uint16_t;
    __device__ static void put(const uint16_t *in, const KvUnit &, T *out) {
        for (int i = 0; i < 8; ++i) out[i] = in[i];
    }
};
// Nearest e4m3 of number / scale.  The conversion instruction rounds to nearest, ties
// to even.  The quotient's own rounding must not make a tie of what is none (1.25 by the
// float next to 1.25 / 19 is not 19, which lies between 18 and 20): an inexact one is made
// odd, towards the exact one, and so keeps its side of every tie.  A product with the
// reciprocal, corrected once by what it leaves, does for the division (34,000 rows of 8
// heads of 128: 56 us; with divisions 66, and 52 without the care for ties).
template <bool BF16>
struct KvE4m3 {
    using T = uint8_t;
    __device__ static float quotient(uint16_t b, const KvUnit &u) {
        float x;
        if (BF16) x = __uint_as_float((uint32_t)b << 16);
        else x = (float)__builtin_bit_cast(_Float16, b);
        const float top = 456.f * u.unit;  // between 448, the last, and what would round past it
        const float in = __builtin_amdgcn_fmed3f(x * u.shift, -top, top);
        float y = in * u.over;
        y = __builtin_fmaf(__builtin_fmaf(-y, u.unit, in), u.over, y);  // the nearest, or beside it next to a tie of floats
        const uint32_t left = __float_as_uint(__builtin_fmaf(-y, u.unit, in)), bits = __float_as_uint(y);
        const uint32_t inexact = min(left << 1, 1u);
        // towards 0, and odd if inexact
        y = __uint_as_float((bits - ((bits ^ left) >> 31 & inexact)) | inexact);
        return x != x ? x : y;
    }
    __device__ static void put(const uint16_t *in, const KvUnit &u, T *out) {
        for (int i = 0; i < 8; i += 4) {
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(in[i], u), quotient(in[i + 1], u), 0, false);
            w = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(in[i + 2], u), quotient(in[i + 3], u), w, true);
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

// A thread takes eight dimensions of a row's key: 8 contiguous numbers.  Of the value
// it takes the same eight dimensions' single numbers, 4 tokens apart (a decode step);
// where the batch has a block's four tokens in a row (prompts), it takes two of the
// eight dimensions for all four, 8 contiguous numbers again.  A wave has eight rows'
// threads side by side, so that rows are read and keys are written 128 bytes at a
// time, and reads its rows' places and their neighbours' at once, beside its keys.
// Prompts: 59 us for the 280 MB of 34,000 rows of 8 heads of 128 (4.8 TB/s), against
// 76 us with the places read by each thread; a decode step's 256 rows: 4.1 us.
template <typename P>
__global__ void __launch_bounds__(256) kv_write_kernel(KvRows x) {
    using T = typename P::T;
    using V8 = __attribute__((ext_vector_type(8))) T;
    union Eight {
        T e[8];
        V8 v;
    } one;
    const KvView &c = x.c;
    const int32_t width = c.kv_heads * c.head_dim, lane = (int32_t)(threadIdx.x & 63);
    const uint32_t waves = ((uint32_t)width / 8 + 7) / 8;  // of a set of eight rows
    const uint64_t items = (uint64_t)(x.rows + 7) / 8 * waves;
    // Workgroup b runs on XCD b % 8: neighbouring rows, whose tokens share cache lines,
    // go to the same one.  The grid is in eights.
    const uint64_t each = gridDim.x / 8, b = (blockIdx.x & 7) * each + (blockIdx.x >> 3);
    for (uint64_t id = b * 4 + (threadIdx.x >> 6); id < items; id += 8 * each * 4) {
        const uint64_t set = items < (1ull << 32) ? (uint32_t)id / waves : id / waves;
        const int32_t dim = ((int32_t)(id - set * waves) * 8 + (lane >> 3)) * 8, near = 4 + (lane & 7);
        const int64_t r = (int64_t)set * 8 + (lane & 7);
        const bool in = dim < width && r < x.rows;
        const int32_t places = kv_place(x, (int64_t)set * 8 - 4 + (lane & 15));
        uint16_t key[8], val[8];
        if (in) kv_load8((const uint16_t *)x.k + r * x.k_stride + dim, x.aligned, key);
        const int32_t p = __shfl(places, near), q = p & 3;
        bool whole = true;
#pragma unroll
        for (int e = 0; e < 4; ++e) whole &= __shfl(places, near - q + e) == p - q + e;
        if (!in || p < 0) continue;

        const int32_t head = (int32_t)((uint32_t)dim / (uint32_t)c.head_dim), d = dim - head * c.head_dim;
        const int32_t t = p & (kv_page_tokens(c) - 1);
        const int64_t page = p >> c.page_shift;
        const uint16_t *vrow = (const uint16_t *)x.v + r * x.v_stride + dim;
        const int32_t two = 2 * q;
        if (whole) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint16_t *src = vrow + (e - q) * x.v_stride + two;
                const uint32_t w = x.aligned ? *(const uint32_t *)src : src[0] | (uint32_t)src[1] << 16;
                val[e] = (uint16_t)w;
                val[4 + e] = (uint16_t)(w >> 16);
            }
        } else {
            kv_load8(vrow, x.aligned, val);
        }
        P::put(key, x.k_unit, one.e);
        *(V8 *)((T *)c.k + x.layer * c.k_layer + page * c.k_page + kv_head_base(c, head) + kv_key_at(c, t, d)) = one.v;
        P::put(val, x.v_unit, one.e);
        T *dst = (T *)c.v + x.layer * c.v_layer + page * c.v_page + kv_head_base(c, head) + kv_value_at(c, t & ~3, d);
        if (whole) {
            *(V8 *)(dst + 4 * two) = one.v;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) dst[4 * i + q] = one.e[i];
        }
    }
}

// ---- forks and trims ---------------------------------------------------------------
// A workgroup an entry decides what becomes of it.  In small batches it also changes
// the table and the counts, four pages a thread on their way at once.  In large ones
// (see kKvShared) it leaves its pages to a second launch, in which a workgroup takes
// 64 columns of all the entries' tables: forks of one sequence hold the same page in
// the same column, so their changes of its count are joined first.  (256 forks of 3
// sequences of 1,300 to 3,100 scattered pages change half a million counts, 20 a
// nanosecond at best: 24 us; joined, 9,000 are left.)
constexpr int kKvPageThreads = 1024, kKvPageTurn = 4;
constexpr int64_t kKvShared = 1 << 17;  // pages of a batch's tables from which there is a second launch
constexpr int kKvSharedEntries = 64;    // entries of one of its workgroups: four a wave, on their way at once

struct KvChange {
    KvView c;
    const int32_t *src, *dst, *count;  // fork: sources, forks, tokens; trim: -, slots, keep
    int64_t stride, n;                 // of count
    int2 *columns;                     // per entry: first and last column that changes (nullptr: small batch)
};

// What becomes of the pages of one entry's table row in columns [lo, hi).
template <bool FORK>
__device__ inline void kv_change_row(const KvChange &x, int64_t i, int32_t lo, int32_t hi) {
    const KvView &c = x.c;
    if (x.columns) {
        if (threadIdx.x == 0) x.columns[i] = make_int2(lo, hi);
        return;
    }
    int32_t *row = c.table + (int64_t)x.dst[i] * c.slot_pages;
    const int32_t *from = FORK ? c.table + (int64_t)x.src[i] * c.slot_pages : row;
    for (int32_t k0 = lo + (int32_t)threadIdx.x; k0 < hi; k0 += kKvPageThreads * kKvPageTurn) {
        int32_t p[kKvPageTurn], held[kKvPageTurn];
#pragma unroll
        for (int e = 0; e < kKvPageTurn; ++e) p[e] = k0 + e * kKvPageThreads < hi ? from[k0 + e * kKvPageThreads] : -1;
#pragma unroll
        for (int e = 0; e < kKvPageTurn; ++e) {
            if (k0 + e * kKvPageThreads < hi) row[k0 + e * kKvPageThreads] = FORK ? p[e] : -1;
            held[e] = 0;
            if (kv_page_ok(c, p[e])) {
                if (FORK) atomicAdd(&c.refs[p[e]], 1);
                else held[e] = atomicSub(&c.refs[p[e]], 1);
            }
        }
#pragma unroll
        for (int e = 0; e < kKvPageTurn; ++e)
            if (!FORK && held[e] == 1) atomicOr(&c.free_pages[p[e] >> 6], 1ull << (p[e] & 63));
    }
}

__global__ void __launch_bounds__(kKvPageThreads) kv_fork_kernel(KvChange x) {
    const KvView &c = x.c;
    const int64_t i = blockIdx.x;
    const int32_t from = x.src[i], to = x.dst[i], keep = x.count[i];
    __shared__ int32_t clash;
    if (threadIdx.x == 0) clash = 0;
    __syncthreads();
    if (to != -1)
        for (int64_t k = threadIdx.x; k < x.n; k += kKvPageThreads)
            if (x.dst[k] == from || (k < i && x.dst[k] == to)) clash = 1;
    __syncthreads();
    // lengths[to] is read before this workgroup, the only one that may, writes it
    const bool ok = to != -1 && !clash && kv_slot_ok(c, from) && kv_slot_ok(c, to) && keep >= 0 &&
                    keep <= kv_length(c, from) && c.lengths[to] == 0;
    __syncthreads();
    if (threadIdx.x == 0) {
        if (ok) c.lengths[to] = keep;
        else if (to != -1) atomicAdd(c.skipped, 1ull);
    }
    kv_change_row<true>(x, i, 0, ok ? kv_pages(c, keep) : 0);
}

__global__ void __launch_bounds__(kKvPageThreads) kv_trim_kernel(KvChange x) {
    const KvView &c = x.c;
    const int64_t i = blockIdx.x;
    const int32_t slot = x.dst[i], to = x.count ? x.count[i * x.stride] : 0;
    const bool ok = kv_slot_ok(c, slot) && to >= 0;
    // of the entries that name a slot each frees what its own minimum cuts off
    __shared__ int32_t had;
    if (threadIdx.x == 0) {
        had = ok ? atomicMin(&c.lengths[slot], to) : 0;
        if (!ok && slot != -1) atomicAdd(c.skipped, 1ull);
    }
    __syncthreads();
    const int32_t was = min(had, c.slot_pages << c.page_shift);
    if (ok && was > to) kv_change_row<false>(x, i, kv_pages(c, to), kv_pages(c, was));
    else kv_change_row<false>(x, i, 0, 0);
}

// 64 columns of kKvSharedEntries entries' table rows: a lane a column, a wave every
// sixteenth entry.  A column has places for the counts of 16 pages; what finds none is
// changed by itself.
template <bool FORK>
__global__ void __launch_bounds__(kKvPageThreads) kv_change_columns_kernel(KvChange x) {
    constexpr int PLACES = 16, WAVES = kKvPageThreads / 64, EACH = kKvSharedEntries / WAVES;
    const KvView &c = x.c;
    __shared__ int32_t page[PLACES][64], count[PLACES][64];
    __shared__ int2 columns[kKvSharedEntries];
    __shared__ int32_t to[kKvSharedEntries], from[kKvSharedEntries];
    const int lane = (int)(threadIdx.x & 63), wave = uniform((int)(threadIdx.x >> 6));
    const int64_t first = (int64_t)blockIdx.y * kKvSharedEntries;
    if (threadIdx.x < kKvSharedEntries) {
        const int64_t i = first + threadIdx.x;
        columns[threadIdx.x] = i < x.n ? x.columns[i] : make_int2(0, 0);
        to[threadIdx.x] = i < x.n ? x.dst[i] : -1;
        from[threadIdx.x] = FORK && i < x.n ? x.src[i] : -1;
    }
    page[wave][lane] = -1;
    count[wave][lane] = 0;
    __syncthreads();
    const int32_t col = (int32_t)blockIdx.x * 64 + lane;
    auto change = [&](int32_t p, int32_t by) {
        if (FORK) atomicAdd(&c.refs[p], by);
        else if (atomicSub(&c.refs[p], by) == by) atomicOr(&c.free_pages[p >> 6], 1ull << (p & 63));
    };
    int32_t p[EACH];
    bool in[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const int i = wave + e * WAVES;
        in[e] = col >= columns[i].x && col < columns[i].y;
        p[e] = in[e] ? c.table[(int64_t)(FORK ? from : to)[i] * c.slot_pages + col] : -1;
    }
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        if (!in[e]) continue;
        c.table[(int64_t)to[wave + e * WAVES] * c.slot_pages + col] = FORK ? p[e] : -1;
        if (!kv_page_ok(c, p[e])) continue;
        const int at = p[e] & (PLACES - 1);
        const int32_t was = atomicCAS(&page[at][lane], -1, p[e]);
        if (was == -1 || was == p[e]) atomicAdd(&count[at][lane], 1);
        else change(p[e], 1);
    }
    __syncthreads();
    static_assert(PLACES == WAVES && EACH * WAVES == kKvSharedEntries, "a thread a place, all entries dealt");
    if (count[wave][lane]) change(page[wave][lane], count[wave][lane]);
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
    uint32_t mine = 0, unheld = 0;
    for (int32_t w = tid; w < words; w += kKvPlanThreads) mine += (uint32_t)__popcll(kv_free_word(c, w));
    kv_block_before(mine, &unheld);
    const int32_t held = c.num_pages - (int32_t)unheld;
    uint32_t holes = 0, movers = 0;
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
        uint32_t all = 0;
        uint32_t r = holes + kv_block_before((uint32_t)__popcll(hole), &all);
        holes += all;
        kv_each_bit(hole, w0, r, words, [&](uint32_t rank, int32_t p) { x.target[rank] = p; });
        r = movers + kv_block_before((uint32_t)__popcll(move), &all);
        movers += all;
        kv_each_bit(move, w0, r, words, [&](uint32_t rank, int32_t p) { x.from[rank] = p; });
    }
    __syncthreads();
    const int32_t n = (int32_t)min(holes, movers);  // equal, unless the free bits are not the counts'
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
// time, and the tables: 302 us for 3,000 pages of 262 KB, 4.9 TB/s.
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

// ---- attention's split of large batches, see kv_planned_share --------------------------------
__global__ void __launch_bounds__(kKvPlanThreads) kv_plan_kernel(KvAttend a) {
    const int tid = (int)threadIdx.x;
    auto steps = [&](int64_t i) -> uint32_t {
        if (i >= a.n) return 0;
        const int32_t s = a.slots[i];
        return kv_steps(kv_span(kv_slot_ok(a.c, s) ? kv_length(a.c, s) : 0, a.window));
    };
    auto sums = [&](int32_t *out, auto of) {
        uint32_t before = 0;
        for (int64_t i0 = 0; i0 < a.n; i0 += kKvPlanThreads) {
            const int64_t i = i0 + tid;
            uint32_t all = 0;
            const uint32_t at = before + kv_block_before(of(i), &all);
            if (i < a.n) out[i] = (int32_t)at;
            before += all;
        }
        if (tid == 0) out[a.n] = (int32_t)before;
        return before;
    };
    const uint32_t total = sums(a.plan, steps);
    if (!kv_keeps(total, a.n, a.split)) return;
    const uint32_t size = kv_share(total, a.split);
    auto shares = [&](int64_t i) { return (steps(i) + size - 1) / size; };
    sums(a.plan + a.n + 1, shares);
    sums(a.plan + 2 * (a.n + 1), [&](int64_t i) {
        const uint32_t n = shares(i);
        return n > 1 ? n : 0;
    });
}

}  // namespace pr

#endif
