// kv_attend.h -- attention of one new token a sequence over the paged cache.
//
// out = sum_t 2^(x_t - m) v_t / sum_t 2^(x_t - m), x_t = scale log2(e) q . k_t, m
// the largest x_t met so far: one pass over keys and values with a running
// maximum and sum.  Nothing is read twice and a token's 4 head_dim bytes (16-bit
// types) meet 4 * group * head_dim operations, so the pass is bound by the HBM
// reads; the matrix units have an order of magnitude to spare (5.7% busy).  128
// sequences of 4,096 to 16,384 tokens, 64 heads on 8 of 128, bfloat16: 908 us, 6.0 TB/s.
#ifndef PR_KV_ATTEND_H
#define PR_KV_ATTEND_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "kv_launch.h"
#include "kv_layout.h"
#include "wave_ops.h"

namespace pr {

using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
using f16x2 = __attribute__((ext_vector_type(2))) _Float16;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using f16x8 = __attribute__((ext_vector_type(8))) _Float16;
using f32x4 = __attribute__((ext_vector_type(4))) float;
using u32x2 = __attribute__((ext_vector_type(2))) uint32_t;
using u32x4 = __attribute__((ext_vector_type(4))) uint32_t;

// The two 16-bit types the matrix units take.
struct Bf16 {
    __device__ static f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    }
    __device__ static uint32_t pack(float x, float y) {
        return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x, (__bf16)y});
    }
    __device__ static float low(uint32_t p) { return __builtin_bit_cast(float, p << 16); }
    __device__ static float high(uint32_t p) { return __builtin_bit_cast(float, p & 0xffff0000u); }
    template <bool HI>
    __device__ static uint32_t from_e4m3(uint32_t w) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HI));
    }
};
struct F16 {
    __device__ static f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
                                                      0, 0);
    }
    __device__ static uint32_t pack(float x, float y) {
        return __builtin_bit_cast(uint32_t, f16x2{(_Float16)x, (_Float16)y});
    }
    __device__ static float low(uint32_t p) { return (float)__builtin_bit_cast(f16x2, p)[0]; }
    __device__ static float high(uint32_t p) { return (float)__builtin_bit_cast(f16x2, p)[1]; }
    template <bool HI>
    __device__ static uint32_t from_e4m3(uint32_t w) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, HI));
    }
};

// Eight numbers of the cache as they are loaded, and as the matrix units take
// them.  An e4m3 number is a bfloat16 and a half number exactly.
template <typename IO, bool E4M3>
struct Eight;
template <typename IO>
struct Eight<IO, false> {
    using Raw = u32x4;
    __device__ static u32x4 wide(Raw r) { return r; }
};
template <typename IO>
struct Eight<IO, true> {
    using Raw = u32x2;
    __device__ static u32x4 wide(Raw r) {
        return u32x4{IO::template from_e4m3<false>(r[0]), IO::template from_e4m3<true>(r[0]),
                     IO::template from_e4m3<false>(r[1]), IO::template from_e4m3<true>(r[1])};
    }
};

// Eight values of the cache as bfloat16, whose exponents the weights need (see the
// kernel).  A half number is the sum of two bfloat16 numbers, exactly: the nearest
// leaves at most three bits.
template <typename IO, bool E4M3>
struct Values {
    static constexpr bool kTwo = std::is_same_v<IO, F16> && !E4M3;
    u32x4 first, rest;  // rest: kTwo only
    __device__ explicit Values(typename Eight<IO, E4M3>::Raw r) {
        if constexpr (kTwo) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = F16::low(r[i]), y = F16::high(r[i]);
                first[i] = Bf16::pack(x, y);
                rest[i] = Bf16::pack(x - Bf16::low(first[i]), y - Bf16::high(first[i]));
            }
        } else {
            first = Eight<Bf16, E4M3>::wide(r);
        }
    }
};

// The larger of / the sum over the four lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ float rows_max(float x) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float rows_sum(float x) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

using Scalar = const __attribute__((address_space(4))) int32_t;  // read by scalar loads
__device__ __forceinline__ Scalar *scalar(const int32_t *p) { return (Scalar *)(uintptr_t)p; }

// The steps [begin, end) a workgroup takes, `first` of which are before those of the
// entry it begins with (-1: nothing to take).  Of shares of `size` steps it is number
// `index`.  Sequences follow each other in the numbering of the steps, or, where
// shares keep to sequences, each has a numbering of its own (first = index = 0).
struct KvShare {
    uint32_t begin, end, size, first, index;
    int32_t entry;
    uint32_t number;  // see kv_part_at
};
__device__ __forceinline__ KvShare kv_share_of(uint32_t u, uint32_t size, uint32_t steps, const KvSplit &s) {
    KvShare r{kv_share_begin(u, size, steps, s), steps, size, 0, u, -1, u};
    r.end = min(r.begin + size, steps);
    return r;
}
// Share k of an entry's own, `split` the shares of the entries before it that have several.
__device__ __forceinline__ KvShare kv_own_share(int32_t entry, uint32_t steps, uint32_t shares, uint32_t k,
                                                uint32_t split) {
    const uint32_t size = kv_even(steps, shares);
    return KvShare{k * size, min((k + 1) * size, steps), size, 0, 0, entry, split + k};
}

// Share u of a batch of at most E * 64 entries, found by every wave for itself from
// the lengths: two loads and two dozen lane operations, about 1 us, where a launch
// before this one that wrote the same down is 2.5 us and its work.  The loads have no
// conditions, behind which each would be waited for before the next.
template <int E>
__device__ inline KvShare kv_find_share(const KvAttend &a, uint32_t u) {
    const int lane = (int)(threadIdx.x & 63);
    int32_t slot[E], length[E];
    uint32_t mine[E], upto[E], total = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) slot[e] = a.slots[min(e * 64 + lane, (int32_t)a.n - 1)];
#pragma unroll
    for (int e = 0; e < E; ++e) length[e] = kv_length(a.c, kv_slot_ok(a.c, slot[e]) ? slot[e] : 0);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if (!kv_slot_ok(a.c, slot[e])) length[e] = 0;
        mine[e] = e * 64 + lane < a.n ? kv_steps(kv_span(length[e], a.window)) : 0;
    }
    auto add = [&] {
        total = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            upto[e] = total + (uint32_t)lanes_upto((int32_t)mine[e]);
            total = (uint32_t)__builtin_amdgcn_readlane((int)upto[e], 63);
        }
    };
    // lane `i` of the batch's
    auto of = [&](const uint32_t *x, int i) {
        uint32_t r = 0;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e == i >> 6) r = (uint32_t)__builtin_amdgcn_readlane((int)x[e], i & 63);
        return r;
    };
    // the entry in whose part of the sums v lies
    int entry = -1;
    uint32_t before = 0, its = 0;
    auto find = [&](uint32_t v) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint64_t past = __ballot(upto[e] > v);
            if (past && entry < 0) {
                const int src = __builtin_ctzll(past);
                entry = e * 64 + src;
                its = (uint32_t)__builtin_amdgcn_readlane((int)mine[e], src);
                before = (uint32_t)__builtin_amdgcn_readlane((int)upto[e], src) - its;
            }
        }
    };
    add();
    const uint32_t size = kv_share(total, a.split);
    if (!kv_keeps(total, a.n, a.split)) {
        KvShare r = kv_share_of(u, size, total, a.split);
        find(r.begin);
        r.entry = entry;
        r.first = before;
        return r;
    }
    uint32_t steps[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        steps[e] = mine[e];
        mine[e] = (mine[e] + size - 1) / size;
    }
    add();
    find(u);
    if (entry < 0) return KvShare{0, 0, 1, 0, 0, -1, 0};
    uint32_t split = 0;
    if (its > 1) {
#pragma unroll
        for (int e = 0; e < E; ++e) mine[e] = mine[e] > 1 ? mine[e] : 0;
        add();
        split = of(upto, entry) - its;
    }
    return kv_own_share(entry, of(steps, entry), its, u - before, split);
}

// The same from a plan (kv_plan_kernel) for larger batches: a.plan[i] is the steps
// before entry i, a.plan[n] all of them; where shares keep to sequences, a.plan[n + 1 + i]
// is the shares before entry i, a.plan[2 n + 2 + i] those of entries that have several.
__device__ inline KvShare kv_planned_share(const KvAttend &a, uint32_t u) {
    Scalar *before = scalar(a.plan);
    const uint32_t total = (uint32_t)before[a.n];
    const bool keeps = kv_keeps(total, a.n, a.split);
    KvShare r = kv_share_of(u, kv_share(total, a.split), total, a.split);
    Scalar *sums = keeps ? before + a.n + 1 : before;
    const uint32_t v = keeps ? u : r.begin;
    if (v >= (uint32_t)sums[a.n]) return r;
    int32_t lo = 0, hi = (int32_t)a.n;  // sums[lo] <= v < sums[hi]
    while (hi - lo > 1) {
        const int32_t mid = (lo + hi) >> 1;
        if ((uint32_t)sums[mid] <= v) lo = mid;
        else hi = mid;
    }
    if (keeps)
        return kv_own_share(lo, (uint32_t)before[lo + 1] - (uint32_t)before[lo], (uint32_t)sums[lo + 1] - (uint32_t)sums[lo],
                            u - (uint32_t)sums[lo], (uint32_t)sums[a.n + 1 + lo]);
    r.entry = lo;
    r.first = (uint32_t)before[lo];
    return r;
}

// A share's part of one entry: its tokens from `from` to `to`, of those from `begin` on.
struct KvWork {
    int32_t entry, slot, length, begin, from, to;
    uint32_t steps;    // of the entry
    bool whole, begins, last;  // all of the entry; its first part; the share ends with it
};

// One workgroup: an equal share of the batch's tokens, mostly a part of one entry's,
// one key head, 16 R of its query heads ("rows").  Its waves take the 32-token tiles in
// turn, each with a running maximum and sum of its own, and are joined at the end of
// an entry's part.
//
// Scores are taken transposed, S^T = K Q^T (16 tokens x 16 rows, head_dim / 32
// MFMAs): a lane then holds eight of the tile's tokens of one row, which are the
// operand's eight numbers of O^T = V^T P^T over 32 tokens, so weights never leave
// their lane; and all of a lane's output numbers are of that row, so neither does
// the rescaling.  Which token is which of a lane's eight is free as long as V's
// operand agrees: a lane takes tokens 4g..4g+3 of each 16 (g = lane / 16), two
// dimensions of four tokens being 16 contiguous bytes of a page; keys come in 16
// contiguous bytes too.  Keys and values go from memory to the matrix units'
// registers without LDS.
//
// Weights are rounded to bfloat16 twice, once for the weight and once for what that
// left over, so that each term of the sum is good to 2^-17, however small its weight
// (half numbers end at 2^-24 of the largest: thousands of such weights beside one large
// one whose value is 0 are the output), and the output's error is its own rounding; the
// second MFMA costs nothing next to the loads.  Half values are two bfloat16 numbers
// and take a third MFMA (the rest of the value by the rest of the weight is 2^-18).
template <typename IO, bool E4M3, int D, int R, int W>
__global__ void __launch_bounds__(64 * W, kv_resident(E4M3, D, R, W)) kv_attend_kernel(KvAttend a) {
    using Raw = typename Eight<IO, E4M3>::Raw;
    constexpr int KB = D / 32;  // MFMAs of a score; pairs of 16 dimensions
    constexpr int kStep = kKvTile * W;
    constexpr float kSlack = 8.f;
    constexpr int SZ = E4M3 ? 1 : 2;
    const KvView &c = a.c;
    const int wave = uniform((int)(threadIdx.x >> 6));

    // Blocks of the same keys differ by 8, so that they share an XCD's L2.
    const int32_t rg = (int32_t)((blockIdx.x >> 3) % (unsigned)a.row_groups);
    const int32_t uh = (int32_t)((blockIdx.x >> 3) / (unsigned)a.row_groups * 8 + (blockIdx.x & 7));
    const int32_t unit = (int32_t)((uint32_t)uh / (uint32_t)c.kv_heads), head = uh - unit * c.kv_heads;
    if (unit >= a.units) return;  // the grid is in eights
    // Without a.where, and always in a workgroup of many waves, a share is an entry.
    const bool shares = W == kKvWaves && a.where;
    KvShare w{0, 1, 1, 0, 0, unit, 0};
    if (shares) {
        if (a.plan) w = kv_planned_share(a, (uint32_t)unit);
        else w = a.n <= 64    ? kv_find_share<1>(a, (uint32_t)unit)
                 : a.n <= 128 ? kv_find_share<2>(a, (uint32_t)unit)
                              : kv_find_share<kKvScan / 64>(a, (uint32_t)unit);
        w.begin = (uint32_t)uniform((int)w.begin);
        w.end = (uint32_t)uniform((int)w.end);
        w.first = (uint32_t)uniform((int)w.first);
        w.entry = uniform(w.entry);
        w.number = (uint32_t)uniform((int)w.number);
        if (w.entry < 0) return;
    }
    const uint32_t share_begin = w.begin, share_end = w.end;
    uint32_t first = w.first;
    __shared__ f32x4 so[W][R * KB * 2][64];
    __shared__ float sm[W][R][16], sl[W][R][16];

    const int32_t row0 = rg * 16 * R, inside = kv_page_tokens(c) - 1, room = c.slot_pages << c.page_shift;
    const char *kbase = (const char *)c.k + SZ * (a.layer * c.k_layer + kv_head_base(c, head));
    const char *vbase = (const char *)c.v + SZ * (a.layer * c.v_layer + kv_head_base(c, head));

    // A tile's page ids, and those of the wave's next tile, are `here` and `next`.
    Scalar *pages = nullptr;
    int32_t t = 0, here[2], next[2];
    auto page_of = [&](int32_t tok) { return pages[min(tok, room - 1) >> c.page_shift]; };
    auto first_pages = [&](int32_t slot) __attribute__((always_inline)) {
        pages = scalar(c.table + (int64_t)slot * c.slot_pages);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            here[h] = page_of(t + 16 * h);
            next[h] = page_of(t + kStep + 16 * h);
        }
    };
    // Where a workgroup takes a whole sequence from its first token on, its first pages
    // are known before its length, and are read beside it (one sequence of 611 tokens:
    // 5.4 us, 5.8 with one after the other).
    const bool whole = !shares && !a.window;

    // The share's part of entry i, whose first step is the batch's step `first`.
    auto part_of = [&](int32_t i, uint32_t first) __attribute__((always_inline)) {
        const int32_t slot = scalar(a.slots)[i];
        const bool known = kv_slot_ok(c, slot);
        KvWork x;
        x.entry = i;
        x.slot = known ? slot : 0;
        const int32_t had = scalar(c.lengths)[x.slot];
        if (whole) {
            t = kKvTile * wave;
            first_pages(x.slot);
        }
        x.length = !known || had < 0 ? 0 : min(had, room);
        x.begin = 0;
        if (a.window > 0) x.begin = kv_first(x.length, a.window);
        const int32_t tile0 = x.begin & ~(kKvTile - 1);
        x.steps = shares ? kv_steps(x.length - tile0) : 1;
        const KvPart part = shares ? kv_part(share_begin, share_end, first, x.steps) : KvPart{0, 1, true};
        x.whole = part.whole;
        x.begins = part.from == 0;
        x.last = !shares || first + part.to >= share_end;
        x.from = tile0 + (int32_t)part.from * kKvStep;
        x.to = part.to == x.steps ? x.length : tile0 + (int32_t)part.to * kKvStep;
        if (x.begins && head == 0 && rg == 0 && threadIdx.x == 0) {
            if (shares) {
                a.where[2 * (int64_t)i] = (int32_t)kv_part_at(w.number, true);
                a.where[2 * (int64_t)i + 1] = (int32_t)kv_parts(w.index, w.size, first, x.steps);
            }
            if (!known && slot != -1) atomicAdd(c.skipped, 1ull);
        }
        return x;
    };

    // A tile's two halves of 16 tokens lie in one page each.  Page ids are read by scalar
    // loads: as vector loads they would be waited for behind every key and value on its
    // way.  The next tile's keys are asked for once this one's scores are taken, its values
    // once this one's are used, the next part's first tile and queries before this part's
    // waves are joined: the registers are free by then, and what is left to do hides the way.
    Raw kr[2][KB], vr[2][KB];
    u32x4 q[R][KB];
    KvWork part;
    uint32_t kl = 0, vl = 0;  // the lane's place in a tile of keys and of values
    auto load_keys = [&](int32_t t, const int32_t *pg) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t p = kv_page_ok(c, pg[h]) ? pg[h] : 0;
            const char *ks = kbase + SZ * (p * c.k_page + kv_key_at(c, (t + 16 * h) & inside, 0));
#pragma unroll
            for (int j = 0; j < KB; ++j) kr[h][j] = *(const Raw *)(ks + (SZ * 32 * j << c.page_shift) + kl);
        }
    };
    auto load_values = [&](int32_t t, const int32_t *pg) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t p = kv_page_ok(c, pg[h]) ? pg[h] : 0;
            const char *vs = vbase + SZ * (p * c.v_page + kv_value_at(c, (t + 16 * h) & inside, 0));
#pragma unroll
            for (int j = 0; j < KB; ++j) vr[h][j] = *(const Raw *)(vs + SZ * 128 * j + vl);
        }
    };
    // The lane is taken anew where a part begins and ends: what is computed from it would
    // otherwise be kept in registers over the loops, some twenty of them.
    auto fresh_lane = [] {
        int lane = (int)(threadIdx.x & 63);
        asm volatile("" : "+v"(lane));
        return lane;
    };
    auto start = [&]() __attribute__((always_inline)) {
        const int lane = fresh_lane(), col = lane & 15, g = lane >> 4;
        kl = (uint32_t)SZ * kv_key_at(c, col, 8 * g);
        vl = (uint32_t)SZ * kv_value_at(c, 4 * g, 2 * col);
        if (!whole) {
            t = part.from + kKvTile * wave;
            first_pages(part.slot);
        }
        auto load_queries = [&](auto aligned) __attribute__((always_inline)) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int32_t row = row0 + 16 * r + col;
                const uint16_t *src = (const uint16_t *)a.q + part.entry * a.q_stride +
                                      (int64_t)(head * a.group + (row < a.group ? row : 0)) * D + 8 * g;
#pragma unroll
                for (int j = 0; j < KB; ++j) {
                    if (decltype(aligned)::value) {
                        q[r][j] = *(const u32x4 *)(src + 32 * j);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            q[r][j][e] = src[32 * j + 2 * e] | (uint32_t)src[32 * j + 2 * e + 1] << 16;
                    }
                }
            }
        };
        // The queries before the keys, as what is loaded after them is not waited for with
        // them, and masked beside the loads, where what is on its way is known.
        if (t < part.to) {
            if (a.q_aligned) load_queries(std::true_type());
            else load_queries(std::false_type());
            load_keys(t, here);
            load_values(t, here);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                uint32_t keep = row0 + 16 * r + col < a.group ? ~0u : 0;
                asm volatile("" : "+v"(keep));  // a mask, no branch, past which the queries might be on their way
#pragma unroll
                for (int j = 0; j < KB; ++j) q[r][j] &= keep;
            }
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int j = 0; j < KB; ++j) q[r][j] = u32x4{0, 0, 0, 0};
        }
    };

    part = part_of(w.entry, first);
    start();
    for (;;) {
        const int lane = fresh_lane(), g = lane >> 4;
        f32x4 o[R][KB][2];  // dimensions 32 j + 2 (4 g + i) + e of row lane % 16: o[.][j][e][i]
        float m[R], l[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            m[r] = -INFINITY;
            l[r] = 0.f;
#pragma unroll
            for (int j = 0; j < KB; ++j) o[r][j][0] = o[r][j][1] = f32x4{0, 0, 0, 0};
        }

        // A wave's last tile is code of its own: loads behind a branch would have to be
        // waited for as if they might not be there, that is all of them at each use.
        auto tile = [&](auto another) __attribute__((always_inline)) {
            constexpr bool more = decltype(another)::value;
            const bool good[2] = {kv_page_ok(c, here[0]), kv_page_ok(c, here[1])};
            const bool full = good[0] && good[1] && t >= part.begin && t + kKvTile <= part.to;
            auto counts = [&](int h, int i) {  // the lane's token i of half h
                const int32_t tok = t + 16 * h + 4 * g + i;
                return good[h] && tok >= part.begin && tok < part.to;
            };

            u32x4 hi[R], lo[R];
            {
                f32x4 s[R][2];
#pragma unroll
                for (int r = 0; r < R; ++r) s[r][0] = s[r][1] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < KB; ++j) {
                        const u32x4 kk = Eight<IO, E4M3>::wide(kr[h][j]);
#pragma unroll
                        for (int r = 0; r < R; ++r) s[r][h] = IO::mfma(kk, q[r][j], s[r][h]);
                    }
                if (more) load_keys(t + kStep, next);
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int h = 0; h < 2; ++h) s[r][h] *= a.scale;
                if (!full) {
                    // Kept a branch: most tiles are full, and selections and masks that do
                    // nothing are a fifth of a tile's vector instructions (0.2 us of one
                    // sequence of 611 tokens).
                    asm volatile("");
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const bool in = counts(i >> 2, i & 3);
#pragma unroll
                        for (int r = 0; r < R; ++r) s[r][i >> 2][i & 3] = in ? s[r][i >> 2][i & 3] : -INFINITY;
                    }
                }
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    float x[8], top = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        x[i] = s[r][i >> 2][i & 3];
                        top = fmaxf(top, x[i]);
                    }
                    top = rows_max(top);
                    // m follows the maximum only once that is kSlack past it: until then weights
                    // up to 2^kSlack do no harm, and rescaling costs as much as a tile's scores
                    if (__ballot(!(top <= m[r] + kSlack))) {
                        const float most = fmaxf(m[r], top), base = most == -INFINITY ? 0.f : most;
                        const float shrink = exp2_fast(m[r] - base);
                        m[r] = most;
                        l[r] *= shrink;
#pragma unroll
                        for (int j = 0; j < KB; ++j) {
                            o[r][j][0] *= shrink;
                            o[r][j][1] *= shrink;
                        }
                    }
                    const float base = m[r] == -INFINITY ? 0.f : m[r];  // nothing yet, or nothing but -infinity
                    float sum = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        x[i] = exp2_fast(x[i] - base);
                        sum += x[i];
                    }
                    l[r] += sum;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        hi[r][i] = Bf16::pack(x[2 * i], x[2 * i + 1]);
                        lo[r][i] = Bf16::pack(x[2 * i] - Bf16::low(hi[r][i]), x[2 * i + 1] - Bf16::high(hi[r][i]));
                    }
                }
            }
            if (!full) {  // 0 times what lies behind a sequence could be NaN
                asm volatile("");
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    constexpr int bits = 8 * SZ, per = 4 / SZ;  // a token's, and tokens of a word
                    uint32_t keep[SZ] = {};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (counts(h, i)) keep[i / per] |= (0xffffffffu >> (32 - bits)) << (bits * (i % per));
#pragma unroll
                    for (int j = 0; j < KB; ++j)
#pragma unroll
                        for (int e = 0; e < 2 * SZ; ++e) vr[h][j][e] &= keep[e % SZ];
                }
            }
#pragma unroll
            for (int j = 0; j < KB; ++j) {
                const Values<IO, E4M3> v0(vr[0][j]), v1(vr[1][j]);
                auto pair = [](u32x4 a, u32x4 b, int e) { return u32x4{a[2 * e], a[2 * e + 1], b[2 * e], b[2 * e + 1]}; };
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const u32x4 vv = pair(v0.first, v1.first, e);
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        o[r][j][e] = Bf16::mfma(vv, hi[r], o[r][j][e]);
                        o[r][j][e] = Bf16::mfma(vv, lo[r], o[r][j][e]);
                        if constexpr (Values<IO, E4M3>::kTwo)
                            o[r][j][e] = Bf16::mfma(pair(v0.rest, v1.rest, e), hi[r], o[r][j][e]);
                    }
                }
            }
            if (more) load_values(t + kStep, next);
        };
        for (; t + kStep < part.to; t += kStep) {
            tile(std::true_type());
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                here[h] = next[h];
                next[h] = page_of(t + 2 * kStep + 16 * h);
            }
        }
        if (t < part.to) tile(std::false_type());
#pragma unroll
        for (int r = 0; r < R; ++r) l[r] = rows_sum(l[r]);

        const KvWork done = part;
        if (!done.last) {  // the share goes on with the next entry
            first += part.steps;
            part = part_of(part.entry + 1, first);
            start();
        }

        // Join the waves: all outputs on the largest maximum, then a wave sums the W of a
        // pair of 16 dimensions (each lane's eight are a row's, in a row).  Two barriers;
        // a tree takes two a level and leaves the last sums to one wave.
        if (g == 0)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                sm[wave][r][lane] = m[r];
                sl[wave][r][lane] = l[r];
            }
        __syncthreads();
        float total[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float most = -INFINITY;
            total[r] = 0.f;
#pragma unroll
            for (int k = 0; k < W; ++k) most = fmaxf(most, sm[k][r][lane & 15]);
            const float base = most == -INFINITY ? 0.f : most, x = exp2_fast(m[r] - base);
#pragma unroll
            for (int k = 0; k < W; ++k) total[r] += sl[k][r][lane & 15] * exp2_fast(sm[k][r][lane & 15] - base);
            m[r] = most;
#pragma unroll
            for (int j = 0; j < KB; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) so[wave][(r * KB + j) * 2 + e][lane] = o[r][j][e] * x;
        }
        __syncthreads();
        {
            const int lane = fresh_lane(), col = lane & 15, g = lane >> 4;
            for (int y = wave; y < R * KB; y += W) {
                const int r = R == 1 ? 0 : y / KB, j = R == 1 ? y : y % KB;
                const int32_t row = row0 + 16 * r + col;
                f32x4 u = so[0][2 * y][lane], v = so[0][2 * y + 1][lane];
#pragma unroll
                for (int k = 1; k < W; ++k) {
                    u += so[k][2 * y][lane];
                    v += so[k][2 * y + 1][lane];
                }
                if (row >= a.group) continue;
                const float most = R == 1 || r == 0 ? m[0] : m[R - 1], sum = R == 1 || r == 0 ? total[0] : total[R - 1];
                const int64_t at = ((int64_t)head * a.group) + row;
                if (done.whole) {
                    const int64_t to_row = (int64_t)done.entry * a.q_heads + at;
                    if (a.lse && j == 0 && g == 0)
                        a.lse[to_row] = (most + log2f(sum)) * 0.6931471805599453f;
                    const bool none = sum == 0.f;  // no token counts, whatever 0 times its value is
                    const float unit_v = none ? 0.f : c.v_scale / sum;
                    if (none) u = v = f32x4{0, 0, 0, 0};
                    *(u32x4 *)((uint32_t *)a.out + (to_row * D + 32 * j + 8 * g) / 2) =
                        u32x4{IO::pack(u[0] * unit_v, v[0] * unit_v), IO::pack(u[1] * unit_v, v[1] * unit_v),
                              IO::pack(u[2] * unit_v, v[2] * unit_v), IO::pack(u[3] * unit_v, v[3] * unit_v)};
                } else {
                    const int64_t to_row = (int64_t)kv_part_at(w.number, done.begins) * a.q_heads + at;
                    if (j == 0 && g == 0) *(float2 *)(a.part_ml + 2 * to_row) = make_float2(most, sum);
                    float *dst = a.part_o + to_row * D + 32 * j + 8 * g;
                    *(f32x4 *)dst = f32x4{u[0], v[0], u[1], v[1]};
                    *(f32x4 *)(dst + 4) = f32x4{u[2], v[2], u[3], v[3]};
                }
            }
        }
        if (done.last) return;
        __syncthreads();  // the arrays are the next part's from here
    }
}

// Joins the parts of entries that have more than one.  A row's numbers are dealt to
// D / 4 threads; a workgroup takes ROWS query heads of an entry with as many teams as
// are left over, each with some of the parts: one row where few are to be joined
// (they have the most parts), eight where many are (mostly to find that there is
// nothing to join: 3,584 workgroups that only leave take 5 us to start).
constexpr int kv_join_threads(int D, bool many) { return many || D < 128 ? 256 : 512; }

template <typename IO, int D, bool MANY>
__global__ void __launch_bounds__(kv_join_threads(D, MANY)) kv_join_kernel(KvAttend a) {
    constexpr int COLS = D / 4, SETS = kv_join_threads(D, MANY) / COLS, ROWS = MANY ? SETS : 1, TEAMS = SETS / ROWS;
    const int32_t per_entry = (a.q_heads + ROWS - 1) / ROWS;
    const int64_t entry = blockIdx.x / (unsigned)per_entry;
    const int32_t first = a.where[2 * entry], parts = a.where[2 * entry + 1];
    if (parts <= 1) return;
    const int col = (int)threadIdx.x % COLS, set = (int)threadIdx.x / COLS, team = set / ROWS;
    const int32_t row = (int32_t)(blockIdx.x % (unsigned)per_entry) * ROWS + set % ROWS;
    const bool in = team < TEAMS && row < a.q_heads;
    __shared__ f32x4 so[TEAMS][COLS];
    __shared__ float sm[TEAMS], sl[TEAMS];
    float m = -INFINITY, l = 0.f;
    f32x4 o{0, 0, 0, 0};
    if (in) {
        constexpr int UP = MANY ? 4 : 8;  // parts whose numbers are on their way at once
        for (int32_t k0 = team; k0 < parts; k0 += UP * TEAMS) {
            float2 ml[UP];
            f32x4 po[UP];
            float most = m;
#pragma unroll
            for (int i = 0; i < UP; ++i) {
                const int32_t k = k0 + i * TEAMS;
                const int64_t at = (int64_t)kv_part_next((uint32_t)first, (uint32_t)(k < parts ? k : k0)) * a.q_heads + row;
                ml[i] = *(const float2 *)(a.part_ml + 2 * at);
                po[i] = *(const f32x4 *)(a.part_o + at * D + 4 * col);
                if (k >= parts) ml[i] = make_float2(-INFINITY, 0.f);
            }
#pragma unroll
            for (int i = 0; i < UP; ++i) most = fmaxf(most, ml[i].x);
            const float base = most == -INFINITY ? 0.f : most, x = exp2_fast(m - base);
            m = most;
            l *= x;
            o *= x;
#pragma unroll
            for (int i = 0; i < UP; ++i) {
                if (k0 + i * TEAMS >= parts) break;
                const float y = exp2_fast(ml[i].x - base);
                l += ml[i].y * y;
                o += po[i] * y;
            }
        }
    }
    if (TEAMS > 1) {
        if (in && col == 0) sm[team] = m;
        __syncthreads();
        float most = -INFINITY;
#pragma unroll
        for (int k = 0; k < TEAMS; ++k) most = fmaxf(most, sm[k]);
        const float x = exp2_fast(m - (most == -INFINITY ? 0.f : most));
        m = most;
        l *= x;
        o *= x;
        if (in) {
            so[team][col] = o;
            if (col == 0) sl[team] = l;
        }
        __syncthreads();
        if (team) return;
#pragma unroll
        for (int k = 1; k < TEAMS; ++k) {
            l += sl[k];
            o += so[k][col];
        }
    }
    if (!in) return;
    const int64_t to_row = entry * a.q_heads + row;
    if (a.lse && col == 0) a.lse[to_row] = (m + log2f(l)) * 0.6931471805599453f;
    const bool none = l == 0.f;
    const float unit_v = none ? 0.f : a.c.v_scale / l;
    if (none) o = f32x4{0, 0, 0, 0};
    *(u32x2 *)((uint32_t *)a.out + (to_row * D + 4 * col) / 2) =
        u32x2{IO::pack(o[0] * unit_v, o[1] * unit_v), IO::pack(o[2] * unit_v, o[3] * unit_v)};
}

}  // namespace pr

#endif
