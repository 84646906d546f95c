/*
 * A plain C11 client of the KV cache's calls (include/prefix_router.h): two
 * sequences that share a prefix are written, forked, extended, trimmed, moved
 * and attended to on the GPU.  Keys are 0, so that every weight is the same and
 * an output is the mean of the values: each is worked out by hand, and exact in
 * 16 bits.
 *
 * Exit status 0 on success; every failed check prints its line and the
 * library's last error.
 */
#include <hip/hip_runtime_api.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "prefix_router.h"

enum { DIM = 64, TOKENS = 16, PAGES = 5, SLOTS = 3, SLOT_PAGES = 2, HEADS = 2, ROWS = 22, MIB = 1 << 20 };

static int failures = 0;

#define CHECK(cond)                                                                   \
    do {                                                                              \
        if (!(cond)) {                                                                \
            fprintf(stderr, "check failed at line %d: %s (last error: %s)\n", __LINE__, \
                    #cond, pr_last_error());                                          \
            failures++;                                                               \
        }                                                                             \
    } while (0)

static void *device(const void *src, size_t bytes) {
    void *d = NULL;
    if (hipMalloc(&d, bytes) != hipSuccess) return NULL;
    if (src && hipMemcpy(d, src, bytes, hipMemcpyHostToDevice) != hipSuccess) return NULL;
    return d;
}

/* Half-precision bits of a number that is one exactly, 0 or in [2^-14, 65504]. */
static uint16_t half_of(float x) {
    int e;
    if (x == 0.f) return 0;
    const float m = frexpf(x, &e); /* x = m 2^e, m in [1/2, 1) */
    return (uint16_t)(((e + 14) << 10) + (int)((m * 2.f - 1.f) * 1024.f));
}

/* All of a sequence's outputs are `value`, its lse is log(tokens). */
static void attended(const pr_kv *c, int32_t slot, int32_t window, float value, int tokens, void *q, void *out,
                     float *lse, void *work, int64_t work_bytes) {
    uint16_t o[HEADS * DIM];
    float l[HEADS];
    int32_t *slots = device(&slot, sizeof slot);
    CHECK(slots != NULL);
    CHECK(pr_kv_attend(c, 0, slots, 1, q, HEADS * DIM, HEADS, PR_KV_F16, 0.125f, window, out, lse, work, work_bytes,
                       NULL) == PR_OK);
    CHECK(hipMemcpy(o, out, sizeof o, hipMemcpyDeviceToHost) == hipSuccess);
    CHECK(hipMemcpy(l, lse, sizeof l, hipMemcpyDeviceToHost) == hipSuccess);
    int same = 0;
    for (int i = 0; i < HEADS * DIM; ++i) same += o[i] == half_of(value);
    CHECK(same == HEADS * DIM);
    for (int h = 0; h < HEADS; ++h) CHECK(tokens ? fabsf(l[h] - logf((float)tokens)) < 1e-5f : l[h] == -INFINITY);
    CHECK(hipFree(slots) == hipSuccess);
}

int main(void) {
    pr_kv c;
    memset(&c, 0, sizeof c);
    c.dtype = PR_KV_F16;
    c.layers = c.kv_heads = 1;
    c.head_dim = DIM;
    c.page_tokens = TOKENS;
    c.num_pages = PAGES;
    c.num_slots = SLOTS;
    c.slot_pages = SLOT_PAGES;
    c.k_scale = c.v_scale = 1.f;
    c.k_page = c.v_page = DIM * TOKENS;
    c.k_layer = c.v_layer = DIM * TOKENS * PAGES;
    static uint16_t nan_bits[DIM * TOKENS * PAGES];
    memset(nan_bits, 0xff, sizeof nan_bits); /* what is never written reaches nothing */
    c.k = device(nan_bits, sizeof nan_bits);
    c.v = device(nan_bits, sizeof nan_bits);
    c.table = device(NULL, SLOTS * SLOT_PAGES * 4);
    c.lengths = device(NULL, SLOTS * 4);
    c.refs = device(NULL, PAGES * 4);
    c.free_pages = device(NULL, 8);
    c.skipped = device(NULL, 8);
    void *work = device(NULL, MIB);
    CHECK(c.k && c.v && c.table && c.lengths && c.refs && c.free_pages && c.skipped && work);
    if (failures) return 1;
    int64_t need = 0;
    CHECK(pr_kv_workspace(&c, PR_KV_WORK_EXTEND, 2, ROWS, &need) == PR_OK && need > 0 && need <= MIB);
    CHECK(pr_kv_workspace(&c, PR_KV_WORK_COMPACT, 0, 0, &need) == PR_OK && need > 0 && need <= MIB);
    CHECK(pr_kv_workspace(&c, PR_KV_WORK_ATTEND, 1, HEADS, &need) == PR_OK && need <= MIB);
    CHECK(pr_kv_workspace(&c, PR_KV_WORK_CHANGE, 1, 0, &need) == PR_OK && need == 0);
    CHECK(pr_kv_init(&c, NULL) == PR_OK);

    /* slot 0: 20 tokens whose values are 0, 1, ..., 19; then 2 of value 21 (slot 1's, below) */
    uint16_t k[ROWS * DIM], v[ROWS * DIM], q[HEADS * DIM];
    memset(k, 0, sizeof k);
    for (int t = 0; t < ROWS; ++t)
        for (int d = 0; d < DIM; ++d) v[t * DIM + d] = half_of(t < 20 ? (float)t : 21.f);
    for (int i = 0; i < HEADS * DIM; ++i) q[i] = half_of(1.f);
    const int32_t ids[3] = {0, 1, 10};
    const int64_t offsets[3] = {0, 20, 22};
    int32_t *zero = device(ids, sizeof ids), *place = device(NULL, ROWS * 4);
    int64_t *off = device(offsets, sizeof offsets);
    uint16_t *kd = device(k, sizeof k), *vd = device(v, sizeof v), *qd = device(q, sizeof q);
    void *out = device(NULL, HEADS * DIM * 2);
    float *lse = device(NULL, HEADS * 4);
    int32_t *moved = device(NULL, 8);
    CHECK(zero && place && off && kd && vd && qd && out && lse && moved);
    if (failures) return 1;
    CHECK(pr_kv_extend(&c, zero, off, 1, 20, place, work, MIB, NULL) == PR_OK);
    CHECK(pr_kv_write(&c, 0, place, kd, DIM, vd, DIM, 20, PR_KV_F16, NULL) == PR_OK);
    attended(&c, 0, 0, 9.5f, 20, qd, out, lse, work, MIB);
    attended(&c, 0, 3, 18.f, 3, qd, out, lse, work, MIB);
    attended(&c, 2, 0, 0.f, 0, qd, out, lse, work, MIB);

    /* slot 1: slot 0's first 10 tokens, then two of value 21 on a page of its own */
    CHECK(pr_kv_fork(&c, zero, zero + 1, zero + 2, 1, NULL, 0, NULL) == PR_OK);
    attended(&c, 1, 0, 4.5f, 10, qd, out, lse, work, MIB);
    const int64_t two[2] = {0, 2};
    CHECK(hipMemcpy(off, two, sizeof two, hipMemcpyHostToDevice) == hipSuccess);
    CHECK(pr_kv_extend(&c, zero + 1, off, 1, 2, place, work, MIB, NULL) == PR_OK);
    CHECK(pr_kv_write(&c, 0, place, kd, DIM, vd + 20 * DIM, DIM, 2, PR_KV_F16, NULL) == PR_OK);
    attended(&c, 1, 0, 7.25f, 12, qd, out, lse, work, MIB);
    attended(&c, 0, 0, 9.5f, 20, qd, out, lse, work, MIB);

    /* slot 0 is given up: its two pages become free, slot 1's moves to the first */
    CHECK(pr_kv_trim(&c, zero, NULL, 1, 1, NULL, 0, NULL) == PR_OK);
    CHECK(pr_kv_compact(&c, moved, work, MIB, NULL) == PR_OK);
    int32_t m[2], table[SLOTS * SLOT_PAGES], refs[PAGES];
    uint64_t bits;
    CHECK(hipMemcpy(m, moved, sizeof m, hipMemcpyDeviceToHost) == hipSuccess && m[0] == 1 && m[1] == 1);
    CHECK(hipMemcpy(table, c.table, sizeof table, hipMemcpyDeviceToHost) == hipSuccess);
    CHECK(hipMemcpy(refs, c.refs, sizeof refs, hipMemcpyDeviceToHost) == hipSuccess);
    CHECK(hipMemcpy(&bits, c.free_pages, 8, hipMemcpyDeviceToHost) == hipSuccess);
    CHECK(table[0] == -1 && table[1] == -1 && table[2] == 0 && table[3] == -1);
    CHECK(refs[0] == 1 && refs[1] == 0 && refs[2] == 0 && bits == 0x1e);
    attended(&c, 1, 0, 7.25f, 12, qd, out, lse, work, MIB);
    attended(&c, 0, 0, 0.f, 0, qd, out, lse, work, MIB);
    CHECK(pr_kv_check(&c, NULL) == PR_OK);

    /* a slot that is none is left out and counted */
    attended(&c, SLOTS, 0, 0.f, 0, qd, out, lse, work, MIB);
    CHECK(pr_kv_check(&c, NULL) == PR_EINVAL && strstr(pr_last_error(), "1 batch entries"));
    CHECK(pr_kv_check(&c, NULL) == PR_OK);
    printf("kv_check: %s\n", failures ? "failed" : "ok");
    return failures != 0;
}
