// kvcache.hip -- the pr_kv calls of the C ABI (include/prefix_router.h): argument
// checks and launches.  Device side: kv_pages.h, and kv_attend.h compiled in
// kv_attend_bf16.hip and kv_attend_f16.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <utility>

#include "kv_launch.h"
#include "kv_pages.h"
#include "last_error.h"
#include "prefix_router.h"

namespace {

using pr::KvView;

pr_status fail(pr_status s, const char *msg) { return pr::set_last_error(s, msg); }
pr_status ok() { return pr::set_last_error(PR_OK, ""); }

pr_status launched(hipError_t e, const char *what) {
    if (e == hipSuccess) return ok();
    char msg[160];
    snprintf(msg, sizeof msg, "%s launch failed: %s", what, hipGetErrorString(e));
    return fail(PR_EDEVICE, msg);
}

// Makes the cache's device current for the duration of a call.
class DeviceScope {
   public:
    explicit DeviceScope(int device) : device_(device) {
        ok_ = hipGetDevice(&prev_) == hipSuccess && (prev_ == device || hipSetDevice(device) == hipSuccess);
    }
    ~DeviceScope() {
        if (ok_ && prev_ != device_) (void)hipSetDevice(prev_);
    }
    bool ok() const { return ok_; }

   private:
    int prev_ = -1, device_;
    bool ok_ = false;
};

constexpr int64_t kMostGrid = ((int64_t)1 << 32) / 256 - 1;  // workgroups of 256 threads in a launch
constexpr int64_t kMostEntries = ((int64_t)1 << 32) / pr::kKvPageThreads - 2;  // of a fork or trim, a workgroup each
constexpr int64_t kMostForks = 65536;  // every entry looks through all for its slots
constexpr int64_t kMostSpan = (int64_t)pr::kKvStep << 31;  // tokens of a batch's tables: their steps are counted in 32 bits
constexpr int64_t kMostRows = INT32_MAX;

int element_bytes(const pr_kv *c) { return c->dtype == PR_KV_E4M3 ? 1 : 2; }

// Whether of the blocks of `page` elements at i * a + j * b (0 <= i < na, 0 <= j < nb)
// two overlap.
bool overlap(int64_t page, int64_t a, int64_t na, int64_t b, int64_t nb) {
    if ((na > 1 && a < page) || (nb > 1 && b < page)) return true;
    if (na == 1 || nb == 1) return false;
    if (a > b) {
        std::swap(a, b);
        std::swap(na, nb);
    }
    // Each row of the smaller stride ends before the next begins, but for orders that
    // nothing has; there, the blocks next to each row's first are looked at.
    const __int128 row = (__int128)a * (na - 1) + page;
    for (int64_t j = 1; j < nb && (__int128)j * b < row; ++j) {
        const __int128 at = (__int128)j * b;
        const int64_t i = (int64_t)(at / a), past = (int64_t)(at % a);
        if ((i < na && past < page) || (i + 1 < na && a - past < page)) return true;
    }
    return false;
}

// nullptr if c describes a cache, else what is wrong with it.
const char *wrong(const pr_kv *c) {
    if (!c) return "pr_kv is NULL";
    if (c->dtype != PR_KV_BF16 && c->dtype != PR_KV_F16 && c->dtype != PR_KV_E4M3) return "dtype is none of PR_KV_*";
    if (c->device < 0) return "device is negative";
    if (c->layers < 1 || c->kv_heads < 1 || c->num_pages < 1 || c->num_slots < 1 || c->slot_pages < 1)
        return "layers, kv_heads, num_pages, num_slots and slot_pages must be at least 1";
    const int d = c->head_dim, t = c->page_tokens;
    if (d != 64 && d != 96 && d != 128 && d != 192 && d != 256) return "head_dim must be 64, 96, 128, 192 or 256";
    if (t != 16 && t != 32 && t != 64 && t != 128 && t != 256) return "page_tokens must be 16, 32, 64, 128 or 256";
    if ((int64_t)c->num_pages * t > INT32_MAX) return "num_pages * page_tokens must be below 2^31";
    if ((int64_t)c->slot_pages * t > pr::kKvMostTokens) return "slot_pages * page_tokens must be at most 2^30";
    if (!c->k || !c->v || !c->table || !c->lengths || !c->refs || !c->free_pages || !c->skipped)
        return "pr_kv has a NULL pointer";
    if (((uintptr_t)c->k | (uintptr_t)c->v) & 15) return "k and v must be 16-byte aligned";
    if ((int64_t)c->layers * c->kv_heads > (1 << 30)) return "layers * kv_heads must be at most 2^30";
    const int64_t unit = 16 / element_bytes(c), page = (int64_t)c->kv_heads * d * t;
    if (c->kv_heads > (1 << 20) || page * 2 > INT32_MAX) return "a page must be smaller than 2^31 bytes";
    for (const int64_t s : {c->k_layer, c->k_page, c->v_layer, c->v_page})
        if (s < 0 || s % unit) return "strides must be non-negative multiples of 16 bytes";
    auto extent = [&](int64_t layer, int64_t each) {
        return (__int128)layer * (c->layers - 1) + (__int128)each * (c->num_pages - 1);
    };
    if (std::max(extent(c->k_layer, c->k_page), extent(c->v_layer, c->v_page)) > ((int64_t)1 << 60))
        return "strides are too large";
    if (overlap(page, c->k_layer, c->layers, c->k_page, c->num_pages) ||
        overlap(page, c->v_layer, c->layers, c->v_page, c->num_pages))
        return "pages must not overlap";
    if (c->dtype == PR_KV_E4M3) {
        if (!(std::isfinite(c->k_scale) && c->k_scale > 0 && std::isfinite(c->v_scale) && c->v_scale > 0))
            return "k_scale and v_scale must be finite and positive";
    } else if (c->k_scale != 1.f || c->v_scale != 1.f) {
        return "k_scale and v_scale of a 16-bit cache must be 1";
    }
    return nullptr;
}

KvView view(const pr_kv *c) {
    KvView v{};
    v.k = c->k;
    v.v = c->v;
    v.k_layer = c->k_layer;
    v.k_page = c->k_page;
    v.v_layer = c->v_layer;
    v.v_page = c->v_page;
    v.table = c->table;
    v.lengths = c->lengths;
    v.refs = c->refs;
    v.free_pages = (unsigned long long *)c->free_pages;
    v.skipped = (unsigned long long *)c->skipped;
    v.layers = c->layers;
    v.kv_heads = c->kv_heads;
    v.head_dim = c->head_dim;
    v.page_shift = __builtin_ctz((unsigned)c->page_tokens);
    v.num_pages = c->num_pages;
    v.num_slots = c->num_slots;
    v.slot_pages = c->slot_pages;
    v.k_scale = c->k_scale;
    v.v_scale = c->v_scale;
    return v;
}

// Parts of a workspace, each 16-byte aligned.
struct Parts {
    char *base;
    int64_t bytes = 0;
    explicit Parts(void *p) : base((char *)p) {}
    template <typename T>
    T *take(int64_t count) {
        T *p = base ? (T *)(base + bytes) : nullptr;
        bytes += (count * (int64_t)sizeof(T) + 15) / 16 * 16;
        return p;
    }
};

// Room for the keys and values is at most what these rows can need, two pages an
// entry besides whole ones, and what there is.
int64_t pages_needed(const pr_kv *c, int64_t n, int64_t rows) {
    return std::min<int64_t>(c->num_pages, rows / c->page_tokens + 2 * n);
}

int64_t extend_parts(const pr_kv *c, int64_t n, int64_t rows, void *work, pr::KvExtend *x) {
    Parts p(work);
    x->most = pages_needed(c, n, rows);
    x->owner = p.take<int32_t>(c->num_slots);
    x->grant = p.take<pr::KvGrant>(n);
    x->rank = p.take<int32_t>(n);
    x->fresh = p.take<int32_t>(x->most);
    x->copies = p.take<int32_t>(n);
    x->count = p.take<int32_t>(2);
    return p.bytes;
}

// A fork or trim whose tables have kKvShared pages changes them in a second launch, if its
// grid can be had.  What sequences hold is not known here.  A fork and a trim, in one launch
// each and in two: 256 entries with all of 513 scattered pages 80 and 15 us, with 64 of
// them 15 and 13; 16 entries with 8,193 34 and 12, with 64 6 and 11.  Batches of less than
// 16 have one launch, as room for so many pages each is mostly not used: 2 entries with 64
// of 65,537 pages 6 and 13 us (but with all of them 236 and 18).
dim3 column_grid(const pr_kv *c, int64_t n) {
    return dim3((unsigned)((c->slot_pages + 63) / 64), (unsigned)((n + pr::kKvSharedEntries - 1) / pr::kKvSharedEntries));
}

int64_t change_parts(const pr_kv *c, int64_t n, void *work, pr::KvChange *x) {
    const dim3 grid = column_grid(c, n);
    if (n < 16 || n * c->slot_pages < pr::kKvShared || grid.y > 65535 || grid.x > kMostEntries) return 0;
    Parts p(work);
    x->columns = p.take<int2>(n);
    return p.bytes;
}

int64_t compact_parts(const pr_kv *c, void *work, pr::KvCompact *x) {
    Parts p(work);
    x->from = p.take<int32_t>(c->num_pages / 2 + 1);
    x->target = p.take<int32_t>(c->num_pages / 2 + 1);
    x->to = p.take<int32_t>(c->num_pages);
    x->count = p.take<int32_t>(2);
    return p.bytes;
}

constexpr int kComputeUnits = 256;

// How an attention is split, as far as that goes by the host's numbers, and its
// workspace.
int64_t attend_parts(const pr_kv *c, int64_t n, int32_t q_heads, int32_t window, void *work, pr::KvAttend *a) {
    const bool e4m3 = c->dtype == PR_KV_E4M3;
    const int32_t group = q_heads / c->kv_heads;
    int64_t span = (int64_t)c->slot_pages * c->page_tokens;
    if (window > 0) span = std::min<int64_t>(span, (int64_t)window + pr::kKvTile - 1);
    a->group = group;
    a->q_heads = q_heads;
    // Few sequences that cannot be long: a workgroup of many waves each, and nothing to
    // join.  That takes less than shares where a wave has a few tiles (one sequence of 611
    // tokens, 14 heads of 64: 5.4 us, in shares 8.1; of 1,000: 6.7 and 8.3; of 2,000: 10.7
    // and 8.3; 8 of 500 on 4 key heads of 256: 13.2 and 11.7), or where the workgroups fill
    // the GPU anyway (32 of 500 to 1,500 on 8 key heads of 128: 24.2, 30.0).
    const int64_t pairs = n * c->kv_heads * ((group + 15) / 16);
    const int32_t step = pr::kKvWideWaves * pr::kKvTile, few = c->head_dim <= 128 ? 4 : 1;
    a->wide = pairs <= kComputeUnits && span <= (pairs * 2 > kComputeUnits ? 8 : few) * step;
    const int32_t rows = a->wide ? 1 : pr::kv_rows(group, c->head_dim);
    a->row_groups = (group + 16 * rows - 1) / (16 * rows);
    const int32_t heads = c->kv_heads * a->row_groups;
    const int32_t beside = kComputeUnits * pr::kv_resident(e4m3, c->head_dim, rows, pr::kKvWaves);
    a->split.fill = (uint32_t)std::max(1, beside / heads);
    a->split.least = n * heads * 8 >= beside ? 4 : 2;
    const int64_t steps = (span + pr::kKvStep - 1) / pr::kKvStep;  // of a sequence, at most
    const bool split = !a->wide && steps > a->split.least;
    // shares across sequences are at most `fill`, shares that keep to them one more for each
    const int64_t most = a->split.fill + (n >= a->split.fill ? n : 0);
    const int64_t units = split ? std::min<int64_t>(n * steps, most) : n;
    a->units = (int32_t)std::min<int64_t>(units, INT32_MAX);
    a->where = a->plan = nullptr;
    a->part_ml = a->part_o = nullptr;
    if (!split) return 0;
    Parts p(work);
    const int64_t parts = pr::kv_parts_kept(n, units, a->split);
    a->where = p.take<int32_t>(2 * n);
    a->plan = n > pr::kKvScan ? p.take<int32_t>(3 * n + 3) : nullptr;
    a->part_ml = p.take<float>(parts * q_heads * 2);
    a->part_o = p.take<float>(parts * q_heads * c->head_dim);
    return p.bytes;
}

const char *wrong_work(const void *work, int64_t have, int64_t need) {
    if (need == 0) return nullptr;
    if (!work || have < need) return "workspace is smaller than pr_kv_workspace says";
    if ((uintptr_t)work & 15) return "workspace must be 16-byte aligned";
    return nullptr;
}

const char *wrong_io(const pr_kv *c, int32_t io) {
    if (io != PR_KV_BF16 && io != PR_KV_F16) return "io must be PR_KV_BF16 or PR_KV_F16";
    if (c->dtype != PR_KV_E4M3 && io != c->dtype) return "io must be the type of a 16-bit cache";
    return nullptr;
}

unsigned blocks(int64_t items, int64_t most) { return (unsigned)std::max<int64_t>(1, std::min((items + 255) / 256, most)); }

}  // namespace

extern "C" {

pr_status pr_kv_init(const pr_kv *c, void *hip_stream) {
    if (const char *w = wrong(c)) return fail(PR_EINVAL, w);
    DeviceScope ds(c->device);
    if (!ds.ok()) return fail(PR_EDEVICE, "cannot select the cache's device");
    const int64_t items = std::max<int64_t>((int64_t)c->num_slots * c->slot_pages, c->num_pages);
    pr::kv_init_kernel<<<blocks(items, 2048), 256, 0, (hipStream_t)hip_stream>>>(view(c));
    return launched(hipGetLastError(), "pr_kv_init");
}

pr_status pr_kv_workspace(const pr_kv *c, int32_t call, int64_t n, int64_t m, int64_t *bytes) {
    if (const char *w = wrong(c)) return fail(PR_EINVAL, w);
    if (!bytes) return fail(PR_EINVAL, "bytes is NULL");
    if (n < 0 || m < 0 || n > kMostRows || m > kMostRows) return fail(PR_EINVAL, "a count is negative or past 2^31 - 1");
    if (call == PR_KV_WORK_EXTEND) {
        pr::KvExtend x;
        *bytes = extend_parts(c, n, m, nullptr, &x);
    } else if (call == PR_KV_WORK_ATTEND) {
        if (m < 1 || m % c->kv_heads) return fail(PR_EINVAL, "q_heads must be a positive multiple of kv_heads");
        if (n * m > kMostGrid) return fail(PR_EINVAL, "the batch has too many entries and query heads");
        if (n * c->slot_pages * c->page_tokens >= kMostSpan) return fail(PR_EINVAL, "the batch may have too many tokens");
        pr::KvAttend a;
        *bytes = attend_parts(c, n, (int32_t)m, 0, nullptr, &a);
    } else if (call == PR_KV_WORK_CHANGE) {
        if (n > kMostEntries) return fail(PR_EINVAL, "n is past 2^22 - 2");
        pr::KvChange x;
        *bytes = change_parts(c, n, nullptr, &x);
    } else if (call == PR_KV_WORK_COMPACT) {
        pr::KvCompact x;
        *bytes = compact_parts(c, nullptr, &x);
    } else {
        return fail(PR_EINVAL, "call is none of PR_KV_WORK_*");
    }
    return ok();
}

pr_status pr_kv_extend(const pr_kv *c, const int32_t *slots, const int64_t *offsets, int64_t n, int64_t rows,
                       int32_t *place, void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (const char *w = wrong(c)) return fail(PR_EINVAL, w);
    if (n < 0 || rows < 0 || n > kMostRows || rows > kMostRows)
        return fail(PR_EINVAL, "a count is negative or past 2^31 - 1");
    if (n == 0 && rows == 0) return ok();
    if ((n > 0 && (!slots || !offsets)) || (rows > 0 && !place)) return fail(PR_EINVAL, "NULL device pointer");
    pr::KvExtend x{};
    if (const char *w = wrong_work(workspace, workspace_bytes, extend_parts(c, n, rows, workspace, &x)))
        return fail(PR_EINVAL, w);
    DeviceScope ds(c->device);
    if (!ds.ok()) return fail(PR_EDEVICE, "cannot select the cache's device");
    hipStream_t st = (hipStream_t)hip_stream;
    x.c = view(c);
    x.slots = slots;
    x.offsets = offsets;
    x.n = n;
    x.rows = rows;
    x.place = place;
    pr::kv_extend_plan_kernel<<<1, pr::kKvPlanThreads, 0, st>>>(x);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return launched(e, "pr_kv_extend");
    // a thread a row or new page; a wave a copied page's (layer, head, keys or values)
    const unsigned row_blocks = blocks(std::max(rows, x.most), 8192);
    const int64_t copies = std::min<int64_t>(n * c->layers, 1 << 20) * c->kv_heads * 2;
    const unsigned grid = row_blocks + (n > 0 ? (unsigned)std::min<int64_t>((copies + 3) / 4, 1024) : 0);
    if (c->dtype == PR_KV_E4M3) pr::kv_extend_place_kernel<uint8_t><<<grid, 256, 0, st>>>(x, row_blocks);
    else pr::kv_extend_place_kernel<uint16_t><<<grid, 256, 0, st>>>(x, row_blocks);
    return launched(hipGetLastError(), "pr_kv_extend");
}

pr_status pr_kv_write(const pr_kv *c, int32_t layer, const int32_t *place, const void *k_rows, int64_t k_stride,
                      const void *v_rows, int64_t v_stride, int64_t rows, int32_t io, void *hip_stream) {
    if (const char *w = wrong(c)) return fail(PR_EINVAL, w);
    if (layer < 0 || layer >= c->layers) return fail(PR_EINVAL, "layer out of range");
    if (const char *w = wrong_io(c, io)) return fail(PR_EINVAL, w);
    if (rows < 0 || rows > kMostRows) return fail(PR_EINVAL, "rows is negative or past 2^31 - 1");
    if (rows == 0) return ok();
    if (!place || !k_rows || !v_rows) return fail(PR_EINVAL, "NULL device pointer");
    if (((uintptr_t)k_rows | (uintptr_t)v_rows) & 1) return fail(PR_EINVAL, "rows must be 2-byte aligned");
    const int64_t width = (int64_t)c->kv_heads * c->head_dim;
    if (rows > 1 && (k_stride < width || v_stride < width)) return fail(PR_EINVAL, "rows must not overlap");
    DeviceScope ds(c->device);
    if (!ds.ok()) return fail(PR_EDEVICE, "cannot select the cache's device");
    const bool aligned = !((((uintptr_t)k_rows | (uintptr_t)v_rows) & 15) || (rows > 1 && (k_stride | v_stride) & 7));
    auto unit = [](float scale) {
        const int e = std::min(std::max(std::ilogb(scale), -126), 126);  // both powers are floats
        const float u = std::ldexp(scale, -e);
        return pr::KvUnit{std::ldexp(1.f, -e), u, 1.f / u};
    };
    const pr::KvRows x{view(c), place, k_rows, v_rows, k_stride, v_stride, rows, layer, aligned, unit(c->k_scale), unit(c->v_scale)};
    hipStream_t st = (hipStream_t)hip_stream;
    const unsigned grid = (blocks((rows + 7) / 8 * ((width + 63) / 64) * 64, kMostGrid - 7) + 7) / 8 * 8;
    if (c->dtype != PR_KV_E4M3) pr::kv_write_kernel<pr::KvSame><<<grid, 256, 0, st>>>(x);
    else if (io == PR_KV_BF16) pr::kv_write_kernel<pr::KvE4m3<true>><<<grid, 256, 0, st>>>(x);
    else pr::kv_write_kernel<pr::KvE4m3<false>><<<grid, 256, 0, st>>>(x);
    return launched(hipGetLastError(), "pr_kv_write");
}

pr_status pr_kv_attend(const pr_kv *c, int32_t layer, const int32_t *slots, int64_t n, const void *q,
                       int64_t q_stride, int32_t q_heads, int32_t io, float scale, int32_t window, void *out,
                       float *lse, void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (const char *w = wrong(c)) return fail(PR_EINVAL, w);
    if (layer < 0 || layer >= c->layers) return fail(PR_EINVAL, "layer out of range");
    if (const char *w = wrong_io(c, io)) return fail(PR_EINVAL, w);
    if (q_heads < 1 || q_heads % c->kv_heads) return fail(PR_EINVAL, "q_heads must be a positive multiple of kv_heads");
    if (window < 0) return fail(PR_EINVAL, "window is negative");
    if (!std::isfinite(scale)) return fail(PR_EINVAL, "scale must be finite");
    if (n < 0) return fail(PR_EINVAL, "n is negative");
    if (n > kMostGrid / q_heads) return fail(PR_EINVAL, "the batch has too many entries and query heads");
    if (n * c->slot_pages * c->page_tokens >= kMostSpan) return fail(PR_EINVAL, "the batch may have too many tokens");
    if (n == 0) return ok();
    if (!slots || !q || !out) return fail(PR_EINVAL, "NULL device pointer");
    if ((uintptr_t)q & 1) return fail(PR_EINVAL, "q must be 2-byte aligned");
    if ((uintptr_t)out & 15) return fail(PR_EINVAL, "out must be 16-byte aligned");
    const int64_t width = (int64_t)q_heads * c->head_dim;
    if (n > 1 && q_stride < width) return fail(PR_EINVAL, "rows of q must not overlap");
    // workgroups read a query after others have written their part of the output
    if ((uintptr_t)out < (uintptr_t)q + 2 * ((n - 1) * q_stride + width) &&
        (uintptr_t)q < (uintptr_t)out + 2 * n * width)
        return fail(PR_EINVAL, "out must not overlap q");
    pr::KvAttend a{};
    if (const char *w = wrong_work(workspace, workspace_bytes, attend_parts(c, n, q_heads, window, workspace, &a)))
        return fail(PR_EINVAL, w);
    a.c = view(c);
    a.slots = slots;
    a.n = n;
    a.q = q;
    a.q_stride = q_stride;
    a.out = out;
    a.lse = lse;
    a.layer = layer;
    a.window = window;
    a.scale = (float)((double)scale * c->k_scale * 1.4426950408889634);
    if (!std::isfinite(a.scale)) return fail(PR_EINVAL, "scale times k_scale must be finite");
    a.q_aligned = !((uintptr_t)q & 15) && (n == 1 || !(q_stride & 7));
    if (((int64_t)a.units * c->kv_heads + 7) / 8 * 8 * a.row_groups > kMostGrid)
        return fail(PR_EINVAL, "the batch has too many entries and key heads");
    DeviceScope ds(c->device);
    if (!ds.ok()) return fail(PR_EDEVICE, "cannot select the cache's device");
    hipStream_t st = (hipStream_t)hip_stream;
    if (a.plan) {
        pr::kv_plan_kernel<<<1, pr::kKvPlanThreads, 0, st>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return launched(e, "pr_kv_attend");
    }
    const bool e4m3 = c->dtype == PR_KV_E4M3;
    return launched(io == PR_KV_BF16 ? pr::kv_launch_bf16(a, e4m3, st) : pr::kv_launch_f16(a, e4m3, st),
                    "pr_kv_attend");
}

pr_status pr_kv_fork(const pr_kv *c, const int32_t *src, const int32_t *dst, const int32_t *tokens, int64_t n,
                     void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (const char *w = wrong(c)) return fail(PR_EINVAL, w);
    if (n < 0 || n > kMostForks) return fail(PR_EINVAL, "n is negative or past 65536");
    if (n == 0) return ok();
    if (!src || !dst || !tokens) return fail(PR_EINVAL, "NULL device pointer");
    pr::KvChange x{view(c), src, dst, tokens, 1, n, nullptr};
    if (const char *w = wrong_work(workspace, workspace_bytes, change_parts(c, n, workspace, &x)))
        return fail(PR_EINVAL, w);
    DeviceScope ds(c->device);
    if (!ds.ok()) return fail(PR_EDEVICE, "cannot select the cache's device");
    hipStream_t st = (hipStream_t)hip_stream;
    pr::kv_fork_kernel<<<(unsigned)n, pr::kKvPageThreads, 0, st>>>(x);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && x.columns) {
        pr::kv_change_columns_kernel<true><<<column_grid(c, n), pr::kKvPageThreads, 0, st>>>(x);
        e = hipGetLastError();
    }
    return launched(e, "pr_kv_fork");
}

pr_status pr_kv_trim(const pr_kv *c, const int32_t *slots, const int32_t *keep, int64_t keep_stride, int64_t n,
                     void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (const char *w = wrong(c)) return fail(PR_EINVAL, w);
    if (n < 0 || n > kMostEntries) return fail(PR_EINVAL, "n is negative or past 2^22 - 2");
    if (keep && keep_stride < 0) return fail(PR_EINVAL, "keep_stride is negative");
    if (n == 0) return ok();
    if (!slots) return fail(PR_EINVAL, "NULL device pointer");
    pr::KvChange x{view(c), nullptr, slots, keep, keep_stride, n, nullptr};
    if (const char *w = wrong_work(workspace, workspace_bytes, change_parts(c, n, workspace, &x)))
        return fail(PR_EINVAL, w);
    DeviceScope ds(c->device);
    if (!ds.ok()) return fail(PR_EDEVICE, "cannot select the cache's device");
    hipStream_t st = (hipStream_t)hip_stream;
    pr::kv_trim_kernel<<<(unsigned)n, pr::kKvPageThreads, 0, st>>>(x);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && x.columns) {
        pr::kv_change_columns_kernel<false><<<column_grid(c, n), pr::kKvPageThreads, 0, st>>>(x);
        e = hipGetLastError();
    }
    return launched(e, "pr_kv_trim");
}

pr_status pr_kv_compact(const pr_kv *c, int32_t *moved, void *workspace, int64_t workspace_bytes,
                        void *hip_stream) {
    if (const char *w = wrong(c)) return fail(PR_EINVAL, w);
    pr::KvCompact x{};
    if (const char *w = wrong_work(workspace, workspace_bytes, compact_parts(c, workspace, &x)))
        return fail(PR_EINVAL, w);
    DeviceScope ds(c->device);
    if (!ds.ok()) return fail(PR_EDEVICE, "cannot select the cache's device");
    hipStream_t st = (hipStream_t)hip_stream;
    x.c = view(c);
    x.moved = moved;
    pr::kv_compact_plan_kernel<<<1, pr::kKvPlanThreads, 0, st>>>(x);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return launched(e, "pr_kv_compact");
    const int64_t items = std::max<int64_t>((int64_t)c->num_slots * c->slot_pages,
                                            (int64_t)(c->num_pages / 2) * c->layers * 2 * 256);
    pr::kv_compact_move_kernel<<<blocks(items, 2048), 256, 0, st>>>(x, element_bytes(c));
    return launched(hipGetLastError(), "pr_kv_compact");
}

pr_status pr_kv_check(const pr_kv *c, void *hip_stream) {
    if (const char *w = wrong(c)) return fail(PR_EINVAL, w);
    DeviceScope ds(c->device);
    if (!ds.ok()) return fail(PR_EDEVICE, "cannot select the cache's device");
    hipStream_t st = (hipStream_t)hip_stream;
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(st, &cap) != hipSuccess) return fail(PR_EDEVICE, "hipStreamIsCapturing failed");
    if (cap != hipStreamCaptureStatusNone) return fail(PR_ESTATE, "pr_kv_check waits: not under graph capture");
    int64_t skipped = 0;
    if (hipMemcpyAsync(&skipped, c->skipped, sizeof skipped, hipMemcpyDeviceToHost, st) != hipSuccess ||
        hipStreamSynchronize(st) != hipSuccess)
        return fail(PR_EDEVICE, "reading the skipped entries failed");
    if (skipped == 0) return ok();
    // what attentions on other streams count meanwhile stays for the next check
    pr::kv_reported_kernel<<<1, 1, 0, st>>>((unsigned long long *)c->skipped, (unsigned long long)skipped);
    if (hipGetLastError() != hipSuccess || hipStreamSynchronize(st) != hipSuccess)
        return fail(PR_EDEVICE, "resetting the skipped entries failed");
    char msg[96];
    snprintf(msg, sizeof msg, "%lld batch entries were skipped", (long long)skipped);
    return fail(PR_EINVAL, msg);
}

}  // extern "C"
