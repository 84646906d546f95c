// kv_launch.h -- what the KV cache's host code and its attention kernels share:
// argument structs and launches.
#ifndef PR_KV_LAUNCH_H
#define PR_KV_LAUNCH_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kv_layout.h"

namespace pr {

constexpr int kKvScan = 256;  // entries whose lengths every wave of an attention looks at itself

struct KvAttend {
    KvView c;
    const int32_t *slots;
    int64_t n;
    const void *q;
    int64_t q_stride;
    void *out;
    float *lse;
    int32_t *where;  // per entry: its first unit and its chunks (nullptr: no entry has two)
    int32_t *plan;   // see kv_planned_unit (nullptr: units are found from the lengths)
    float *part_o, *part_ml;
    int64_t layer;
    int32_t q_heads, group, row_groups, window;
    int32_t chunks, least;  // chunks a key head's tokens are cut into, and a chunk's least tokens
    int32_t units;          // chunks there may be at most
    float scale;            // with the keys' scale and log2 e
    bool q_aligned;
};

// Rows of query heads a workgroup takes, in sixteens: two share the keys and values
// that one would read twice; past 192 dimensions two rows' output does not fit the
// registers next to a tile.
constexpr int kv_rows(int group, int head_dim) { return group > 16 && head_dim <= 192 ? 2 : 1; }

hipError_t kv_launch_bf16(const KvAttend &a, bool e4m3, hipStream_t st);
hipError_t kv_launch_f16(const KvAttend &a, bool e4m3, hipStream_t st);

}  // namespace pr

#endif
