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
    int32_t *where;  // per entry: its first part and their number (nullptr: no entry has two)
    int32_t *plan;   // see kv_planned_share (nullptr: shares are found from the lengths)
    float *part_o, *part_ml;
    int64_t layer;
    int32_t q_heads, group, row_groups, window;
    KvSplit split;          // of one key head's tokens
    int32_t units;          // shares there may be at most
    float scale;            // with the keys' scale and log2 e
    bool q_aligned;
    bool wide;  // one workgroup of many waves takes a sequence
};

// Sixteens of query heads ("rows") a workgroup takes: two share the keys and values
// that one would read twice, but past 128 dimensions two rows' output leaves room
// for one wave a SIMD, which loses more (48 rows of 192 dimensions, e4m3: 52 us with
// one, 72 with two, 58 with three).
constexpr int kv_rows(int group, int head_dim) { return group > 16 && head_dim <= 128 ? 2 : 1; }

// Waves a SIMD holds of the attention kernel, by its registers (and, of a workgroup
// of many waves, at least its own).  One for 256 dimensions in 16 bits: two would
// spill (64 sequences of 2,000 tokens, 4 key heads: 97 us with one, 119 with two).
constexpr int kv_resident(bool e4m3, int head_dim, int rows, int waves) {
    const int n = head_dim * rows;
    const int many = e4m3 ? (n <= 64 ? 5 : (n <= 128 ? 4 : (n <= 192 ? 3 : 2)))
                          : (n <= 64 ? 5 : (n <= 96 ? 4 : (n <= 128 ? 3 : (head_dim < 256 ? 2 : 1))));
    return waves == kKvWaves ? many : waves / 4;
}

constexpr int kKvJoinMany = 1024;  // rows from which a joining workgroup takes several

hipError_t kv_launch_bf16(const KvAttend &a, bool e4m3, hipStream_t st);
hipError_t kv_launch_f16(const KvAttend &a, bool e4m3, hipStream_t st);

}  // namespace pr

#endif
