// kv_attend_launch.h -- which attention kernel (kv_attend.h) a call takes.
#ifndef PR_KV_ATTEND_LAUNCH_H
#define PR_KV_ATTEND_LAUNCH_H

#include "kv_attend.h"

namespace pr {

template <typename IO, bool E4M3, int D>
hipError_t kv_launch_dim(const KvAttend &a, hipStream_t st) {
    // whole eights of (unit, key head) pairs, see the kernel's first lines
    const int64_t pairs = ((int64_t)a.units * a.c.kv_heads + 7) / 8 * 8;
    const dim3 grid((unsigned)(pairs * a.row_groups)), block(64 * kKvWaves);
    const int rows = kv_rows(a.group, D);
    if (a.wide)
        kv_attend_kernel<IO, E4M3, D, 1, kKvWideWaves><<<grid, dim3(64 * kKvWideWaves), 0, st>>>(a);
    else if (rows == 1)
        kv_attend_kernel<IO, E4M3, D, 1, kKvWaves><<<grid, block, 0, st>>>(a);
    else if constexpr (kv_rows(17, D) == 2)
        kv_attend_kernel<IO, E4M3, D, 2, kKvWaves><<<grid, block, 0, st>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.where) return e;
    constexpr int kSets = kv_join_threads(D, true) / (D / 4);
    if (a.n * a.q_heads > kKvJoinMany)
        kv_join_kernel<IO, D, true><<<dim3((unsigned)(a.n * ((a.q_heads + kSets - 1) / kSets))), dim3(kv_join_threads(D, true)), 0, st>>>(a);
    else
        kv_join_kernel<IO, D, false><<<dim3((unsigned)(a.n * a.q_heads)), dim3(kv_join_threads(D, false)), 0, st>>>(a);
    return hipGetLastError();
}

template <typename IO, bool E4M3>
hipError_t kv_launch_type(const KvAttend &a, hipStream_t st) {
    switch (a.c.head_dim) {
        case 64: return kv_launch_dim<IO, E4M3, 64>(a, st);
        case 96: return kv_launch_dim<IO, E4M3, 96>(a, st);
        case 128: return kv_launch_dim<IO, E4M3, 128>(a, st);
        case 192: return kv_launch_dim<IO, E4M3, 192>(a, st);
        case 256: return kv_launch_dim<IO, E4M3, 256>(a, st);
        default: return hipErrorInvalidValue;
    }
}

template <typename IO>
hipError_t kv_launch(const KvAttend &a, bool e4m3, hipStream_t st) {
    return e4m3 ? kv_launch_type<IO, true>(a, st) : kv_launch_type<IO, false>(a, st);
}

}  // namespace pr

#endif
