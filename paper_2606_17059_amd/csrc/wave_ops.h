// wave_ops.h -- small wavefront (64-lane) helpers shared by the kernels.
#ifndef PR_WAVE_OPS_H
#define PR_WAVE_OPS_H

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pr {

// Value of v in the wave's first active lane, as a wave-uniform scalar.
__device__ __forceinline__ int32_t uniform(int32_t v) { return __builtin_amdgcn_readfirstlane(v); }

// 64-bit value of v in lane src (src must be wave-uniform).
__device__ __forceinline__ uint64_t readlane64(uint64_t v, int src) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, src);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), src);
    return ((uint64_t)hi << 32) | lo;
}

// v of the lanes up to this one joined by op(a, b), whose neutral element is 0.
template <typename T, typename Op>
__device__ __forceinline__ T lanes_upto(T v, Op op) {
    static_assert(sizeof(T) == 4, "32-bit values");
    v = op(v, (T)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, true));  // the lane 1, 2, 4, 8 before,
    v = op(v, (T)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, true));  // in each 16
    v = op(v, (T)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, true));
    v = op(v, (T)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, true));
    v = op(v, (T)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false));  // the 16 before, into 2nd and 4th
    v = op(v, (T)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false));  // the first half, into the second
    return v;
}

// Sum of v over the lanes up to this one.
__device__ __forceinline__ int32_t lanes_upto(int32_t v) {
    return lanes_upto(v, [](int32_t a, int32_t b) { return a + b; });
}

}  // namespace pr

#endif
