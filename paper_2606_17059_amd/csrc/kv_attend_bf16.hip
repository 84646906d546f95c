// kv_attend_bf16.hip -- the attention kernels (kv_attend.h) for bfloat16 queries and outputs.
#include "kv_attend_launch.h"

namespace pr {

hipError_t kv_launch_bf16(const KvAttend &a, bool e4m3, hipStream_t st) { return kv_launch<Bf16>(a, e4m3, st); }

}  // namespace pr
