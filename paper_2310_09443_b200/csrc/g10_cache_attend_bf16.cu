// Attention over a bf16 cache.
#include "g10_cache_attend.cuh"

namespace g10 {
cudaError_t launch_cache_attend_bf16(const AttendArgs &a, const AttendShape &z, cudaStream_t s) { return attend::launch_type<__nv_bfloat16>(a, z, s); }
}  // namespace g10
