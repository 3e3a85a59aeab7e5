// Attention over a bf16 cache for many rows.
#include "g10_cache_rows.cuh"

namespace g10 {
cudaError_t launch_cache_rows_bf16(const AttendArgs &a, const AttendShape &z, cudaStream_t s) { return attend::launch_wide_type<__nv_bfloat16>(a, z, s); }
}  // namespace g10
