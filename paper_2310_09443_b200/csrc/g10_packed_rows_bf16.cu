// Attention over rows of 8-bit codes for more than 16 rows: bf16 queries.
#include "g10_cache_rows.cuh"

namespace g10 {

cudaError_t launch_packed_rows_bf16(const AttendArgs &a, const float2 *scales, const AttendShape &z, int code, cudaStream_t s)
{
    auto launch = [&](auto p) -> cudaError_t {
        static_cast<AttendArgs &>(p) = a;
        p.scales = scales;
        return attend::launch_wide_type<__nv_bfloat16>(p, z, s);
    };
    return code == G10_INT8 ? launch(PackedRowsArgs<Int8>()) : launch(PackedRowsArgs<E4m3>());
}

}  // namespace g10
