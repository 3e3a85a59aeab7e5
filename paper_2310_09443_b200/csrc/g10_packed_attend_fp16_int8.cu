// Attention over rows of 8-bit codes: fp16 queries, int8 codes; and what does not go by the types.
#include "g10_packed_attend.cuh"

namespace g10 {

cudaError_t launch_packed_fp16_int8(const PackedArgs &a, const AttendShape &z, cudaStream_t s) { return attend::launch_packed_type<__half, Int8>(a, z, s); }

cudaError_t launch_packed_rows_bf16(const AttendArgs &a, const float2 *scales, const AttendShape &z, int code, cudaStream_t s);      // (g10_packed_rows_*.cu)
cudaError_t launch_packed_rows_fp16(const AttendArgs &a, const float2 *scales, const AttendShape &z, int code, cudaStream_t s);

AttendShape packed_shape(const CacheView &c, int rows, int new_tokens, int window, int sinks)
{
    AttendShape z = attend_shape(c, rows, new_tokens, window, sinks);
    const int groups = (c.head_dim + 31) / 32;
    if (z.block_rows <= 16) {
        z.padded_dim = 32 * (groups <= 2 ? 2 : groups <= 4 ? groups : groups <= 6 ? 6 : 8);
        if (z.items > 0) z.tiles = (z.tiles / z.items + 1) / 2 * 2 * z.items;    // (they may be taken two at a time)
    }
    return z;
}

cudaError_t launch_packed_attend(const AttendArgs &a, const float2 *scales, int dtype, int code, cudaStream_t s)
{
    const AttendShape z = packed_shape(a.c, a.rows, a.new_tokens, a.window, a.sinks);
    if (z.block_rows > 16) return dtype == G10_BF16 ? launch_packed_rows_bf16(a, scales, z, code, s) : launch_packed_rows_fp16(a, scales, z, code, s);
    PackedArgs p;
    static_cast<AttendArgs &>(p) = a;
    p.scales = scales;
    if (code == G10_INT8) return dtype == G10_BF16 ? launch_packed_bf16_int8(p, z, s) : launch_packed_fp16_int8(p, z, s);
    return dtype == G10_BF16 ? launch_packed_bf16_e4m3(p, z, s) : launch_packed_fp16_e4m3(p, z, s);
}

}  // namespace g10
