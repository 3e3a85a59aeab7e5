// Attention of a batch behind a shared beginning: fp16, and the choice of the type.
#include "g10_cache_shared.cuh"

namespace g10 {

cudaError_t launch_cache_shared_fp16(const BeginArgs &begin, const RestArgs &rest, const int32_t *shared, cudaStream_t s)
{
    return attend::launch_shared<__half>(begin, rest, shared, s);
}

AttendShape begin_shape(const CacheView &c, int rows, int new_tokens)
{
    AttendShape z = attend_shape(c, rows, new_tokens, 0, 0);
    // (up to 128 rows are one operand, wider heads leave tensor memory for one: g10_cache_rows.cuh)
    if (rows <= attend::kWideRows || c.head_dim > 128) return z;
    const int64_t tiles = z.items > 0 ? z.tiles / z.items : 0;
    z.block_rows = attend::kBeginRows;
    z.row_blocks = (rows + z.block_rows - 1) / z.block_rows;
    z.items = (int64_t)c.num_seqs * c.kv_heads * z.row_blocks;
    z.tiles = z.items * tiles;
    z.pieces = z.items + attend::kMaxWideBlocks;
    return z;
}

cudaError_t launch_cache_shared_bf16(const BeginArgs &begin, const RestArgs &rest, const int32_t *shared, cudaStream_t s);
cudaError_t launch_cache_shared(const BeginArgs &begin, const RestArgs &rest, const int32_t *shared, int dtype, cudaStream_t s)
{
    return dtype == G10_BF16 ? launch_cache_shared_bf16(begin, rest, shared, s) : launch_cache_shared_fp16(begin, rest, shared, s);
}

}  // namespace g10
