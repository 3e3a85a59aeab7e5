// Attention over an fp16 cache, and what does not go by the type.
#include "g10_cache_attend.cuh"

namespace g10 {

cudaError_t launch_cache_attend_fp16(const AttendArgs &a, const AttendShape &z, cudaStream_t s) { return attend::launch_type<__half>(a, z, s); }

AttendShape attend_shape(const CacheView &c, int rows, int new_tokens, int window, int sinks)
{
    AttendShape z;
    const int steps = (c.head_dim + 15) / 16;
    const bool wide = rows > 16;                         // (what 16 rows of registers do not hold goes to tensor memory)
    z.padded_dim = wide ? (c.head_dim + 63) / 64 * 64 : 16 * (steps <= 4 ? 4 : steps <= 6 ? steps : steps <= 8 ? 8 : steps <= 12 ? 12 : 16);
    z.block_rows = rows <= 8 ? 8 : rows <= 16 ? 16 : 128;
    z.row_blocks = (rows + z.block_rows - 1) / z.block_rows;
    int64_t tiles = ((int64_t)c.capacity + attend::kTile - 1) / attend::kTile;
    if (window > 0) {
        const int64_t seen = ((int64_t)sinks + attend::kTile - 1) / attend::kTile + ((int64_t)window + new_tokens + attend::kTile - 2) / attend::kTile + 1;
        tiles = seen < tiles ? seen : tiles;
    }
    z.logit_rows = wide ? 0 : logit_rows(rows);
    const int64_t items = (int64_t)c.num_seqs * c.kv_heads * z.row_blocks;
    z.items = items;
    z.tiles = items * tiles;
    z.pieces = items + (wide ? attend::kMaxWideBlocks : attend::kMaxBlocks);
    return z;
}

cudaError_t launch_cache_attend(const AttendArgs &a, int dtype, cudaStream_t s)
{
    const AttendShape z = attend_shape(a.c, a.rows, a.new_tokens, a.window, a.sinks);
    if (z.block_rows == 128) return dtype == G10_BF16 ? launch_cache_rows_bf16(a, z, s) : launch_cache_rows_fp16(a, z, s);
    return dtype == G10_BF16 ? launch_cache_attend_bf16(a, z, s) : launch_cache_attend_fp16(a, z, s);
}

}  // namespace g10
