// What the calls on the key-value cache share: the cache as the kernels see it, checked lengths and pages.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "g10_device.cuh"
#include "g10_internal.h"

namespace g10 {

// g10_cache with checked sizes; passed to kernels by value.
struct CacheView {
    const char *k, *v;                   // (written by append and evict through the same addresses)
    int64_t page_stride, slot_stride, head_stride;       // units of 16 bytes
    const int32_t *table;
    int64_t table_stride, num_pages;
    const int32_t *lengths, *seen;
    float *scores;
    int32_t *positions;
    ull *status;
    int num_seqs, kv_heads, head_dim, page_size, max_pages;
    int capacity;                        // max_pages * page_size
    unsigned page_mul, page_shift;       // slot / page_size = slot * page_mul >> page_shift
};

// Where a slot lies.
struct Spot {
    int page, place;                     // page -1: nowhere
};

// Slots that sequence s holds, as far as the table reaches.
__device__ __forceinline__ int cache_length(const CacheView &c, int s, ull &bad)
{
    const int n = __ldg(&c.lengths[s]);
    if (n < 0 || n > c.capacity) bad |= G10_DEV_BAD_LENGTH;
    return n < 0 ? 0 : min(n, c.capacity);
}
// New tokens of sequence s that count, never more than its slots.
__device__ __forceinline__ int cache_count(const int32_t *counts, int s, int new_tokens, int length, ull &bad)
{
    int n = new_tokens;
    if (counts != nullptr) {
        n = __ldg(&counts[s]);
        if (n < 0 || n > new_tokens) bad |= G10_DEV_BAD_LENGTH;
        n = n < 0 ? 0 : min(n, new_tokens);
    }
    return min(n, length);
}
// Page and place of a slot (0 <= slot < capacity).  With l = ceil(log2 page_size), page_mul = floor(2^(31 + l) / page_size) + 1: the product is too
// large by slot * e / (page_size * 2^(31 + l)), 0 < e <= page_size <= 2^l, which is less than 1 / page_size for slots below 2^31: the quotient is exact.
__device__ __forceinline__ Spot cache_spot(const CacheView &c, int s, int slot, ull &bad)
{
    const int at = (int)(((ull)(unsigned)slot * c.page_mul) >> c.page_shift);
    Spot o;
    o.page = __ldg(&c.table[(int64_t)s * c.table_stride + at]);
    o.place = slot - at * c.page_size;
    if (o.page < 0 || o.page >= (int)c.num_pages) { bad |= G10_DEV_BAD_PAGE; o.page = -1; }
    return o;
}
// Where a row of k and v begins, in units of 16 bytes (the host has checked that it fits).
__device__ __forceinline__ unsigned cache_row(const CacheView &c, const Spot &o, int head)
{
    return (unsigned)((int64_t)o.page * c.page_stride + (int64_t)o.place * c.slot_stride + (int64_t)head * c.head_stride);
}
// Entry of scores and positions.
__device__ __forceinline__ int64_t cache_cell(const CacheView &c, const Spot &o, int head)
{
    return ((int64_t)o.page * c.kv_heads + head) * c.page_size + o.place;
}

// ---- the blocks of a cluster ----
__device__ __forceinline__ unsigned cluster_rank()
{
    unsigned r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// Executed by warps as one, whatever came before.
__device__ __forceinline__ void cluster_arrive()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait()
{
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_sync() { cluster_arrive(); cluster_wait(); }
// A word of another block's shared memory.
__device__ __forceinline__ unsigned read_of(const unsigned *p, unsigned rank)
{
    unsigned at, v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((unsigned)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}

__device__ __forceinline__ float2 read_of(const float2 *p, unsigned rank)
{
    unsigned at;
    float2 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((unsigned)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ float4 read_of(const float4 *p, unsigned rank)
{
    unsigned at;
    float4 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((unsigned)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
    return v;
}

template <typename T>
struct Pair;
template <>
struct Pair<__nv_bfloat16> {
    static __device__ __forceinline__ unsigned pack(float a, float b)
    {
        const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
        return *(const unsigned *)&p;
    }
    static __device__ __forceinline__ float2 unpack(unsigned u) { return __bfloat1622float2(*(const __nv_bfloat162 *)&u); }
};
template <>
struct Pair<__half> {
    static __device__ __forceinline__ unsigned pack(float a, float b)
    {
        const __half2 p = __floats2half2_rn(a, b);
        return *(const unsigned *)&p;
    }
    static __device__ __forceinline__ float2 unpack(unsigned u) { return __half22float2(*(const __half2 *)&u); }
};

// Rows of the logits that are kept for a slot (up to 16), rounded up for wide accesses.
__host__ __device__ __forceinline__ int logit_rows(int rows) { return rows <= 2 ? rows : (rows + 3) & ~3; }

// ---- launchers ----
struct AppendArgs {
    CacheView c;
    const char *q, *k, *v;
    int64_t q_seq, q_token, q_head, k_seq, k_token, k_head, v_seq, v_token, v_head;
    char *q_out;
    const int32_t *counts;
    const char *q_weight, *k_weight;
    float eps, inv_dim;                  // (1 / head_dim)
    const float *cos_table, *sin_table;
    int64_t table_rows;
    int new_tokens, q_heads, rotary, interleaved;
    float *scales;                       // (rows of codes)
};
cudaError_t launch_cache_append(const AppendArgs &a, int dtype, cudaStream_t s);
cudaError_t launch_packed_append(const AppendArgs &a, int dtype, int code, cudaStream_t s);

// What the booking kernel has to know of a tile.
struct __align__(16) TileNote {
    int s, head, slot, length;           // sequence, key-value head, first slot, the sequence's slots (0: no tile has this number)
};
static_assert(sizeof(TileNote) == 16, "read at a time");
struct AttendArgs {
    CacheView c;
    const char *q;
    int64_t q_seq, q_token, q_head;
    const int32_t *counts;
    char *out;
    float *lse;
    float scale_log2;                    // scale * log2 e
    int new_tokens, q_heads, group, rows, window, sinks;
    int row_blocks;                      // blocks of rows per key-value head
    int64_t pieces;                      // (room for so many)
    float2 *ml;                          // [block rows][pieces] running maximum and sum of every piece
    float *part;                         // [pieces][block rows][padded head_dim] its sums, not divided yet
    float *logits;                       // [tiles][64][logit_rows] scaled by log2 e (null: weights are not booked, or for more than 16 rows)
    bool books;
    float *sums;                         // [items][block rows] lse of every row, to base 2
    TileNote *notes;                     // [tiles]
    int64_t *total;                      // number of tiles
#ifdef G10_TEST_HOOKS
    int mute;                            // which arrival the first block of the kernels for many rows keeps to itself (0: none)
#endif
};
// Attention of a batch behind a shared beginning, in two parts.
struct SharedArgs : AttendArgs {
    int32_t *shared;                     // [1] slots that are shared: whole tiles, checked
    int each;                            // new tokens of a sequence
    float2 *begin_ml;                    // [sequences][new tokens][query heads] maximum and sum over the beginning
    float *begin_o;                      // ... [head_dim] its sums, not divided
};
struct BeginArgs : SharedArgs {};        // the beginning: one sequence, whose tokens are all sequences'
struct RestArgs : SharedArgs {};         // what each sequence has behind it
// Sizes that the workspace goes by.
struct AttendShape {
    int row_blocks, block_rows, logit_rows, padded_dim;  // (logit_rows 0: the rows' kernels, which leave no logits)
    int64_t items, pieces, tiles;        // upper bounds for the sequences' capacity
};
AttendShape attend_shape(const CacheView &c, int rows, int new_tokens, int window, int sinks);
cudaError_t launch_cache_attend(const AttendArgs &a, int dtype, cudaStream_t s);
// shared: as the caller has it.  begin_shape: attend_shape for the beginning.
AttendShape begin_shape(const CacheView &c, int rows, int new_tokens);
cudaError_t launch_cache_shared(const BeginArgs &begin, const RestArgs &rest, const int32_t *shared, int dtype, cudaStream_t s);

struct EvictArgs {
    CacheView c;
    int budget, sinks, recent;
    g10_cache_move *moves;
    int32_t *counts, *new_lengths;
    int row_units;                       // 16-byte units of a row
    float2 *scales;                      // of rows of codes, or null
};
cudaError_t launch_cache_plan(const EvictArgs &a, cudaStream_t s);
cudaError_t launch_cache_evict(const EvictArgs &a, cudaStream_t s);

// ---- rows of 8-bit codes (the view's row strides and addresses as those of the other cache, in units of 16 bytes) ----
struct ReadArgs {
    CacheView c;
    const float2 *scales;
    char *k, *v;
    int64_t k_seq, k_token, k_head, v_seq, v_token, v_head;
    const int32_t *starts;
    int tokens;
};
cudaError_t launch_packed_read(const ReadArgs &a, int dtype, int code, cudaStream_t s);
AttendShape packed_shape(const CacheView &c, int rows, int new_tokens, int window, int sinks);
cudaError_t launch_packed_attend(const AttendArgs &a, const float2 *scales, int dtype, int code, cudaStream_t s);

}  // namespace g10
