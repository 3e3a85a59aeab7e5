// Attention of a batch whose sequences begin alike, their pages of the beginning being the same.
//
// The maximum, the sum and the sums (m, l, o) of a row over its slots are those over the shared slots and those over the rest, joined (see g10_cache_attend.cuh).
// The shared slots are visible to every row, so all sequences' rows of a key-value head together are one operand: keys and values of the beginning are read
// once (or, for many rows, once for each 128 of them, out of the L2 cache) instead of once for each sequence, and with S sequences the products are S times as large
// beside them, which is work for the tensor cores.  To the kernels the beginning is one sequence with all sequences' new tokens; what they leave is (m, l, o) in
// 32 bits.  The rest of every sequence is attended as ever, from its first slot behind the beginning on, and joined with that where its result is written.
//
// Whole tiles of 64 slots count as shared; those behind the last of them are read for each sequence.
#pragma once
#include "g10_cache_rows.cuh"

namespace g10 {
namespace attend {

constexpr int kCheckThreads = 1024;

// Slots that are shared by all that have new tokens, at most as many as the caller says, in whole tiles.
static __global__ void __launch_bounds__(kCheckThreads) k_cache_shared(const RestArgs a, const int32_t *shared)
{
    __shared__ int s_least;
    const int said = __ldg(shared);
    ull bad = said < 0 ? G10_DEV_BAD_LENGTH : 0;
    int least = max(0, min(said, a.c.capacity));
    if (threadIdx.x == 0) s_least = least;
    __syncthreads();
    for (int s = threadIdx.x; s < a.c.num_seqs; s += kCheckThreads) {
        const int length = cache_length(a.c, s, bad), count = cache_count(a.counts, s, a.new_tokens, length, bad);
        if (count > 0 && length - count < said) { bad |= G10_DEV_BAD_LENGTH; least = min(least, length - count); }
    }
    atomicMin(&s_least, least);
    if (bad != 0) raise_status(a.c.status, bad);
    __syncthreads();
    if (threadIdx.x == 0) *a.shared = s_least / kTile * kTile;
}

template <typename T>
cudaError_t launch_shared(const BeginArgs &begin, const RestArgs &rest, const int32_t *shared, cudaStream_t s)
{
    k_cache_shared<<<1, kCheckThreads, 0, s>>>(rest, shared); count_launch();
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const AttendShape y = attend_shape(begin.c, begin.rows, begin.new_tokens, 0, 0), z = attend_shape(rest.c, rest.rows, rest.new_tokens, 0, 0);
    e = y.block_rows == kWideRows ? launch_wide_type<T>(begin, y, s) : launch_type<T>(begin, y, s);
    if (e != cudaSuccess) return e;
    return z.block_rows == kWideRows ? launch_wide_type<T>(rest, z, s) : launch_type<T>(rest, z, s);
}

}  // namespace attend

cudaError_t launch_cache_shared_fp16(const BeginArgs &begin, const RestArgs &rest, const int32_t *shared, cudaStream_t s);

}  // namespace g10
