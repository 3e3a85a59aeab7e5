// Which tokens leave the key-value cache, and the moves that close the gaps.
#include "g10_cache.cuh"

namespace g10 {
namespace {

constexpr int kPlanCluster = 8;          // blocks that share one (sequence, head), at most (16 find room for few at a time: 35 -> 55 us for 16 of 65 537 slots)
constexpr int kMoveThreads = 256;
constexpr int kMoves = 8;                // a warp takes at a time

// A slot's rank among those of its head, as a number: what has to stay first, then by score; NaN last.  (Slots with equal numbers: the lower
// one first.)
__device__ __forceinline__ unsigned worth_of(const EvictArgs &a, float score, int position, int seen)
{
    if (position < a.sinks || (int64_t)position >= (int64_t)seen - a.recent) return 0xffffffffu;
    if (score != score) return 0u;
    const unsigned u = __float_as_uint(score + 0.0f);    // (-0 counts as 0)
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ unsigned worth_at(const EvictArgs &a, int s, int head, int slot, int seen, ull &bad)
{
    const Spot o = cache_spot(a.c, s, slot, bad);
    if (o.page < 0) return 0u;
    const int64_t cell = cache_cell(a.c, o, head);
    return worth_of(a, __ldg(&a.c.scores[cell]), a.c.positions != nullptr ? __ldg(&a.c.positions[cell]) : slot, seen);
}

__device__ __forceinline__ void add_to(unsigned *p, unsigned rank, unsigned v)
{
    unsigned at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((unsigned)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("red.shared::cluster.add.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory");
}

// Of a run of slots: with the number that decides before and behind the budget, with a larger one before and behind it, slots before it.
struct Census {
    int even_before, even_behind, over_before, over_behind, before;
};
// What becomes of it when `rank` slots with the number come before the run and the first `left` of all are kept: the run's own are kept in order.
__device__ __forceinline__ void settle(const Census &c, int rank, int left, int &movers, int &holes)
{
    const int kept = min(max(left - rank, 0), c.even_before + c.even_behind), kept_before = min(kept, c.even_before);
    movers = c.over_behind + kept - kept_before;
    holes = c.before - c.over_before - kept_before;
}

// One cluster of blocks per (sequence, head); each has a run of the slots, and their numbers in shared memory (kKept; a run that is too long for it is
// read again for every pass).  The budget-th largest number is found in three digits, from the top: counts over the slots that agree with what is known
// so far, and the digit at which they reach the budget.  A block adds its counts that are not zero to those of all blocks of the cluster, so that one
// meeting a digit does.  The first digit has 11 bits, sign, exponent and two more: with 8, nearly all scores of a head share a handful of
// counters.  Then every slot is known to be kept or not; movers and holes are numbered from a census of each warp's slots (votes) and
// prefix sums over warps and blocks.  A chain of short steps, bound by their meetings, not by the 8 bytes read per slot.
template <bool kKept, int kThreads>
__global__ void __launch_bounds__(kThreads) k_cache_plan(const EvictArgs a, int blocks)
{
    constexpr int kDigits = 2048, kCounts = 2 * kDigits + kDigits / 2, kWarps = kThreads / 32;
    __shared__ __align__(16) unsigned s_count[kCounts], s_sum[kCounts];            // of the three digits; the block's, the cluster's
    __shared__ unsigned s_warp[kWarps], s_found[2];
    __shared__ Census s_census[kWarps];
    __shared__ int s_mine[5];
    extern __shared__ unsigned s_worth[];
    const int rank = (int)cluster_rank(), item = blockIdx.x / blocks, s = item / a.c.kv_heads, head = item % a.c.kv_heads;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    ull bad = 0;
    const int length = cache_length(a.c, s, bad);
    const int seen = __ldg(&a.c.seen[s]);
    if (head == 0 && rank == 0 && tid == 0 && a.new_lengths != nullptr) a.new_lengths[s] = min(length, a.budget);
    if (length <= a.budget) {                            // (the whole cluster alike)
        if (rank == 0 && tid == 0) a.counts[item] = 0;
        if (bad != 0) raise_status(a.c.status, bad);
        return;
    }
    const int each = (length + blocks - 1) / blocks, from = min(length, rank * each), n = min(length, from + each) - from;
    auto worth = [&](int i) -> unsigned { return kKept ? s_worth[i] : worth_at(a, s, head, from + i, seen, bad); };
    for (int i = tid; i < kCounts / 4; i += kThreads) {
        ((uint4 *)s_count)[i] = make_uint4(0, 0, 0, 0);
        if (blocks > 1) ((uint4 *)s_sum)[i] = make_uint4(0, 0, 0, 0);
    }
    if (kKept) {
        // (no branch between the loads of a round: all pages are on the way together, then all scores)
        constexpr int kAhead = kThreads >= 512 ? 8 : 12;
        const int32_t *const table = a.c.table + (int64_t)s * a.c.table_stride;
        const bool any = a.c.num_pages > 0;
        for (int i0 = tid; i0 < n; i0 += kAhead * kThreads) {
            Spot o[kAhead];
            float score[kAhead];
            int position[kAhead];
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                const int slot = from + min(i0 + q * kThreads, n - 1), at = (int)(((ull)(unsigned)slot * a.c.page_mul) >> a.c.page_shift);
                o[q].page = __ldg(&table[at]); o[q].place = slot - at * a.c.page_size;
                position[q] = slot;
            }
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                const bool there = o[q].page >= 0 && o[q].page < (int)a.c.num_pages;
                const int64_t cell = there ? cache_cell(a.c, o[q], head) : 0;
                score[q] = any ? __ldg(&a.c.scores[cell]) : 0.0f;
                if (a.c.positions != nullptr && any) position[q] = __ldg(&a.c.positions[cell]);
                if (!there) { bad |= G10_DEV_BAD_PAGE; o[q].page = -1; }
            }
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
                if (i0 + q * kThreads < n) s_worth[i0 + q * kThreads] = o[q].page < 0 ? 0u : worth_of(a, score[q], position[q], seen);
        }
    }
    if (blocks > 1) cluster_sync();                      // (all have begun, and cleared their sums)
    else __syncthreads();
    unsigned known = 0, left = (unsigned)a.budget;       // the number's upper digits; how many of those that agree are kept
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11, digits = 1 << bits, few = digits / kThreads;
        unsigned *const count = s_count + pass * kDigits;
        for (int i = tid; i < n; i += kThreads) {
            const unsigned w = worth(i);
            if (pass == 0 || w >> (shift + bits) == known >> (shift + bits)) atomicAdd(&count[(w >> shift) & (digits - 1)], 1u);
        }
        __syncthreads();
        const unsigned *counts = count;
        if (blocks > 1) {
            for (int i = tid; i < digits; i += kThreads) {
                const unsigned v = count[i];
                if (v != 0) for (int r = 0; r < blocks; ++r) add_to(&s_sum[pass * kDigits + i], (unsigned)r, v);
            }
            cluster_sync();
            counts = s_sum + pass * kDigits;
        }
        // from the largest digit down: a few neighbours a thread (2, 4 or 8)
        const int lowest = digits - (tid + 1) * few;
        unsigned of_digit[8], mine = 0;
#pragma unroll
        for (int i = 0; i < few; i += 2) { const uint2 v = *(const uint2 *)&counts[lowest + i]; of_digit[i] = v.x; of_digit[i + 1] = v.y; mine += v.x + v.y; }
        unsigned upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const unsigned v = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += v; }
        if (lane == 31) s_warp[warp] = upto;
        __syncthreads();
        upto += __reduce_add_sync(0xffffffffu, lane < warp ? s_warp[lane] : 0u);
        unsigned above = upto - mine;
        if (above < left && left <= upto) {
            bool found = false;
#pragma unroll
            for (int i = few - 1; i >= 0; --i) {
                if (!found && above + of_digit[i] >= left) {
                    found = true;
                    s_found[0] = known | (unsigned)(lowest + i) << shift; s_found[1] = left - above;
                }
                above += of_digit[i];
            }
        }
        __syncthreads();
        known = s_found[0]; left = s_found[1];
    }

    // ---- who is kept: more than the number, and the first `left` of those that have it ----
    const int run = ((n + kWarps - 1) / kWarps + 31) & ~31, w0 = min(n, warp * run), w1 = min(n, w0 + run);        // the warp's slots
    const unsigned below = (1u << lane) - 1u;
    Census c{0, 0, 0, 0, min(max(a.budget - from - w0, 0), w1 - w0)};
    for (int i0 = w0; i0 < w1; i0 += 32) {
        const int i = i0 + lane;
        const unsigned w = i < w1 ? worth(i) : 0u, front = __ballot_sync(0xffffffffu, from + i < a.budget);
        const unsigned even = __ballot_sync(0xffffffffu, i < w1 && w == known), over = __ballot_sync(0xffffffffu, i < w1 && w > known);
        c.even_before += __popc(even & front); c.even_behind += __popc(even & ~front);
        c.over_before += __popc(over & front); c.over_behind += __popc(over & ~front);
    }
    if (lane == 0) s_census[warp] = c;
    __syncthreads();
    // (lane i looks after warp i, in every warp)
    const Census of = lane < kWarps ? s_census[lane] : Census{0, 0, 0, 0, 0};
    const int evens = of.even_before + of.even_behind;
    int evens_upto = evens;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(0xffffffffu, evens_upto, o); if (lane >= o) evens_upto += v; }
    int evens_before = 0, at_mover = 0, at_hole = 0, all_movers = 0;               // of the blocks before this one, and of all
    if (blocks > 1) {
        const int sums[5] = {(int)__reduce_add_sync(0xffffffffu, of.even_before), (int)__reduce_add_sync(0xffffffffu, of.even_behind),
                             (int)__reduce_add_sync(0xffffffffu, of.over_before), (int)__reduce_add_sync(0xffffffffu, of.over_behind),
                             (int)__reduce_add_sync(0xffffffffu, of.before)};
        if (tid == 0) {
#pragma unroll
            for (int q = 0; q < 5; ++q) s_mine[q] = sums[q];
        }
        cluster_sync();
        Census x{0, 0, 0, 0, 0};
        if (lane < blocks) {
            x.even_before = (int)read_of((const unsigned *)&s_mine[0], (unsigned)lane); x.even_behind = (int)read_of((const unsigned *)&s_mine[1], (unsigned)lane);
            x.over_before = (int)read_of((const unsigned *)&s_mine[2], (unsigned)lane); x.over_behind = (int)read_of((const unsigned *)&s_mine[3], (unsigned)lane);
            x.before = (int)read_of((const unsigned *)&s_mine[4], (unsigned)lane);
        }
        cluster_arrive();                                // (read: who waits for it, at the end, may leave)
        int upto = x.even_before + x.even_behind, movers, holes;
        const int own = upto;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += v; }
        settle(x, upto - own, (int)left, movers, holes);
        evens_before = (int)__reduce_add_sync(0xffffffffu, lane < rank ? own : 0);
        at_mover = (int)__reduce_add_sync(0xffffffffu, lane < rank ? movers : 0);
        at_hole = (int)__reduce_add_sync(0xffffffffu, lane < rank ? holes : 0);
        all_movers = (int)__reduce_add_sync(0xffffffffu, movers);
    }
    int movers, holes;
    settle(of, evens_before + evens_upto - evens, (int)left, movers, holes);
    at_mover += (int)__reduce_add_sync(0xffffffffu, lane < warp ? movers : 0);
    at_hole += (int)__reduce_add_sync(0xffffffffu, lane < warp ? holes : 0);
    if (blocks == 1) all_movers = (int)__reduce_add_sync(0xffffffffu, movers);
    int even_rank = evens_before + (int)__reduce_add_sync(0xffffffffu, lane < warp ? evens : 0);
    g10_cache_move *const moves = a.moves + (int64_t)item * a.budget;
    for (int i0 = w0; i0 < w1; i0 += 32) {
        const int i = i0 + lane, slot = from + i;
        const unsigned w = i < w1 ? worth(i) : 0u, even = __ballot_sync(0xffffffffu, i < w1 && w == known);
        const bool kept = i < w1 && (w > known || (w == known && even_rank + __popc(even & below) < (int)left));
        const unsigned mv = __ballot_sync(0xffffffffu, kept && slot >= a.budget), ho = __ballot_sync(0xffffffffu, i < w1 && !kept && slot < a.budget);
        // (in bounds whatever happens to the scores meanwhile)
        if ((mv >> lane & 1u) && at_mover + __popc(mv & below) < a.budget) moves[at_mover + __popc(mv & below)].source = slot;
        if ((ho >> lane & 1u) && at_hole + __popc(ho & below) < a.budget) moves[at_hole + __popc(ho & below)].target = slot;
        even_rank += __popc(even); at_mover += __popc(mv); at_hole += __popc(ho);
    }
    if (rank == 0 && tid == 0) a.counts[item] = all_movers;
    if (bad != 0) raise_status(a.c.status, bad);
    if (blocks > 1) cluster_wait();
}

// A warp takes kMoves moves at a time: a lane each looks source and target up and moves score and position, then the rows go, 16 bytes a lane, all
// 128 units under way before the first is stored.  Pure traffic: 4 * head_dim bytes read and written per move.
__global__ void __launch_bounds__(kMoveThreads, 5) k_cache_evict(const EvictArgs a, unsigned unit_mul)
{
    const int item = blockIdx.y, s = item / a.c.kv_heads, head = item % a.c.kv_heads;
    const int lane = threadIdx.x & 31;
    ull bad = 0;
    const int length = cache_length(a.c, s, bad);
    int n = __ldg(&a.counts[item]);
    if (n < 0 || n > a.budget) { bad |= G10_DEV_BAD_MOVE; n = 0; }
    const int units = a.c.head_dim / 4, half = units / 2;                          // 16-byte units of a move: half of k, half of v
    for (int r0 = (blockIdx.x * (kMoveThreads / 32) + (threadIdx.x >> 5)) * kMoves; r0 < n; r0 += gridDim.x * (kMoveThreads / 32) * kMoves) {
        unsigned row = 0xffffffffu;                      // lanes 0 .. 7: sources, 8 .. 15: targets
        int64_t cell = -1;
        if (lane < 2 * kMoves && r0 + (lane & (kMoves - 1)) < n) {
            const g10_cache_move m = a.moves[(int64_t)item * a.budget + r0 + (lane & (kMoves - 1))];
            // (a source before the budget, or a target behind it, could be another move's)
            if (m.source < a.budget || m.source >= length || m.target < 0 || m.target >= a.budget) bad |= G10_DEV_BAD_MOVE;
            else {
                const Spot o = cache_spot(a.c, s, lane < kMoves ? m.source : m.target, bad);
                if (o.page >= 0) { row = cache_row(a.c, o, head); cell = cache_cell(a.c, o, head); }
            }
        }
        const int64_t to_cell = __shfl_down_sync(0xffffffffu, cell, kMoves);
        if (lane < kMoves && cell >= 0 && to_cell >= 0) {
            if (a.c.scores != nullptr) a.c.scores[to_cell] = a.c.scores[cell];
            if (a.c.positions != nullptr) a.c.positions[to_cell] = a.c.positions[cell];
        }
        constexpr int kAhead = 4;
#pragma unroll 1
        for (int u0 = 0; u0 < kMoves * units; u0 += kAhead * 32) {
            uint4 x[kAhead];
            unsigned to[kAhead];                         // 16-byte units
            bool key[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int u = u0 + i * 32 + lane, move = min((int)(((unsigned)u * unit_mul) >> 20), kMoves - 1), unit = u - move * units;
                const unsigned source = __shfl_sync(0xffffffffu, row, move), target = __shfl_sync(0xffffffffu, row, kMoves + move);
                key[i] = unit < half;
                const unsigned at = (unsigned)(key[i] ? unit : unit - half);
                to[i] = 0xffffffffu;
                if (u < kMoves * units && source != 0xffffffffu && target != 0xffffffffu) {
                    x[i] = *(const uint4 *)((key[i] ? a.c.k : a.c.v) + 16 * ((int64_t)source + at));
                    to[i] = target + at;
                }
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) if (to[i] != 0xffffffffu) *(uint4 *)(const_cast<char *>(key[i] ? a.c.k : a.c.v) + 16 * (int64_t)to[i]) = x[i];
        }
    }
    if (bad != 0) raise_status(a.c.status, bad);
}

}  // namespace

cudaError_t launch_cache_plan(const EvictArgs &a, cudaStream_t s)
{
    const int64_t items = (int64_t)a.c.num_seqs * a.c.kv_heads;
    // Blocks for one (sequence, head): one does for 2048 slots, more as long as all find room on the device at once.
    static int known[kMaxDevices], room[kMaxDevices];
    const void *const kernels[] = {(const void *)k_cache_plan<true, 512>};
    const int most_bytes = dynamic_smem_room(kernels[0], room);
    if (most_bytes <= 0) return cudaErrorInvalidDevice;
    int most = largest_cluster(kernels, false, 512, (size_t)most_bytes, known), blocks = 1;
    most = most > kPlanCluster ? kPlanCluster : most;
    while (2 * blocks <= most && a.c.capacity > 2048 * blocks && items * 2 * blocks <= 2 * 148) blocks *= 2;
    // (numbers that shared memory cannot take are worked out anew in each pass: some 48 000 slots a block)
    while (2 * blocks <= most && ((int64_t)a.c.capacity + blocks - 1) / blocks * 4 > most_bytes) blocks *= 2;
    const int64_t slots = ((int64_t)a.c.capacity + blocks - 1) / blocks, bytes = slots * 4;
    const bool kept = bytes <= most_bytes;
    // (few threads meet sooner)
    const bool small = slots <= 4096;
    const auto kernel = !kept ? k_cache_plan<false, 512> : small ? k_cache_plan<true, 256> : k_cache_plan<true, 512>;
    cudaError_t e = allow_launch((const void *)kernel, kept ? (size_t)most_bytes : 0, blocks);
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)blocks; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(items * blocks)); cfg.blockDim = dim3(kept && small ? 256u : 512u); cfg.dynamicSmemBytes = kept ? (size_t)bytes : 0; cfg.stream = s;
    cfg.attrs = at; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a, blocks);
}

cudaError_t launch_cache_evict(const EvictArgs &a, cudaStream_t s)
{
    const int64_t items = (int64_t)a.c.num_seqs * a.c.kv_heads, step = 65535 / a.c.kv_heads * a.c.kv_heads;      // (gridDim.y ends at 65 535)
    const int64_t each = kMoveThreads / 32 * kMoves, most = (a.budget + each - 1) / each, want = (148 * 8 + items - 1) / items;
    const unsigned units = (unsigned)a.c.head_dim / 4, unit_mul = ((1u << 20) + units - 1) / units;              // (u / units, u < 512, is exact)
    for (int64_t i = 0; i < items; i += step) {
        const int64_t n = items - i < step ? items - i : step, seq = i / a.c.kv_heads;
        EvictArgs b = a;
        b.c.table += seq * a.c.table_stride; b.c.lengths += seq; b.moves += i * a.budget; b.counts += i;
        k_cache_evict<<<dim3((unsigned)(most < want ? most : want), (unsigned)n), kMoveThreads, 0, s>>>(b, unit_mul); count_launch();
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace g10
