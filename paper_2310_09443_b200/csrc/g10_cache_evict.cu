// Which tokens leave the key-value cache, and the moves that close the gaps.
#include "g10_cache.cuh"

namespace g10 {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWarps = kPlanThreads / 32;
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

__device__ __forceinline__ unsigned cluster_rank()
{
    unsigned r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() { asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// A word of another block's shared memory.
__device__ __forceinline__ unsigned read_of(const unsigned *p, unsigned rank)
{
    unsigned at, v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((unsigned)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}

// Sum of the words of the warps before this one (all of them, if `all`).
__device__ __forceinline__ int sum_before(const unsigned *s_warp, bool all)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    return (int)__reduce_add_sync(0xffffffffu, all || lane < warp ? s_warp[lane] : 0u);
}
static_assert(kPlanWarps == 32, "a lane for each warp's word");

// One cluster of blocks per (sequence, head); each has a run of the slots, and their numbers in shared memory (kKept; a run that is too long for it is
// read again for every pass).  The budget-th largest number is found in three digits, from the top: counts over the slots that agree with what is known
// so far, added up over the cluster, and the digit at which they reach the budget.  The first digit has 11 bits, sign, exponent and two
// more: with 8, nearly all scores of a head share a handful of counters.  Then every slot is known to be kept or not, and
// movers and holes are numbered by counting: within a warp by votes, over warps and blocks by prefix sums.
template <bool kKept>
__global__ void __launch_bounds__(kPlanThreads) k_cache_plan(const EvictArgs a, int blocks)
{
    constexpr int kDigits = 2048;
    __shared__ unsigned s_count[kDigits], s_sum[kDigits], s_warp[kPlanWarps], s_warp2[kPlanWarps], s_found[2], s_mine[3];
    extern __shared__ unsigned s_worth[];
    const int rank = (int)cluster_rank(), item = blockIdx.x / blocks, s = item / a.c.kv_heads, head = item % a.c.kv_heads;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    ull bad = 0;
    const int length = cache_length(a.c, s, bad);
    if (head == 0 && rank == 0 && tid == 0 && a.new_lengths != nullptr) a.new_lengths[s] = min(length, a.budget);
    if (length <= a.budget) {                            // (the whole cluster alike)
        if (rank == 0 && tid == 0) a.counts[item] = 0;
        if (bad != 0) raise_status(a.c.status, bad);
        return;
    }
    const int seen = __ldg(&a.c.seen[s]);
    const int each = (length + blocks - 1) / blocks, from = min(length, rank * each), n = min(length, from + each) - from;
    auto worth = [&](int i) -> unsigned { return kKept ? s_worth[i] : worth_at(a, s, head, from + i, seen, bad); };
    if (kKept) {
        for (int i0 = tid; i0 < n; i0 += 4 * kPlanThreads) {
            unsigned w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) w[q] = i0 + q * kPlanThreads < n ? worth_at(a, s, head, from + i0 + q * kPlanThreads, seen, bad) : 0u;
#pragma unroll
            for (int q = 0; q < 4; ++q) if (i0 + q * kPlanThreads < n) s_worth[i0 + q * kPlanThreads] = w[q];
        }
    }
    unsigned known = 0, left = (unsigned)a.budget;       // the number's upper digits; how many of those that agree are kept
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11, digits = 1 << bits;
        for (int i = tid; i < digits; i += kPlanThreads) s_count[i] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kPlanThreads) {
            const unsigned w = worth(i);
            if (pass == 0 || w >> (shift + bits) == known >> (shift + bits)) atomicAdd(&s_count[(w >> shift) & (digits - 1)], 1u);
        }
        // the cluster's counts: each block adds a part of the digits up, then all read all parts
        const unsigned *counts = s_count;
        __syncthreads();
        if (blocks > 1) {
            cluster_sync();
            const int part = digits / blocks;
            for (int i = tid; i < part; i += kPlanThreads) {
                unsigned sum = 0;
                for (int r = 0; r < blocks; ++r) sum += read_of(&s_count[rank * part + i], (unsigned)r);
                s_sum[rank * part + i] = sum;
            }
            cluster_sync();
            for (int i = tid; i < digits; i += kPlanThreads)
                if (i / part != rank) s_sum[i] = read_of(&s_sum[i], (unsigned)(i / part));
            counts = s_sum;
            __syncthreads();
        }
        // from the largest digit down: a few neighbours a thread
        const int few = digits / kPlanThreads, top = digits - 1 - tid * few;
        unsigned mine = 0;
        for (int i = 0; i < few; ++i) mine += counts[top - i];
        unsigned upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const unsigned v = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += v; }
        if (lane == 31) s_warp[warp] = upto;
        __syncthreads();
        upto += (unsigned)sum_before(s_warp, false);
        unsigned above = upto - mine;
        if (above < left && left <= upto) {
            int i = 0;
            while (above + counts[top - i] < left) { above += counts[top - i]; ++i; }
            s_found[0] = known | (unsigned)(top - i) << shift; s_found[1] = left - above;
        }
        __syncthreads();
        known = s_found[0]; left = s_found[1];
    }

    // ---- who is kept: more than the number, and the first `left` of those that have it ----
    const int run = (n + kPlanWarps - 1) / kPlanWarps, w0 = min(n, warp * run), w1 = min(n, w0 + run);      // the warp's slots
    const unsigned below = (1u << lane) - 1u;
    int equals = 0;                                      // with the number, in the warp's run
    for (int i0 = w0; i0 < w1; i0 += 32) {
        const int i = i0 + lane;
        const unsigned w = i < w1 ? worth(i) : 0u;
        equals += __popc(__ballot_sync(0xffffffffu, i < w1 && w == known));
    }
    if (lane == 0) s_warp[warp] = (unsigned)equals;
    __syncthreads();
    int rank_before = sum_before(s_warp, false);         // slots with the number before the warp's
    if (blocks > 1) {
        const int all = sum_before(s_warp, true);
        if (tid == 0) s_mine[0] = (unsigned)all;
        cluster_sync();
        rank_before += (int)__reduce_add_sync(0xffffffffu, lane < rank ? read_of(&s_mine[0], (unsigned)lane) : 0u);
    }
    __syncthreads();
    auto each_slot = [&](auto &&visit) {                 // visit(slot, kept, votes) for the warp's slots, in order
        int r = rank_before;
        for (int i0 = w0; i0 < w1; i0 += 32) {
            const int i = i0 + lane;
            const unsigned w = i < w1 ? worth(i) : 0u;
            const bool equal = i < w1 && w == known;
            const unsigned votes = __ballot_sync(0xffffffffu, equal);
            const bool kept = i < w1 && (w > known || (equal && r + __popc(votes & below) < (int)left));
            r += __popc(votes);
            visit(from + i, i < w1, kept);
        }
    };
    int movers = 0, holes = 0;
    each_slot([&](int slot, bool real, bool kept) {
        movers += __popc(__ballot_sync(0xffffffffu, kept && slot >= a.budget));
        holes += __popc(__ballot_sync(0xffffffffu, real && !kept && slot < a.budget));
    });
    if (lane == 0) { s_warp[warp] = (unsigned)movers; s_warp2[warp] = (unsigned)holes; }
    __syncthreads();
    int at_mover = sum_before(s_warp, false), at_hole = sum_before(s_warp2, false), all_movers = sum_before(s_warp, true);
    if (blocks > 1) {
        const int all_holes = sum_before(s_warp2, true);
        if (tid == 0) { s_mine[1] = (unsigned)all_movers; s_mine[2] = (unsigned)all_holes; }
        cluster_sync();
        const unsigned x = lane < blocks ? read_of(&s_mine[1], (unsigned)lane) : 0u, y = lane < rank ? read_of(&s_mine[2], (unsigned)lane) : 0u;
        at_mover += (int)__reduce_add_sync(0xffffffffu, lane < rank ? x : 0u);
        at_hole += (int)__reduce_add_sync(0xffffffffu, y);
        all_movers = (int)__reduce_add_sync(0xffffffffu, x);
        cluster_sync();                                  // (nobody leaves while its memory may still be read)
    }
    g10_cache_move *const moves = a.moves + (int64_t)item * a.budget;
    each_slot([&](int slot, bool real, bool kept) {
        const bool mover = kept && slot >= a.budget, hole = real && !kept && slot < a.budget;
        const unsigned mv = __ballot_sync(0xffffffffu, mover), ho = __ballot_sync(0xffffffffu, hole);
        if (mover) moves[at_mover + __popc(mv & below)].source = slot;
        if (hole) moves[at_hole + __popc(ho & below)].target = slot;
        at_mover += __popc(mv); at_hole += __popc(ho);
    });
    if (rank == 0 && tid == 0) a.counts[item] = all_movers;
    if (bad != 0) raise_status(a.c.status, bad);
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
    // Blocks for one (sequence, head): one does for 2048 slots (each thread two), more as long as all find room on the device at once.
    static int known[kMaxDevices], room[kMaxDevices];
    const void *const kernels[] = {(const void *)k_cache_plan<true>};
    const int most_bytes = dynamic_smem_room(kernels[0], room);
    if (most_bytes <= 0) return cudaErrorInvalidDevice;
    int most = largest_cluster(kernels, false, kPlanThreads, (size_t)most_bytes, known), blocks = 1;
    most = most > kPlanCluster ? kPlanCluster : most;
    while (2 * blocks <= most && a.c.capacity > 2048 * blocks && items * 2 * blocks <= 2 * 148) blocks *= 2;
    // (numbers that shared memory cannot take are worked out anew in each pass: some 50 000 slots a block)
    while (2 * blocks <= most && ((int64_t)a.c.capacity + blocks - 1) / blocks * 4 > most_bytes) blocks *= 2;
    const int64_t bytes = ((int64_t)a.c.capacity + blocks - 1) / blocks * 4;
    const bool kept = bytes <= most_bytes;
    const auto kernel = kept ? k_cache_plan<true> : k_cache_plan<false>;
    cudaError_t e = kept ? allow_launch((const void *)kernel, (size_t)most_bytes, blocks) : allow_launch((const void *)kernel, 0, blocks);
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)blocks; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(items * blocks)); cfg.blockDim = dim3(kPlanThreads); cfg.dynamicSmemBytes = kept ? (size_t)bytes : 0; cfg.stream = s;
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
