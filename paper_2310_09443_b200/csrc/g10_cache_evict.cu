// Which tokens leave the key-value cache, and the moves that close the gaps.
#include "g10_cache.cuh"

namespace g10 {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kMoveThreads = 256;

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

// One block per (sequence, head).  The budget-th largest number is found 8 bits at a time (the digit's counts over the slots that agree
// with what is known so far); then one walk over the slots in order says of each whether it is kept, and numbers movers and holes.
__global__ void __launch_bounds__(kPlanThreads) k_cache_plan(const EvictArgs a)
{
    __shared__ unsigned s_hist[256], s_known, s_left;
    __shared__ int3 s_warp[32];
    const int s = blockIdx.x / a.c.kv_heads, head = blockIdx.x % a.c.kv_heads;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    ull bad = 0;
    const int length = cache_length(a.c, s, bad);
    if (head == 0 && tid == 0 && a.new_lengths != nullptr) a.new_lengths[s] = min(length, a.budget);
    if (length <= a.budget) {
        if (tid == 0) a.counts[blockIdx.x] = 0;
        if (bad != 0) raise_status(a.c.status, bad);
        return;
    }
    const int seen = __ldg(&a.c.seen[s]);
    unsigned known = 0, left = (unsigned)a.budget;       // the number's upper digits; how many of those that agree are kept
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += kPlanThreads) s_hist[i] = 0;
        __syncthreads();
        for (int slot = tid; slot < length; slot += kPlanThreads) {
            const unsigned w = worth_at(a, s, head, slot, seen, bad);
            if (shift == 24 || (w >> (shift + 8)) == (known >> (shift + 8))) atomicAdd(&s_hist[(w >> shift) & 255u], 1u);
        }
        __syncthreads();
        if (warp == 0) {                                 // counts from the largest digit down: 8 digits a lane
            unsigned n = 0;
            for (int i = 0; i < 8; ++i) n += s_hist[255 - (lane * 8 + i)];
            unsigned upto = n;
            for (int o = 1; o < 32; o <<= 1) { const unsigned v = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += v; }
            unsigned above = upto - n;
            if (above < left && left <= upto) {
                int i = 0;
                while (above + s_hist[255 - (lane * 8 + i)] < left) { above += s_hist[255 - (lane * 8 + i)]; ++i; }
                s_known = known | (unsigned)(255 - (lane * 8 + i)) << shift;
                s_left = left - above;
            }
        }
        __syncthreads();
        known = s_known; left = s_left;
    }
    // `left` slots with exactly this number are kept, the first ones
    g10_cache_move *const moves = a.moves + (int64_t)blockIdx.x * a.budget;
    int equals = 0, movers = 0, holes = 0;
    for (int slot0 = 0; slot0 < length; slot0 += kPlanThreads) {
        const int slot = slot0 + tid;
        const unsigned w = slot < length ? worth_at(a, s, head, slot, seen, bad) : 0u;
        const bool equal = slot < length && w == known;
        const unsigned below = (1u << lane) - 1u;
        const unsigned eq = __ballot_sync(0xffffffffu, equal);
        if (lane == 0) s_warp[warp].x = __popc(eq);
        __syncthreads();
        int rank = equals + __popc(eq & below);
        for (int i = 0; i < 32; ++i) { const int n = s_warp[i].x; if (i < warp) rank += n; equals += n; }
        const bool kept = slot < length && (w > known || (equal && rank < (int)left));
        const bool mover = kept && slot >= a.budget, hole = slot < length && !kept && slot < a.budget;
        const unsigned mv = __ballot_sync(0xffffffffu, mover), ho = __ballot_sync(0xffffffffu, hole);
        if (lane == 0) { s_warp[warp].y = __popc(mv); s_warp[warp].z = __popc(ho); }
        __syncthreads();
        int at_mover = movers + __popc(mv & below), at_hole = holes + __popc(ho & below);
        for (int i = 0; i < 32; ++i) {
            const int y = s_warp[i].y, z = s_warp[i].z;
            if (i < warp) { at_mover += y; at_hole += z; }
            movers += y; holes += z;
        }
        if (mover) moves[at_mover].source = slot;
        if (hole) moves[at_hole].target = slot;
        __syncthreads();
    }
    if (tid == 0) a.counts[blockIdx.x] = movers;
    if (bad != 0) raise_status(a.c.status, bad);
}

// Moves: a warp per move, rows of k and v by 16 bytes a lane.
__global__ void __launch_bounds__(kMoveThreads) k_cache_evict(const EvictArgs a)
{
    const int item = blockIdx.y, s = item / a.c.kv_heads, head = item % a.c.kv_heads;
    const int lane = threadIdx.x & 31;
    ull bad = 0;
    const int length = cache_length(a.c, s, bad);
    int n = __ldg(&a.counts[item]);
    if (n < 0 || n > a.budget) { bad |= G10_DEV_BAD_MOVE; n = 0; }
    const int chunks = a.c.head_dim / 8;
    for (int r = blockIdx.x * (kMoveThreads / 32) + (threadIdx.x >> 5); r < n; r += gridDim.x * (kMoveThreads / 32)) {
        const g10_cache_move m = a.moves[(int64_t)item * a.budget + r];
        // (a source before the budget, or a target behind it, could be another move's)
        if (m.source < a.budget || m.source >= length || m.target < 0 || m.target >= a.budget) { bad |= G10_DEV_BAD_MOVE; continue; }
        const Spot source = cache_spot(a.c, s, m.source, bad), target = cache_spot(a.c, s, m.target, bad);
        if (source.page < 0 || target.page < 0) continue;
        const int64_t from = 16 * (int64_t)cache_row(a.c, source, head), to = 16 * (int64_t)cache_row(a.c, target, head);
        for (int i = lane; i < 2 * chunks; i += 32) {
            const char *const rows = i < chunks ? a.c.k : a.c.v;
            const int at = 16 * (i < chunks ? i : i - chunks);
            *(uint4 *)(const_cast<char *>(rows) + to + at) = *(const uint4 *)(rows + from + at);
        }
        if (lane == 0) {
            const int64_t x = cache_cell(a.c, source, head), y = cache_cell(a.c, target, head);
            if (a.c.scores != nullptr) a.c.scores[y] = a.c.scores[x];
            if (a.c.positions != nullptr) a.c.positions[y] = a.c.positions[x];
        }
    }
    if (bad != 0) raise_status(a.c.status, bad);
}

}  // namespace

cudaError_t launch_cache_plan(const EvictArgs &a, cudaStream_t s)
{
    k_cache_plan<<<(unsigned)(a.c.num_seqs * a.c.kv_heads), kPlanThreads, 0, s>>>(a); count_launch();
    return cudaGetLastError();
}

cudaError_t launch_cache_evict(const EvictArgs &a, cudaStream_t s)
{
    const int64_t items = (int64_t)a.c.num_seqs * a.c.kv_heads;
    const int64_t most = (a.budget + kMoveThreads / 32 - 1) / (kMoveThreads / 32), want = (148 * 8 + items - 1) / items;
    const unsigned x = (unsigned)(most < want ? most : want);
    // (gridDim.y ends at 65 535)
    for (int64_t i = 0; i < items; i += 65535 / a.c.kv_heads * a.c.kv_heads) {
        const int64_t n = items - i < 65535 / a.c.kv_heads * a.c.kv_heads ? items - i : 65535 / a.c.kv_heads * a.c.kv_heads;
        EvictArgs b = a;
        const int64_t seq = i / a.c.kv_heads;
        b.c.table += seq * a.c.table_stride; b.c.lengths += seq; b.moves += i * a.budget; b.counts += i;
        k_cache_evict<<<dim3(x, (unsigned)n), kMoveThreads, 0, s>>>(b); count_launch();
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace g10
