// Attention of new tokens over the paged key-value cache, and the booking of the weights.
//
// For a row (one query head of one new token) and the slots j that it sees: s_j = scale <q, k_j>, m = max s_j, l = sum exp(s_j - m),
// o = sum exp(s_j - m) v_j; out = o / l.  (m, l, o) over any part of the slots can be joined: m = max m_i,
// l = sum l_i exp(m_i - m), o likewise.  Each key and value is read once, for all rows of its key-value head together; with one new token
// that is 4 * group operations per byte or less, so the bound is the memory's bandwidth and every SM has to load all the time.
//
// Work is cut into tiles of 64 slots.  The tiles of all (sequence, head, block of rows) items, one after the other, are shared out
// evenly over the blocks of the grid, whatever the lengths: a block's share is a run of tiles that may begin and end inside an item.
// A run inside one item is a piece; piece number = item + block, which no two pieces share, since along the run one of the two
// always grows.  A piece that is a whole item gives the answer; of the others (m, l, o) are joined by the second kernel.
//
// The weights w_j = exp(s_j - lse) that the cache books need lse, which nobody knows before the last piece is done.  So the first kernel
// leaves s_j (4 bytes a row, beside 4 * head_dim bytes of key and value), and the third adds the weights up: up to four lanes a slot, each over four rows,
// joined in a fixed order and added to the score once, the same every time.
//
// This file is for up to 16 rows per key-value head (new tokens times heads of the group), one block of rows each; more are g10_cache_rows.cuh's, which has the
// sharing out of tiles and the second kernel from here.
#pragma once
#include <type_traits>

#include "g10_cache.cuh"

namespace g10 {
namespace attend {

constexpr int kTile = 64;                // slots
constexpr int kMaxBlocks = 148 * 8;      // of the grid; the workspace has room for their pieces
constexpr int kMaxWideBlocks = 148 * 4;  // ... with 128 rows each
constexpr int kJoinThreads = 256;

__device__ __forceinline__ unsigned smem_of(const void *p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void ldsm4(unsigned (&r)[4], unsigned at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm4t(unsigned (&r)[4], unsigned at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
template <typename T>
__device__ __forceinline__ void mma(float (&d)[4], const unsigned (&a)[4], unsigned b0, unsigned b1);
template <>
__device__ __forceinline__ void mma<__nv_bfloat16>(float (&d)[4], const unsigned (&a)[4], unsigned b0, unsigned b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma<__half>(float (&d)[4], const unsigned (&a)[4], unsigned b0, unsigned b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_of(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A sequence as the call sees it: its new tokens and the tiles that some row sees.
struct Seq {
    int length, count;       // slots, new tokens
    int tiles, head_tiles;   // tiles in all; the first so many hold the first slots (sinks)
    int skipped;             // tiles between those and the window
};
__device__ __forceinline__ Seq seq_of(const AttendArgs &a, int s, ull &bad)
{
    Seq q;
    q.length = cache_length(a.c, s, bad);
    q.count = cache_count(a.counts, s, a.new_tokens, q.length, bad);
    const int all = (q.length + kTile - 1) / kTile;
    q.tiles = all; q.head_tiles = 0; q.skipped = 0;
    if (a.window > 0) {
        const int first = max(0, q.length - q.count - a.window + 1) / kTile;      // (the first row's window reaches furthest back)
        q.head_tiles = min((int)(((int64_t)min(a.sinks, q.length) + kTile - 1) / kTile), first);
        q.skipped = first - q.head_tiles;
        q.tiles = all - q.skipped;
    }
    if (q.count == 0) q.tiles = 0;
    return q;
}
// Behind a shared beginning (whole tiles of it, and less than a sequence with new tokens holds without them).
__device__ __forceinline__ Seq seq_of(const BeginArgs &a, int, ull &)
{
    Seq q;
    q.length = __ldcg(a.shared); q.count = a.new_tokens;
    q.tiles = q.length / kTile; q.head_tiles = 0; q.skipped = 0;
    return q;
}
__device__ __forceinline__ Seq seq_of(const RestArgs &a, int s, ull &bad)
{
    Seq q;
    q.length = cache_length(a.c, s, bad);
    q.count = cache_count(a.counts, s, a.new_tokens, q.length, bad);
    q.head_tiles = 0; q.skipped = __ldcg(a.shared) / kTile;
    q.tiles = q.count == 0 ? 0 : (q.length + kTile - 1) / kTile - q.skipped;
    return q;
}
// The queries of a sequence's token t, head 0.
__device__ __forceinline__ const char *queries_of(const AttendArgs &a, int s, int t) { return a.q + 2 * (s * a.q_seq + t * a.q_token); }
__device__ __forceinline__ const char *queries_of(const BeginArgs &a, int, int t)
{
    const int s = t / a.each;
    return a.q + 2 * (s * a.q_seq + (t - s * a.each) * a.q_token);
}
// Last slot that token t sees.
template <typename Args>
__device__ __forceinline__ int stands_at(const Args &, const Seq &q, int t) { return std::is_same<Args, BeginArgs>::value ? q.length - 1 : q.length - q.count + t; }
// Slots from here on are not seen by the first token.
template <typename Args>
__device__ __forceinline__ int seen_by_all(const Args &a, const Seq &q) { return stands_at(a, q, 0); }
__device__ __forceinline__ int first_slot(const Seq &q, int idx) { return (idx < q.head_tiles ? idx : idx + q.skipped) * kTile; }

// The tiles of all sequences, added up: every thread of the block has a run of sequences of its own.
struct Tally {
    int from, to;                        // the thread's sequences
    int64_t start, sum;                  // tiles before them and of them (of one item of each sequence)
    int64_t total;
};
// (kUnit: tiles that count as one)
template <int kUnit, typename Args>
__device__ __forceinline__ Seq units_of(const Args &a, int s, ull &bad)
{
    Seq q = seq_of(a, s, bad);
    q.tiles = (q.tiles + kUnit - 1) / kUnit;
    return q;
}
template <int kThreads, int kUnit = 1, typename Args>
__device__ __forceinline__ Tally tally_of(const Args &a, ull &bad)
{
    __shared__ int64_t s_sum[kThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int each = (a.c.num_seqs + kThreads - 1) / kThreads;
    Tally t;
    t.from = min(a.c.num_seqs, (int)threadIdx.x * each); t.to = min(a.c.num_seqs, t.from + each);
    long long sum = 0;
#pragma unroll 1
    for (int s = t.from; s < t.to; ++s) sum += units_of<kUnit>(a, s, bad).tiles;
    const long long upto = warp_inclusive_scan_i64(sum, lane);
    if (lane == 31) s_sum[warp] = upto;
    __syncthreads();
    t.start = upto - sum; t.sum = sum; t.total = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) t.start += s_sum[w];
        t.total += s_sum[w];
    }
    return t;
}

// How the tiles of all items are shared out over blocks.
struct Share {
    int64_t total;                       // tiles in all
    int blocks;                          // that share them
};
// `held` blocks run at a time, and each takes one share, of equal length.  Equal shares do not take equally long (with one share each, the first block of
// 64 sequences of 16 000 slots ended after 75 % of the time): where they are long and not more than two blocks share an SM they are cut into kCuts, and the
// blocks that wait for a place even it out (424 -> 412 us there, with two blocks an SM; with three it no longer tells).  Shorter ones are not: 320
// blocks of 24 tiles, where 296 run at a time, take two rounds (49 -> 71 us).
constexpr int kLong = 128, kCuts = 4;    // tiles
// (kUnit: as many tiles count as one)
template <int kUnit = 1>
__device__ __forceinline__ Share share_of(int64_t tiles, int per, int grid, int held)
{
    Share r;
    r.total = tiles * per;
    r.blocks = r.total >= (int64_t)(kLong / kUnit) * held ? grid : (int)max((int64_t)1, min((int64_t)held, r.total));
    return r;
}
// (a division of 32-bit numbers where they are: a third of the instructions)
__device__ __forceinline__ int64_t divided(int64_t x, int64_t by)
{
    if (((x | by) >> 32) == 0) return (int64_t)((unsigned)x / (unsigned)by);
    return x / by;
}
__device__ __forceinline__ int64_t begin_of(const Share &r, int b) { return b >= r.blocks ? r.total : divided(r.total * b, r.blocks); }
// Block whose share holds tile u.
__device__ __forceinline__ int owner_of(int64_t u, const Share &r) { return (int)divided((u + 1) * r.blocks - 1, r.total); }

// Sequence that tile u lies in, and the tiles before it: written by the one thread that has it among its sequences (u < total).
struct Place {
    int64_t before;
    int s;
};
template <int kUnit = 1, typename Args>
__device__ __forceinline__ void place_of(const Args &a, const Tally &t, int64_t u, int per, Place *to)
{
    if (!(t.start * per <= u && u < (t.start + t.sum) * per)) return;
    int64_t before = t.start * per;
    int s = t.from;
    for (;; ++s) {
        ull ignored = 0;
        const int64_t n = (int64_t)units_of<kUnit>(a, s, ignored).tiles * per;
        if (u < before + n) break;
        before += n;
    }
    to->before = before; to->s = s;
}

// A place in the run of tiles.
struct Cursor {
    int s, item, idx;                    // sequence, item of the sequence, tile of the item
    int head, block;                     // key-value head and block of rows: item = head * row_blocks + block
    Seq q;
};
template <int kUnit = 1, typename Args>
__device__ __forceinline__ void cursor_at(const Args &a, Cursor &u, const Place &p, int64_t tile)
{
    ull ignored = 0;
    u.s = p.s;
    u.q = units_of<kUnit>(a, p.s, ignored);
    const int64_t in = tile - p.before;
    u.item = (int)divided(in, u.q.tiles); u.idx = (int)(in - (int64_t)u.item * u.q.tiles);
    u.head = u.item / a.row_blocks; u.block = u.item - u.head * a.row_blocks;
}
template <int kUnit = 1, typename Args>
__device__ __forceinline__ void cursor_next(const Args &a, Cursor &u, int per)
{
    if (++u.idx < u.q.tiles) return;
    u.idx = 0;
    if (++u.block == a.row_blocks) { u.block = 0; ++u.head; }
    if (++u.item < per) return;
    u.item = u.head = u.block = 0;
    ull ignored = 0;
    do {
        if (++u.s >= a.c.num_seqs) { u.s = a.c.num_seqs; u.q.tiles = 0; return; }       // (behind the last: never used)
        u.q = units_of<kUnit>(a, u.s, ignored);
    } while (u.q.tiles == 0);
}

__device__ __forceinline__ bool sees(const AttendArgs &a, int p, int slot) { return slot <= p && (a.window == 0 || slot < a.sinks || slot > p - a.window); }

// (keys and values leave the L2 cache first: they are read once, and what is left there for the kernels behind is not)
__device__ __forceinline__ uint64_t leaves_first()
{
    uint64_t p;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
    return p;
}
__device__ __forceinline__ uint64_t stays()
{
    uint64_t p;
    asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(p));
    return p;
}
__device__ __forceinline__ void copy16(unsigned dst, const void *src, uint64_t policy)
{
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy) : "memory");
}
__device__ __forceinline__ void copy16_or_zeros(unsigned dst, const void *src, bool there)
{
    const int n = there ? 16 : 0;        // (0: 16 zero bytes)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ unsigned turned8x8(unsigned x)
{
    unsigned y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

constexpr int kParts = 4;                // warps of a block; each takes 16 slots of a tile
constexpr int kThreads = 32 * kParts;

// Weights are taken relative to ref, a maximum of the past, as long as no logit is more than kSlack above it, and multiply the values rounded to the
// cache's type (the second product's operands have to be of one type; a weight in two halves would double it).  bf16 reaches as far down as 32 bits do.
// fp16 is whole down to 2^-14 and ends at 2^-24: of thousands of slots that far below one, whose weights are all rounded alike, too much or nothing
// would be left.  So fp16 weights are 2^kLift times too large, in sums and results alike: up to 2^15, whole down to 2^-24 of the largest, and off
// by 2^-35 of it at most below that.  (16 new tokens of 4 heads, fp16: 70.3 us with a slack of 8, 70.9 with 5, 72.0 with 3; few rows: no difference.)
template <typename T>
struct Weights {
    static constexpr float kSlack = 8.0f, kLift = 0.0f, kUnlift = 1.0f;
};
template <>
struct Weights<__half> {
    static constexpr float kSlack = 5.0f, kLift = 10.0f, kUnlift = 1.0f / 1024.0f;       // (kSlack + kLift: 2^15, below 65504)
};

// Running maximum, sum and (four of) the accumulators of a row over some pieces.
struct Part {
    float top, sum;
    float4 o;
};
__device__ __forceinline__ void part_add(Part &p, float top, float sum, const float4 &o)
{
    const float best = fmaxf(p.top, top), ref = best == -INFINITY ? 0.0f : best;
    const float f = exp2_of(p.top - ref), g = exp2_of(top - ref);
    p.top = best;
    p.sum = p.sum * f + sum * g;
    p.o = make_float4(p.o.x * f + o.x * g, p.o.y * f + o.y * g, p.o.z * f + o.z * g, p.o.w * f + o.w * g);
}
// Kernels of a chain behind a shared beginning begin before the one before them has ended.  The beginning's wait for what is shared; the rest's attends while the beginning's pieces
// are joined, in room that it then uses, and waits before it writes anything.  Every block waits, so that a kernel's end says that those before it have ended.
template <typename Args>
__device__ __forceinline__ void begins_behind(const Args &)
{
    if (std::is_same<Args, BeginArgs>::value) asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
template <typename Args>
__device__ __forceinline__ void ends_behind(const Args &)
{
    if (std::is_same<Args, RestArgs>::value) asm volatile("griddepcontrol.wait;" ::: "memory");
}

// A row's result, four of its elements: maximum, sum of the weights and sums over all slots.  `at`: number of the row among [sequences][new tokens][query heads]; real: it has a
// token; sums: where the booking kernel looks for its lse.
template <typename T, typename Args>
__device__ __forceinline__ void give(const Args &a, int64_t at, int d, bool real, float top, float sum, float4 o, int64_t sums)
{
    if constexpr (std::is_same<Args, BeginArgs>::value) {
        if (d == 0) a.begin_ml[at] = make_float2(top, sum);
        *(float4 *)(a.begin_o + at * a.c.head_dim + d) = o;
        return;
    }
    if constexpr (std::is_same<Args, RestArgs>::value) {
        if (real && __ldcg(a.shared) > 0) {
            const float2 ml = __ldcg(&a.begin_ml[at]);
            Part p{top, sum, o};
            part_add(p, ml.x, ml.y, __ldcg((const float4 *)(a.begin_o + at * a.c.head_dim + d)));
            top = p.top; sum = p.sum; o = p.o;
        }
    }
    const float inv = 1.0f / sum;                        // (sees nothing: zero, whatever the sums hold)
    uint2 w = make_uint2(Pair<T>::pack(o.x * inv, o.y * inv), Pair<T>::pack(o.z * inv, o.w * inv));
    if (sum == 0.0f) w = make_uint2(0, 0);
    *(uint2 *)(a.out + 2 * (at * a.c.head_dim + d)) = w;
    if (d == 0) {
        const float lse = top + log2f(sum * Weights<T>::kUnlift);
        if (a.lse != nullptr) a.lse[at] = sum == 0.0f ? -INFINITY : lse * 0.69314718055994531f;
        if (a.books) a.sums[sums] = sum == 0.0f ? INFINITY : lse;
    }
}
// Blocks that share an SM, and tiles in a block's ring.  What a warp does for a tile is a chain that two warps a scheduler do not fill, so there are as many
// blocks as leave each a ring of two tiles and the registers it needs: four up to 64 dims (24 sequences of 4100 slots against two: 50 -> 39 us, 64 of
// 16 000: 280 -> 238), three above (128 dims: 57.6 -> 55.7, 428 -> 421).  Not so for rows of about 160 bytes, no whole number of the memory's 64: they are
// bound by it, and the more places are read from at a time the worse (a window over 80 dims 46 -> 52 us with three, 64 sequences 407 -> 420).  Wide
// heads: one block.
template <int kSteps, int kCols>
struct Ring {
    static_assert(kCols == 1 || kCols == 2, "8 or 16 rows");
    static constexpr int kOther = (kCols * kSteps <= 16 ? 0 : 8 * kCols * (32 * kSteps + 16)) + kParts * 8 * kCols * 8 + 8 * kCols * (64 * kSteps + 8) + 1024;
    static constexpr int kTileBytes = 2 * kTile * (32 * kSteps + 16);
    static constexpr int fits(int blocks) { return (226 * 1024 / blocks - kOther) / kTileBytes; }
    static constexpr int kBlocks = kSteps > 8 ? 1 : kSteps <= 4 && fits(4) >= 2 ? 4 : kSteps != 5 && fits(3) >= 2 ? 3 : 2;
    static constexpr int kStages = fits(kBlocks) > 6 ? 6 : fits(kBlocks);
    static_assert(kStages >= 2, "a tile in use, and one on its way");
};
template <typename T, int kSteps, int kCols>
struct Config {
    static constexpr int kStages = Ring<kSteps, kCols>::kStages;
    static constexpr int kDim = 16 * kSteps;             // head_dim, padded with zeros
    // bytes of a row in shared memory: an odd number of 16-byte units, so that the 8 rows of a matrix lie in different banks
    static constexpr int kPitch = 2 * kDim + 16;
    static constexpr int kRows = 8 * kCols;
    static constexpr int kPartBytes = 2 * 16 * kPitch;   // a warp's part of a tile: 16 keys, 16 values
    static constexpr bool kHeld = kCols * kSteps <= 16;  // the queries stay in registers
    // what a cluster's blocks read of one another: sums, and maximum and sum of the weights, of every row
    static constexpr int kShared = kRows * kDim * 4 + kRows * 8;
    static constexpr int kSmem = kParts * kStages * kPartBytes + (kHeld ? 0 : kRows * kPitch) + kParts * kRows * 8 + kShared;
    // joining the warps' sums: they fit the part of the ring that the warp has just left
    static constexpr int kMergePitch = kDim + 4;         // floats (2 rows apart: 8 banks)
    static_assert(kRows * kMergePitch * 4 <= kPartBytes, "a warp's sums fit");
};

// The block's four warps go through its tiles side by side, warp p at the 16 slots p of each, with maxima, sums and accumulators of their
// own and a ring of kStages parts each: nothing is waited for across warps before the piece ends and the four are joined.  Keys and values come
// by 16-byte asynchronous copies, row by row from wherever the page lies (bulk copies, one a row, are slower: a row of 256 bytes each 35
// clocks of an SM was measured, 2.1 TB/s in all); a lane looks the page of one slot up two tiles before it is worked on.
//   S^T [16 slots x rows] = K Q^T,  W^T = exp2(S^T - ref),  O^T [dims x rows] += V^T W^T,
// so that 8 rows (one key-value head's group of up to 8 query heads) fill the narrow side of the matrix instruction and keys and values
// its wide one.  W^T reaches the layout that the second product wants through one 8 x 8 transposition in registers.
// With `cluster` > 0, for few and short sequences, where the second kernel would take as long as the first: a cluster of so many blocks takes one
// item, each an equal part of its tiles, and joins the parts itself, through one another's shared memory (16 heads of 517 slots, calls in a graph: 7.1 -> 6.3 us).
// The tiles of an item are then numbered from item * cap on.
// ref is a maximum of the past (see Weights), so that the sums are rescaled and the warp's lanes compared only when a logit is far above it, a few times per
// piece.
template <typename T, int kSteps, int kCols, typename Args>
__global__ void __launch_bounds__(kThreads, Ring<kSteps, kCols>::kBlocks) k_cache_attend(const Args a, int held_blocks, int cluster, int cap)
{
    typedef Config<T, kSteps, kCols> C;
    constexpr int kStages = C::kStages;
    extern __shared__ __align__(128) char smem[];
    float *const s_join = (float *)(smem + kParts * kStages * C::kPartBytes);          // [kRows][kDim], then [kRows] maximum and sum
    float2 *const s_join_ml = (float2 *)(s_join + C::kRows * C::kDim);
    char *const s_q = smem + kParts * kStages * C::kPartBytes + C::kShared;
    float2 *const s_ml = (float2 *)(s_q + (C::kHeld ? 0 : C::kRows * C::kPitch));      // [kParts][kRows]
    __shared__ Place s_place;
    const int tid = threadIdx.x, lane = tid & 31, part = tid >> 5;
    const int per = a.c.kv_heads;                        // (one block of rows a head)
    ull bad = 0;
    begins_behind(a);
    Cursor now, ahead;
    int64_t begin;
    int n, rank = 0, my_item = 0;                        // (clusters)
    if (cluster > 0) {
        my_item = (int)blockIdx.x / cluster; rank = (int)blockIdx.x % cluster;
        now.s = my_item / per; now.item = now.head = my_item % per; now.block = 0;
        now.q = seq_of(a, now.s, bad);
        if (bad != 0) raise_status(a.c.status, bad);
        const int tiles = now.q.tiles;
        now.idx = tiles * rank / cluster;
        n = tiles * (rank + 1) / cluster - now.idx;
        begin = (int64_t)my_item * cap + now.idx;
        if (a.logits != nullptr && rank == 0) {          // (the numbers that the item does not use)
            for (int i = tiles + tid; i < cap; i += kThreads) a.notes[(int64_t)my_item * cap + i].length = 0;
            if (my_item == 0 && tid == 0) *a.total = (int64_t)a.c.num_seqs * per * cap;
        }
        if (tiles == 0) {                                // (the whole cluster alike)
            if (std::is_same<Args, BeginArgs>::value) return;
            const int chunks = a.c.head_dim / 8;
            for (int i = rank * kThreads + tid; i < C::kRows * chunks; i += cluster * kThreads) {
                const int row = i / chunks;
                if (row >= a.rows) continue;
                const int64_t at = ((int64_t)now.s * a.new_tokens + row / a.group) * a.q_heads + now.head * a.group + row % a.group;
                *(uint4 *)(a.out + 2 * at * a.c.head_dim + 16 * (i - row * chunks)) = make_uint4(0, 0, 0, 0);
                if (a.lse != nullptr && i == row * chunks) a.lse[at] = -INFINITY;
            }
            ends_behind(a);
            return;
        }
    } else {
        const Tally tally = tally_of<kThreads>(a, bad);
        const Share share = share_of(tally.total, per, gridDim.x, held_blocks);
        begin = begin_of(share, blockIdx.x);
        n = (int)(begin_of(share, blockIdx.x + 1) - begin);
        if (bad != 0) raise_status(a.c.status, bad);
        if (a.logits != nullptr && blockIdx.x == 0 && tid == 0) *a.total = share.total;
        if (n == 0) { ends_behind(a); return; }
        place_of(a, tally, begin, per, &s_place);
        __syncthreads();
        cursor_at(a, now, s_place, begin);
    }
    bad = 0;
    const int my_s = now.s, my_head = now.head, my_count = now.q.count;
    ahead = now;
    const unsigned ring = smem_of(smem) + part * kStages * C::kPartBytes;
    // where the row of this lane's slot begins (lanes 16 .. 31: as lanes 0 .. 15), in the tile that `ahead` stands at
    constexpr unsigned kNone = 0xffffffffu;              // (nothing to read: zeros)
    auto look_up = [&]() -> unsigned {
        const int slot = first_slot(ahead.q, ahead.idx) + part * 16 + (lane & 15);
        if (slot >= ahead.q.length || !(a.window == 0 || slot < a.sinks || slot > ahead.q.length - ahead.q.count - a.window)) return kNone;
        const Spot o = cache_spot(a.c, ahead.s, slot, bad);
        return o.page < 0 ? kNone : cache_row(a.c, o, ahead.head);
    };
    const uint64_t policy = leaves_first();
    auto issue = [&](int stage, unsigned row_at) {
        constexpr int kChunks = 2 * kSteps;              // of 16 bytes in a row
        const unsigned to = ring + stage * C::kPartBytes;
        const bool all = __all_sync(0xffffffffu, row_at != kNone) && a.c.head_dim == C::kDim;
        if (all) {                                       // (nearly always: an address, a shuffle and two copies)
#pragma unroll
            for (int i = 0; i < 16 * kChunks / 32; ++i) {
                const int c = i * 32 + lane, row = c / kChunks, chunk = c % kChunks;
                const int64_t at = 16 * (int64_t)__shfl_sync(0xffffffffu, row_at, row);
                copy16(to + row * C::kPitch + chunk * 16, a.c.k + 16 * chunk + at, policy);
                copy16(to + (16 + row) * C::kPitch + chunk * 16, a.c.v + 16 * chunk + at, policy);
            }
        } else {
#pragma unroll 1
            for (int i = 0; i < 16 * kChunks / 32; ++i) {
                const int c = i * 32 + lane, row = c / kChunks, chunk = c % kChunks;
                const unsigned from = __shfl_sync(0xffffffffu, row_at, row);
                const bool there = from != kNone && chunk * 8 < a.c.head_dim;
                const int64_t at = there ? 16 * ((int64_t)from + chunk) : 0;
                copy16_or_zeros(to + row * C::kPitch + chunk * 16, a.c.k + at, there);
                copy16_or_zeros(to + (16 + row) * C::kPitch + chunk * 16, a.c.v + at, there);
            }
        }
    };
    unsigned next_row = kNone;                           // of the tile to be issued next
    {
        unsigned rows[kStages];                          // (all on the way together: each is a miss)
#pragma unroll
        for (int i = 0; i < kStages; ++i) {
            rows[i] = kNone;
            if (i < n) { rows[i] = look_up(); cursor_next(a, ahead, per); }
        }
#pragma unroll
        for (int i = 0; i < kStages - 1; ++i) {
            if (i < n) issue(i, rows[i]);
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
        next_row = rows[kStages - 1];
    }

    float acc[kSteps][kCols][4], m[kCols][2], l[kCols][2];
    unsigned held[C::kHeld ? kSteps * kCols * 2 : 1];
    int p[kCols][2];                                     // slot at which a row's token stands, -1: no row
    bool fresh = true;
    int64_t item = 0;
    int stage = 0;
    const int logit_pitch = logit_rows(a.rows);
    for (int u = 0; u < n; ++u) {
        if (fresh) {                                     // a new item: its queries
            fresh = false;
            item = (int64_t)now.s * per + now.item;
            const int head = now.head;
            auto row_of = [&](int row) -> const char * { // (null: no such row)
                const int t = row / a.group;
                if (row >= a.rows || t >= now.q.count) return nullptr;
                return queries_of(a, now.s, t) + 2 * (head * a.group + row % a.group) * a.q_head;
            };
            if (C::kHeld) {
#pragma unroll
                for (int j = 0; j < kCols; ++j) {
                    const char *from = row_of(j * 8 + (lane >> 2));
#pragma unroll
                    for (int k = 0; k < 2 * kSteps; ++k) {
                        const int d = k * 8 + (lane & 3) * 2;
                        held[j * 2 * kSteps + k] = from != nullptr && d < a.c.head_dim ? __ldg((const unsigned *)(from + 2 * d)) : 0u;
                    }
                }
            } else {
                // (all warps have left the queries of the item before: they met when it was joined)
                for (int i = tid; i < C::kRows * 2 * kSteps; i += kThreads) {
                    const int r = i / (2 * kSteps), chunk = i % (2 * kSteps);
                    const char *from = row_of(r);
                    *(uint4 *)(s_q + r * C::kPitch + chunk * 16) = from != nullptr && chunk * 8 < a.c.head_dim ? __ldg((const uint4 *)(from + 16 * chunk)) : make_uint4(0, 0, 0, 0);
                }
                __syncthreads();
            }
#pragma unroll
            for (int j = 0; j < kCols; ++j) {
#pragma unroll
                for (int k = 0; k < kSteps; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[k][j][e] = 0.0f;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    m[j][h] = -INFINITY; l[j][h] = 0.0f;
                    const int row = j * 8 + (lane & 3) * 2 + h, t = row / a.group;
                    p[j][h] = row < a.rows && t < now.q.count ? stands_at(a, now.q, t) : -1;
                }
            }
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
        __syncwarp();
        if (u + kStages - 1 < n) issue(stage == 0 ? kStages - 1 : stage - 1, next_row);
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (u + kStages < n) { next_row = look_up(); cursor_next(a, ahead, per); }

        // ---- S^T ----
        const unsigned keys = ring + stage * C::kPartBytes, values = keys + 16 * C::kPitch;
        float x[kCols][4];
#pragma unroll
        for (int j = 0; j < kCols; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[j][e] = 0.0f;
        const unsigned k_at = keys + ((lane & 7) + ((lane >> 3) & 1) * 8) * C::kPitch + (lane >> 4) * 16;
        if (C::kHeld) {
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                unsigned ka[4];
                ldsm4(ka, k_at + k * 32);
#pragma unroll
                for (int j = 0; j < kCols; ++j) mma<T>(x[j], ka, held[j * 2 * kSteps + 2 * k], held[j * 2 * kSteps + 2 * k + 1]);
            }
        } else {
            // (16 rows of wide heads)
            const unsigned q_at = smem_of(s_q) + ((lane & 7) + (lane >> 4) * 8) * C::kPitch + ((lane >> 3) & 1) * 16;
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                unsigned ka[4], qb[4];
                ldsm4(ka, k_at + k * 32);
                ldsm4(qb, q_at + k * 32);
                mma<T>(x[0], ka, qb[0], qb[1]);
                mma<T>(x[kCols - 1], ka, qb[2], qb[3]);
            }
        }
        // ---- what each row sees ----
        const int slot0 = first_slot(now.q, now.idx) + part * 16, seen0 = seen_by_all(a, now.q);
        const bool whole = slot0 + 15 <= seen0 && (a.window == 0 || slot0 > now.q.length - 1 - a.window);
#pragma unroll
        for (int j = 0; j < kCols; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[j][e] *= a.scale_log2;
                if (!whole && !sees(a, p[j][e & 1], slot0 + (lane >> 2) + (e >> 1) * 8)) x[j][e] = -INFINITY;
            }
        if (a.logits != nullptr) {
            if (tid == 0) *(int4 *)&a.notes[begin + u] = make_int4(now.s, now.head, first_slot(now.q, now.idx), now.q.length);
            float *const to = a.logits + (begin + u) * (int64_t)(logit_pitch * kTile) + (part * 16 + (lane >> 2)) * logit_pitch;
#pragma unroll
            for (int j = 0; j < kCols; ++j) {
                const int r = j * 8 + (lane & 3) * 2;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float2 w = make_float2(p[j][0] < 0 ? -INFINITY : x[j][2 * e], p[j][1] < 0 ? -INFINITY : x[j][2 * e + 1]);
                    float *const at = to + e * 8 * logit_pitch + r;
                    if (logit_pitch > 1) { if (r < logit_pitch) *(float2 *)at = w; }
                    else if (r == 0) *at = w.x;
                }
            }
        }
        // ---- weights ----
        bool over = false;
#pragma unroll
        for (int j = 0; j < kCols; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) over |= fmaxf(x[j][h], x[j][h + 2]) > m[j][h] + Weights<T>::kSlack;
        if (__any_sync(0xffffffffu, over)) {
#pragma unroll
            for (int j = 0; j < kCols; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float top = fmaxf(x[j][h], x[j][h + 2]);
#pragma unroll
                    for (int o = 4; o < 32; o *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                    top = fmaxf(top, m[j][h]);
                    const float by = exp2_of(m[j][h] - (top == -INFINITY ? 0.0f : top));
                    m[j][h] = top;
                    l[j][h] *= by;
#pragma unroll
                    for (int k = 0; k < kSteps; ++k) { acc[k][j][h] *= by; acc[k][j][h + 2] *= by; }
                }
        }
#pragma unroll
        for (int j = 0; j < kCols; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float ref = (m[j][h] == -INFINITY ? 0.0f : m[j][h]) - Weights<T>::kLift;
                x[j][h] = exp2_of(x[j][h] - ref); x[j][h + 2] = exp2_of(x[j][h + 2] - ref);
                l[j][h] += x[j][h] + x[j][h + 2];
            }
        // ---- O^T ----
        __syncwarp();                                    // (a warp executes what follows as one)
        bool apart = false;
        if (!whole && now.q.count > 1) {
            // Slots that only some rows see: a weight of zero times an infinite or undefined value is not zero.
            for (int i = lane; i < 16 * C::kDim / 2; i += 32) {
                unsigned w;
                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(values + i / (C::kDim / 2) * C::kPitch + i % (C::kDim / 2) * 4) : "memory");
                const float2 f = Pair<T>::unpack(w);
                apart |= !(fabsf(f.x) <= 3.4028235e38f) || !(fabsf(f.y) <= 3.4028235e38f);
            }
            apart = __any_sync(0xffffffffu, apart);
        }
        if (!apart) {
            unsigned wb[kCols][2];
#pragma unroll
            for (int j = 0; j < kCols; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) wb[j][e] = turned8x8(Pair<T>::pack(x[j][2 * e], x[j][2 * e + 1]));
            const unsigned v_at = values + ((lane & 7) + ((lane >> 4) & 1) * 8) * C::kPitch + ((lane >> 3) & 1) * 16;
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                unsigned va[4];
                ldsm4t(va, v_at + k * 32);
#pragma unroll
                for (int j = 0; j < kCols; ++j) mma<T>(acc[k][j], va, wb[j][0], wb[j][1]);
            }
        } else {
            for (int o = 0; o < 16; ++o)
#pragma unroll
                for (int j = 0; j < kCols; ++j) {
                    float w[2];
                    bool in[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        w[h] = __shfl_sync(0xffffffffu, o < 8 ? x[j][h] : x[j][h + 2], (o & 7) * 4 + (lane & 3));
                        in[h] = sees(a, p[j][h], slot0 + o);
                    }
#pragma unroll
                    for (int k = 0; k < kSteps; ++k)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            unsigned short v;
                            asm volatile("ld.shared.b16 %0, [%1];" : "=h"(v) : "r"(values + o * C::kPitch + (k * 16 + e * 8 + (lane >> 2)) * 2) : "memory");
                            const float f = Pair<T>::unpack(v).x;
#pragma unroll
                            for (int h = 0; h < 2; ++h) if (in[h]) acc[k][j][2 * e + h] = fmaf(w[h], f, acc[k][j][2 * e + h]);
                        }
                }
        }
        if (now.idx == now.q.tiles - 1 || u == n - 1) {
            // ---- the piece's end: the parts are joined, each warp's sums in the part of its ring that it is done with ----
            ends_behind(a);
            __syncwarp();
#pragma unroll
            for (int j = 0; j < kCols; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int o = 4; o < 32; o *= 2) l[j][h] += __shfl_xor_sync(0xffffffffu, l[j][h], o);
                    if (lane < 4) s_ml[part * C::kRows + j * 8 + lane * 2 + h] = p[j][h] < 0 ? make_float2(-INFINITY, 0.0f) : make_float2(m[j][h], l[j][h]);
                }
            float *const room = (float *)(smem + stage * C::kPartBytes);
            constexpr int kApart = kStages * C::kPartBytes / 4;      // floats from one warp's to the next's
            // is this all of the item?
            const bool all = u >= now.idx && now.idx == now.q.tiles - 1;
            const int64_t piece = item + blockIdx.x;
#pragma unroll
            for (int j = 0; j < kCols; ++j)
#pragma unroll
                for (int k = 0; k < kSteps; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        room[part * kApart + (j * 8 + (lane & 3) * 2 + (e & 1)) * C::kMergePitch + k * 16 + (e >> 1) * 8 + (lane >> 2)] = acc[k][j][e];
            __syncthreads();
            for (int i = tid; i < C::kRows * (C::kDim / 4); i += kThreads) {
                const int row = i / (C::kDim / 4), d = i % (C::kDim / 4) * 4;
                if (row >= a.rows) continue;
                float top = -INFINITY, sum = 0.0f;
#pragma unroll
                for (int q = 0; q < kParts; ++q) top = fmaxf(top, s_ml[q * C::kRows + row].x);
                const float ref = top == -INFINITY ? 0.0f : top;
                float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (int q = 0; q < kParts; ++q) {
                    const float2 ml = s_ml[q * C::kRows + row];
                    const float f = exp2_of(ml.x - ref);
                    const float4 v = *(const float4 *)&room[q * kApart + row * C::kMergePitch + d];
                    sum = fmaf(ml.y, f, sum);
                    o.x = fmaf(v.x, f, o.x); o.y = fmaf(v.y, f, o.y); o.z = fmaf(v.z, f, o.z); o.w = fmaf(v.w, f, o.w);
                }
                if (cluster > 0) {
                    if (d == 0) s_join_ml[row] = make_float2(top, sum);
                    *(float4 *)(s_join + row * C::kDim + d) = o;
                    continue;
                }
                if (d == 0) a.ml[row * a.pieces + piece] = make_float2(top, sum);
                if (!all) {
                    *(float4 *)(a.part + (piece * C::kRows + row) * C::kDim + d) = o;
                } else if (d < a.c.head_dim) {
                    const int64_t at = ((int64_t)now.s * a.new_tokens + row / a.group) * a.q_heads + now.head * a.group + row % a.group;
                    give<T>(a, at, d, row / a.group < now.q.count, top, sum, o, item * C::kRows + row);
                }
            }
            fresh = true;
            __syncthreads();                             // (the ring may be written again)
        }
        stage = stage == kStages - 1 ? 0 : stage + 1;
        cursor_next(a, now, per);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (bad != 0) raise_status(a.c.status, bad);
    if (cluster > 0) {
        ends_behind(a);
        // ---- the item's parts are joined: each block takes some of the elements of all ----
        if (n == 0 && tid < C::kRows) s_join_ml[tid] = make_float2(-INFINITY, 0.0f);
        cluster_sync();
        const int quads = a.c.head_dim / 4;
        for (int e = tid * cluster + rank; e < a.rows * quads; e += kThreads * cluster) {
            const int row = e / quads, d = (e - row * quads) * 4;
            Part p;
            p.top = -INFINITY; p.sum = 0.0f; p.o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
            for (int q = 0; q < cluster; ++q) {
                const float2 ml = read_of(&s_join_ml[row], (unsigned)q);
                const float4 o = read_of((const float4 *)(s_join + row * C::kDim + d), (unsigned)q);
                if (ml.y != 0.0f) part_add(p, ml.x, ml.y, o);                      // (a part that saw nothing has no sums)
            }
            const int64_t at = ((int64_t)my_s * a.new_tokens + row / a.group) * a.q_heads + my_head * a.group + row % a.group;
            give<T>(a, at, d, row / a.group < my_count, p.top, p.sum, p.o, (int64_t)my_item * C::kRows + row);
        }
        cluster_sync();                                  // (nobody leaves while its memory may still be read)
    }
}

// The pieces of blocks b0 .. b1 joined by `lanes` neighbouring threads (a power of two up to 32), each with four pieces on their way at a time; every
// one has the result.
constexpr int kPiecesEach = 4;
__device__ __forceinline__ Part part_join(const AttendArgs &a, int64_t item, int b0, int b1, int block_rows, int r, int padded_dim, int d, int lanes)
{
    const int lane = threadIdx.x & (lanes - 1);
    Part p;
    p.top = -INFINITY; p.sum = 0.0f; p.o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 1
    for (int b = b0 + lane; b <= b1; b += kPiecesEach * lanes) {
        float2 ml[kPiecesEach];
        float4 o[kPiecesEach];
#pragma unroll
        for (int i = 0; i < kPiecesEach; ++i) {
            const int64_t piece = item + b + i * lanes;
            ml[i] = make_float2(-INFINITY, 0.0f); o[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (b + i * lanes <= b1) {
                ml[i] = __ldcg(&a.ml[r * a.pieces + piece]);
                o[i] = __ldcg((const float4 *)(a.part + (piece * block_rows + r) * padded_dim + d));
            }
        }
#pragma unroll
        for (int i = 0; i < kPiecesEach; ++i) part_add(p, ml[i].x, ml[i].y, o[i]);
    }
    for (int o = lanes / 2; o > 0; o >>= 1) {
        const float top = __shfl_xor_sync(0xffffffffu, p.top, o), sum = __shfl_xor_sync(0xffffffffu, p.sum, o);
        const float4 x = make_float4(__shfl_xor_sync(0xffffffffu, p.o.x, o), __shfl_xor_sync(0xffffffffu, p.o.y, o), __shfl_xor_sync(0xffffffffu, p.o.z, o),
                                     __shfl_xor_sync(0xffffffffu, p.o.w, o));
        part_add(p, top, sum, x);
    }
    return p;
}
__device__ __forceinline__ int lanes_for(int pieces)
{
    int n = 1;
    while (n * kPiecesEach < pieces && n < 32) n *= 2;
    return n;
}

// The pieces of an item: of the blocks b0 .. b1.
struct Pieces {
    int64_t item;
    int b0, b1;
};
__device__ __forceinline__ Pieces pieces_of(int64_t item, int64_t first, int tiles, const Share &r)
{
    return Pieces{item, owner_of(first, r), owner_of(first + tiles - 1, r)};
}

// The second kernel.  (1) An item that was cut into pieces is joined by the blocks whose turn its pieces' shares are, each taking a part of its rows
// and dimensions; (2) rows of sequences without tiles are written.  What follows from the lengths alone is worked out while the first
// kernel still runs.
template <typename T, int kUnit, typename Args>
__global__ void __launch_bounds__(kJoinThreads) k_cache_join(const Args a, int held_blocks, int padded_dim, int block_rows)
{
    __shared__ Place s_place[2];
    __shared__ Cursor s_cut[2];
    __shared__ Pieces s_pieces[2];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, per = a.c.kv_heads * a.row_blocks;
    ull ignored = 0;
    const Tally tally = tally_of<kJoinThreads, kUnit>(a, ignored);
    const Share share = share_of<kUnit>(tally.total, per, gridDim.x, held_blocks);        // the first kernel's
    const int b = blockIdx.x;
    const int64_t begin = begin_of(share, b), end = begin_of(share, b + 1);
    if (begin < end) { place_of<kUnit>(a, tally, begin, per, &s_place[0]); place_of<kUnit>(a, tally, end - 1, per, &s_place[1]); }
    __syncthreads();
    if (warp < 2 && begin < end) {
        const int64_t tile = warp == 0 ? begin : end - 1;
        Cursor u;
        cursor_at<kUnit>(a, u, s_place[warp], tile);
        const Pieces p = pieces_of((int64_t)u.s * per + u.item, tile - u.idx, u.q.tiles, share);
        if (lane == 0) { s_cut[warp] = u; s_pieces[warp] = p; }
    }
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    // (only now: a kernel behind this one finds all that the first has written)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // ---- (1): the items of the share's first and last tile (those between are whole), half of the warps each ----
    constexpr int kHalf = kJoinThreads / 64;
    const int side = warp / kHalf;
    const Pieces w = s_pieces[side];
    const int pieces = w.b1 - w.b0 + 1;
    if (begin < end && pieces > 1 && !(side == 1 && w.item == s_pieces[0].item)) {
        const int s = s_cut[side].s, head = s_cut[side].head, first_row = s_cut[side].block * block_rows, rows = min(block_rows, a.rows - first_row);
        const int lanes = lanes_for(pieces), teams = 32 / lanes;
        const int quads = a.c.head_dim / 4, all = rows * quads;
        const int parts = pieces * gridDim.y, nth = (b - w.b0) * gridDim.y + blockIdx.y;         // (128 rows at most: 32 bits)
        const int e0 = all * nth / parts, e1 = all * (nth + 1) / parts;
        for (int e = e0 + warp % kHalf * teams; e < e1; e += kHalf * teams) {                    // (all lanes take part in the shuffles)
            const int mine = min(e + lane / lanes, e1 - 1), r = mine / quads, d = mine % quads * 4, row = first_row + r;
            const Part p = part_join(a, w.item, w.b0, w.b1, block_rows, r, padded_dim, d, lanes);
            if (e + lane / lanes < e1 && (lane & (lanes - 1)) == 0) {
                const int64_t at = ((int64_t)s * a.new_tokens + row / a.group) * a.q_heads + head * a.group + row % a.group;
                give<T>(a, at, d, row / a.group < s_cut[side].q.count, p.top, p.sum, p.o, w.item * block_rows + r);
            }
        }
    }
    // ---- (2) ----
    for (int s = b; s < a.c.num_seqs && blockIdx.y == 0 && !std::is_same<Args, BeginArgs>::value; s += gridDim.x) {
        if (seq_of(a, s, ignored).tiles > 0) continue;
        const int64_t rows = (int64_t)a.new_tokens * a.q_heads, n = rows * (a.c.head_dim / 8);
        for (int64_t i = tid; i < n; i += kJoinThreads) ((uint4 *)(a.out + 2 * s * rows * a.c.head_dim))[i] = make_uint4(0, 0, 0, 0);
        if (a.lse != nullptr)
            for (int64_t i = tid; i < rows; i += kJoinThreads) a.lse[s * rows + i] = -INFINITY;
    }
}

// The third kernel books the weights: a warp per tile, from the note that the first kernel has left for it, so that there is nothing to search for.  A
// slot's rows lie side by side: as many neighbouring lanes as it has groups of four rows read them, add their weights exp2(logit - lse) up and join
// them, always in the same order; the first makes the one addition to the score.  A lane has the same rows of every slot, and so its part of the
// lse in registers.
template <int kTeam>
__device__ __forceinline__ void book_tile(const AttendArgs &a, const TileNote &note, int64_t tile, int block_rows, int pitch, bool &waited, ull &bad)
{
    auto joined = [&]() {                                // (what the second kernel writes: each lse)
        if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
        waited = true;
    };
    const int lane = threadIdx.x & 31, mate = lane & (kTeam - 1), r = 4 * mate;
    const float *const lse = a.sums + ((int64_t)note.s * a.c.kv_heads + note.head) * block_rows + r;
    constexpr int kPasses = 2 * kTeam, kAhead = kPasses < 8 ? kPasses : 8;
#pragma unroll 1
    for (int pass = 0; pass < kPasses; pass += kAhead) {
        Spot spot[kAhead];
        float w[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int slot = note.slot + (pass + i) * (32 / kTeam) + lane / kTeam;
            spot[i] = slot < note.length ? cache_spot(a.c, note.s, slot, bad) : Spot{-1, 0};
            w[i] = 0.0f;
        }
        const float *const from = a.logits + (tile * kTile + pass * (32 / kTeam) + lane / kTeam) * pitch;
        if (pitch >= 4) {
            float4 z = make_float4(INFINITY, INFINITY, INFINITY, INFINITY), x[kAhead];           // (no such row: weight 0)
#pragma unroll
            for (int i = 0; i < kAhead; ++i) x[i] = r < pitch ? __ldcg((const float4 *)(from + i * (32 / kTeam) * pitch + r)) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            joined();
            if (r < pitch) {
                z = __ldcg((const float4 *)lse);
                if (r + 1 >= a.rows) z.y = INFINITY;
                if (r + 2 >= a.rows) z.z = INFINITY;
                if (r + 3 >= a.rows) z.w = INFINITY;
                if (r >= a.rows) z.x = INFINITY;
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) w[i] += (exp2_of(x[i].x - z.x) + exp2_of(x[i].y - z.y)) + (exp2_of(x[i].z - z.z) + exp2_of(x[i].w - z.w));
        } else {
            for (int q = 0; q < pitch; ++q) {
                float x[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i) x[i] = __ldcg(from + i * 32 * pitch + q);
                joined();
                const float z = __ldcg(lse + q);
#pragma unroll
                for (int i = 0; i < kAhead; ++i) w[i] += exp2_of(x[i] - z);
            }
        }
#pragma unroll
        for (int o = kTeam / 2; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < kAhead; ++i) w[i] += __shfl_xor_sync(0xffffffffu, w[i], o);
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (mate == 0 && spot[i].page >= 0 && w[i] != 0.0f) atomicAdd(&a.c.scores[cache_cell(a.c, spot[i], note.head)], w[i]);
    }
}
template <int kTeam>
__global__ void __launch_bounds__(kJoinThreads) k_cache_book(const AttendArgs a, int block_rows, bool behind_join)
{
    // Behind the second kernel, which lets this one begin once the first is done: its notes and logits may be read at once.
    bool waited = !behind_join;
    if (waited) asm volatile("griddepcontrol.wait;" ::: "memory");
    const int pitch = logit_rows(a.rows);
    const int64_t total = __ldcg(a.total), step = (int64_t)gridDim.x * (kJoinThreads / 32);
    ull bad = 0;
    int64_t u = (int64_t)blockIdx.x * (kJoinThreads / 32) + (threadIdx.x >> 5);
    int4 x = make_int4(0, 0, 0, 0);
    if (u < total) x = __ldcg((const int4 *)&a.notes[u]);
    while (u < total) {
        const TileNote note{x.x, x.y, x.z, x.w};
        const int64_t now = u;
        u += step;
        if (u < total) x = __ldcg((const int4 *)&a.notes[u]);
        if (note.length > 0) book_tile<kTeam>(a, note, now, block_rows, pitch, waited, bad);
    }
    if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");      // (this kernel's end says that the second has ended)
    if (bad != 0) raise_status(a.c.status, bad);
}

// ---- host ----
// A launch that may begin before the kernel before it has ended.
inline cudaLaunchAttribute begins_early()
{
    cudaLaunchAttribute a = {};
    a.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    a.val.programmaticStreamSerializationAllowed = 1;
    return a;
}
template <typename... Wanted, typename... Given>
cudaError_t launch_behind(void (*kernel)(Wanted...), dim3 grid, int threads, size_t smem, cudaStream_t s, const Given &...args)
{
    cudaLaunchAttribute at[1] = {begins_early()};
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid; cfg.blockDim = dim3((unsigned)threads); cfg.dynamicSmemBytes = smem; cfg.stream = s; cfg.attrs = at; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}
// Kernels of a chain: see begins_behind().
template <typename Args>
constexpr bool kInChain = std::is_same<Args, BeginArgs>::value || std::is_same<Args, RestArgs>::value;

// The three kernels for up to 16 rows.  `kernel`: the first, kRows rows of kDim dims, `smem` bytes of shared memory; known, most_known: what the device holds of it.
template <typename T, int kRows, int kDim, int kUnit, typename JoinArgs, typename Args>
cudaError_t launch_few(void (*kernel)(const Args, int, int, int), size_t smem, int *known, int *most_known, const Args &a, const AttendShape &z, cudaStream_t s)
{
    int dev = 0, room = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if ((e = allow_launch((const void *)kernel, smem, 1)) != cudaSuccess) return e;
    if (dev < kMaxDevices) room = __atomic_load_n(&known[dev], __ATOMIC_ACQUIRE);
    if (room == 0) {
        int each = 0;
        if ((e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&each, kernel, kThreads, smem)) != cudaSuccess) return e;
        room = each * current_sm_count();
        if (room < 1) return cudaErrorInvalidDevice;
        if (dev < kMaxDevices) __atomic_store_n(&known[dev], room, __ATOMIC_RELEASE);
    }
    const int64_t units = z.tiles / kUnit;
    int64_t held = units < room ? units : room;
    held = held < 1 ? 1 : held > kMaxBlocks ? kMaxBlocks : held;
    const int64_t grid = z.tiles >= kLong * held && kCuts * held <= kMaxBlocks ? kCuts * held : held;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = smem; cfg.stream = s;
    // Clusters: where every item has at most four tiles a block (or as many units of them) and all blocks run at a time.
    const int64_t cap = z.items > 0 ? units / z.items : 0;
    int cluster = 0;
    if (z.items <= room && cap >= 1) {
        const void *const kernels[] = {(const void *)kernel};
        const int most = largest_cluster(kernels, false, kThreads, smem, most_known);
        int n = 1;
        while (2 * n <= 8 && 2 * n <= most && 2 * n <= cap && z.items * 2 * n <= room) n *= 2;
        if (most >= 1 && cap <= 4 * n) cluster = n;
    }
    cudaLaunchAttribute own[2];
    int attributes = 0;
    if (kInChain<Args>) own[attributes++] = begins_early();
    if (cluster > 0) {
        own[attributes].id = cudaLaunchAttributeClusterDimension;
        own[attributes].val.clusterDim.x = (unsigned)cluster; own[attributes].val.clusterDim.y = 1; own[attributes].val.clusterDim.z = 1;
        ++attributes;
        cfg.gridDim = dim3((unsigned)(z.items * cluster));
    }
    cfg.attrs = own; cfg.numAttrs = (unsigned)attributes;
    if ((e = cudaLaunchKernelEx(&cfg, kernel, a, (int)held, cluster, (int)cap)) != cudaSuccess) return e;
    // (the second kernel is brought in, and does its sums over the lengths, while the first still runs)
    cudaLaunchAttribute at[1] = {begins_early()};
    cfg.attrs = at; cfg.numAttrs = 1; cfg.blockDim = dim3(kJoinThreads); cfg.dynamicSmemBytes = 0;
    const JoinArgs &b = a;
    if (cluster == 0 && (e = cudaLaunchKernelEx(&cfg, k_cache_join<T, kUnit, JoinArgs>, b, (int)held, kDim, kRows)) != cudaSuccess) return e;
    if (a.logits == nullptr) return cudaSuccess;
    const int64_t warps = kJoinThreads / 32, blocks = (z.tiles + warps - 1) / warps, most = 148 * 6;
    cfg.gridDim = dim3((unsigned)(blocks < 1 ? 1 : blocks < most ? blocks : most));      // (a table without columns: no tile)
    const auto book = a.rows <= 4 ? k_cache_book<1> : a.rows <= 8 ? k_cache_book<2> : k_cache_book<4>;
    return cudaLaunchKernelEx(&cfg, book, b, kRows, cluster == 0);
}
template <typename T, int kSteps, int kCols, typename Args>
cudaError_t launch(const Args &a, const AttendShape &z, cudaStream_t s)
{
    typedef Config<T, kSteps, kCols> C;
    static int known[kMaxDevices], most_known[kMaxDevices];
    return launch_few<T, C::kRows, C::kDim, 1, Args>(k_cache_attend<T, kSteps, kCols, Args>, C::kSmem, known, most_known, a, z, s);
}
template <typename T, int kSteps, typename Args>
cudaError_t launch_steps(const Args &a, const AttendShape &z, cudaStream_t s)
{
    return z.block_rows == 8 ? launch<T, kSteps, 1>(a, z, s) : launch<T, kSteps, 2>(a, z, s);
}
template <typename T, typename Args>
cudaError_t launch_type(const Args &a, const AttendShape &z, cudaStream_t s)
{
    switch (z.padded_dim / 16) {
    case 4: return launch_steps<T, 4>(a, z, s);
    case 5: return launch_steps<T, 5>(a, z, s);
    case 6: return launch_steps<T, 6>(a, z, s);
    case 8: return launch_steps<T, 8>(a, z, s);
    case 12: return launch_steps<T, 12>(a, z, s);
    default: return launch_steps<T, 16>(a, z, s);
    }
}

}  // namespace attend

cudaError_t launch_cache_attend_bf16(const AttendArgs &a, const AttendShape &z, cudaStream_t s);
cudaError_t launch_cache_attend_fp16(const AttendArgs &a, const AttendShape &z, cudaStream_t s);
cudaError_t launch_cache_rows_bf16(const AttendArgs &a, const AttendShape &z, cudaStream_t s);      // (g10_cache_rows_*.cu)
cudaError_t launch_cache_rows_fp16(const AttendArgs &a, const AttendShape &z, cudaStream_t s);

}  // namespace g10
