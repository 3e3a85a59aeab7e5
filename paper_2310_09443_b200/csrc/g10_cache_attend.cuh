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
// leaves s_j (4 bytes a row, beside 4 * head_dim bytes of key and value), and the second adds the weights up.  Each slot's sum is made by one
// thread over its rows in order and added once: the same every time.
#pragma once
#include "g10_cache.cuh"

namespace g10 {
namespace attend {

constexpr int kTile = 64;                // slots
constexpr int kMaxBlocks = 148 * 8;      // of the grid; the workspace has room for their pieces
constexpr int kJoinThreads = 256;

__device__ __forceinline__ unsigned smem_of(const void *p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(unsigned dst, const void *src, bool there)
{
    const int n = there ? 16 : 0;        // (0: 16 zero bytes)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
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
__device__ __forceinline__ int first_slot(const Seq &q, int idx) { return (idx < q.head_tiles ? idx : idx + q.skipped) * kTile; }

// The tiles of all sequences, added up: every thread of the block has a run of sequences of its own.
struct Tally {
    int from, to;                        // the thread's sequences
    int64_t start, sum;                  // tiles before them and of them (of one item of each sequence)
    int64_t total;
};
template <int kThreads>
__device__ __forceinline__ Tally tally_of(const AttendArgs &a, ull &bad)
{
    __shared__ int64_t s_sum[kThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int each = (a.c.num_seqs + kThreads - 1) / kThreads;
    Tally t;
    t.from = min(a.c.num_seqs, (int)threadIdx.x * each); t.to = min(a.c.num_seqs, t.from + each);
    long long sum = 0;
    for (int s = t.from; s < t.to; ++s) sum += seq_of(a, s, bad).tiles;
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
__device__ __forceinline__ Share share_of(int64_t tiles, int per, int grid, int min_tiles)
{
    Share r;
    r.total = tiles * per;
    r.blocks = (int)min((int64_t)grid, max((int64_t)1, (r.total + min_tiles - 1) / min_tiles));
    return r;
}
__device__ __forceinline__ int64_t begin_of(const Share &r, int b) { return b >= r.blocks ? r.total : r.total * b / r.blocks; }
// Block whose share holds tile u.
__device__ __forceinline__ int owner_of(int64_t u, const Share &r) { return (int)(((u + 1) * r.blocks - 1) / r.total); }

// Sequence that tile u lies in, and the tiles before it: written by the one thread that has it among its sequences (u < total).
struct Place {
    int64_t before;
    int s;
};
__device__ __forceinline__ void place_of(const AttendArgs &a, const Tally &t, int64_t u, int per, Place *to)
{
    if (!(t.start * per <= u && u < (t.start + t.sum) * per)) return;
    int64_t before = t.start * per;
    int s = t.from;
    for (;; ++s) {
        ull ignored = 0;
        const int64_t n = (int64_t)seq_of(a, s, ignored).tiles * per;
        if (u < before + n) break;
        before += n;
    }
    to->before = before; to->s = s;
}

// A place in the run of tiles.
struct Cursor {
    int s, item, idx;                    // sequence, item of the sequence, tile of the item
    Seq q;
};
__device__ __forceinline__ void cursor_at(const AttendArgs &a, Cursor &u, const Place &p, int64_t tile)
{
    ull ignored = 0;
    u.s = p.s;
    u.q = seq_of(a, p.s, ignored);
    const int64_t in = tile - p.before;
    u.item = (int)(in / u.q.tiles); u.idx = (int)(in % u.q.tiles);
}
__device__ __forceinline__ void cursor_next(const AttendArgs &a, Cursor &u, int per)
{
    if (++u.idx < u.q.tiles) return;
    u.idx = 0;
    if (++u.item < per) return;
    u.item = 0;
    ull ignored = 0;
    do {
        if (++u.s >= a.c.num_seqs) { u.s = a.c.num_seqs; u.q.tiles = 0; return; }       // (behind the last: never used)
        u.q = seq_of(a, u.s, ignored);
    } while (u.q.tiles == 0);
}

__device__ __forceinline__ bool sees(const AttendArgs &a, int p, int slot) { return slot <= p && (a.window == 0 || slot < a.sinks || slot > p - a.window); }

template <typename T, int kSteps, int kRowTiles, int kParts, int kStages>
struct Config {
    static constexpr int kWarps = kRowTiles * kParts, kThreads = 32 * kWarps;
    static constexpr int kDim = 16 * kSteps;             // head_dim, padded with zeros
    // bytes of a row in shared memory: an odd number of 16-byte units, so that the 8 rows of a matrix lie in different banks
    static constexpr int kPitch = 2 * kDim + 16;
    static constexpr int kRows = 16 * kRowTiles;
    static constexpr int kStageBytes = 2 * kTile * kPitch;
    static constexpr int kSmem = kStages * kStageBytes + kRows * kPitch + kStages * kTile * 8 + kParts * kRows * 8;
    static constexpr int kTokens = kTile / kParts;       // slots of a tile that one warp takes
    // joining the warps' sums: half of them are put into the stage that the last tile has left
    static constexpr int kMergeParts = kParts / 2;
    static_assert(kMergeParts == 0 || kRowTiles * kMergeParts * 32 * kSteps * 8 * 4 <= kStageBytes, "the warps' sums fit one stage");
};

// A block has kRowTiles * kParts warps: warp (r, p) holds rows 16 r .. 16 r + 15 and looks at the p-th part of every tile, with a
// maximum, a sum and accumulators of its own; the parts are joined when the piece ends.  Keys and values come by 16-byte asynchronous
// copies into a ring of kStages tiles, row by row from wherever the page lies; the addresses of a tile are worked out one tile before its
// copies are issued and the page numbers loaded before that tile's arithmetic, so that no wait for the table is on the way.
template <typename T, int kSteps, int kRowTiles, int kParts, int kStages>
__global__ void __launch_bounds__(32 * kRowTiles *kParts) k_cache_attend(const AttendArgs a, int min_tiles)
{
    typedef Config<T, kSteps, kRowTiles, kParts, kStages> C;
    extern __shared__ __align__(128) char smem[];
    char *const s_q = smem + kStages * C::kStageBytes;
    int64_t *const s_from = (int64_t *)(s_q + C::kRows * C::kPitch);          // [kStages][kTile] first element of each row, -1: zeros
    float2 *const s_ml = (float2 *)(s_from + kStages * kTile);                // [kParts][kRows]
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int wr = warp / kParts, wp = warp % kParts;
    const int per = a.c.kv_heads * a.row_blocks;
    ull bad = 0;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ Place s_place;
    const Tally tally = tally_of<C::kThreads>(a, bad);
    const Share share = share_of(tally.total, per, gridDim.x, min_tiles);
    const int64_t begin = begin_of(share, blockIdx.x);
    const int n = (int)(begin_of(share, blockIdx.x + 1) - begin);
    if (bad != 0) raise_status(a.c.status, bad);
    if (n == 0) return;
    bad = 0;
    place_of(a, tally, begin, per, &s_place);
    __syncthreads();

    Cursor now, ahead;
    cursor_at(a, now, s_place, begin);
    ahead = now;
    // the page of a slot of the tile that `ahead` stands at, for threads 0 .. 63; -1: nothing to read
    auto look_up = [&](int &slot) -> int {
        slot = first_slot(ahead.q, ahead.idx) + tid;
        if (slot >= ahead.q.length || !(a.window == 0 || slot < a.sinks || slot > ahead.q.length - ahead.q.count - a.window)) return -1;
        return cache_page(a.c, ahead.s, slot, bad);
    };
    auto row_from = [&](int page, int slot) -> int64_t { return page < 0 ? -1 : cache_row(a.c, page, slot, ahead.item / a.row_blocks); };
    // copies of one tile into its stage
    auto issue = [&](int stage) {
        constexpr int kChunks = 2 * kSteps;              // of 16 bytes in a row
        const unsigned to = smem_of(smem) + stage * C::kStageBytes;
#pragma unroll 4
        for (int i = tid; i < kTile * kChunks; i += C::kThreads) {
            const int row = i / kChunks, chunk = i % kChunks;
            const int64_t from = s_from[stage * kTile + row];
            const bool there = from >= 0 && chunk * 8 < a.c.head_dim;
            const int64_t at = there ? 2 * from + 16 * chunk : 0;
            copy16(to + row * C::kPitch + chunk * 16, a.c.k + at, there);
            copy16(to + (kTile + row) * C::kPitch + chunk * 16, a.c.v + at, there);
        }
    };
#pragma unroll
    for (int i = 0; i < kStages; ++i) {
        if (i < n) {
            if (tid < kTile) { int slot; const int page = look_up(slot); s_from[i * kTile + tid] = row_from(page, slot); }
            cursor_next(a, ahead, per);
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) {
        if (i < n) issue(i);
        asm volatile("cp.async.commit_group;" ::: "memory");
    }

    float acc[2 * kSteps][4], m[2], l[2];
    bool fresh = true;
    int64_t item = 0;
    int first_row = 0;
    int stage = 0;
    for (int u = 0; u < n; ++u) {
        if (fresh) {                                     // a new item: its queries
            fresh = false;
            item = (int64_t)now.s * per + now.item;
            first_row = (now.item % a.row_blocks) * C::kRows;
            const int head = now.item / a.row_blocks;
            for (int i = tid; i < C::kRows * 2 * kSteps; i += C::kThreads) {
                const int r = i / (2 * kSteps), chunk = i % (2 * kSteps), row = first_row + r;
                uint4 x = make_uint4(0, 0, 0, 0);
                const int t = row / a.group;
                if (row < a.rows && t < now.q.count && chunk * 8 < a.c.head_dim)
                    x = __ldg((const uint4 *)(a.q + 2 * (now.s * a.q_seq + t * a.q_token + (head * a.group + row % a.group) * a.q_head) + 16 * chunk));
                *(uint4 *)(s_q + r * C::kPitch + chunk * 16) = x;
            }
#pragma unroll
            for (int i = 0; i < 2 * kSteps; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][e] = 0.0f;
            m[0] = m[1] = -INFINITY; l[0] = l[1] = 0.0f;
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
        __syncthreads();
        if (u + kStages - 1 < n) issue(stage == 0 ? kStages - 1 : stage - 1);
        asm volatile("cp.async.commit_group;" ::: "memory");
        int page = -1, slot_ahead = 0;
        const bool more = u + kStages < n;
        if (more && tid < kTile) page = look_up(slot_ahead);

        // ---- the tile's products with the queries ----
        const unsigned keys = smem_of(smem) + stage * C::kStageBytes + wp * C::kTokens * C::kPitch, values = keys + kTile * C::kPitch;
        const unsigned queries = smem_of(s_q) + wr * 16 * C::kPitch;
        constexpr int kN = C::kTokens / 8;
        float x[kN][4];
#pragma unroll
        for (int j = 0; j < kN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[j][e] = 0.0f;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            unsigned qa[4], kb[4];
            ldsm4(qa, queries + ((lane & 7) + ((lane >> 3) & 1) * 8) * C::kPitch + (2 * k + (lane >> 4)) * 16);
#pragma unroll
            for (int j = 0; j < kN; j += 2) {
                ldsm4(kb, keys + (j * 8 + (lane & 7) + (lane >> 4) * 8) * C::kPitch + (2 * k + ((lane >> 3) & 1)) * 16);
                mma<T>(x[j], qa, kb[0], kb[1]);
                mma<T>(x[j + 1], qa, kb[2], kb[3]);
            }
        }
        // ---- what each row sees ----
        const int slot0 = first_slot(now.q, now.idx) + wp * C::kTokens, seen0 = now.q.length - now.q.count;
        const bool whole = slot0 + C::kTokens - 1 <= seen0 && (a.window == 0 || slot0 > now.q.length - 1 - a.window);
        int p[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = first_row + wr * 16 + (lane >> 2) + 8 * h, t = row / a.group;
            p[h] = row < a.rows && t < now.q.count ? seen0 + t : -1;
        }
#pragma unroll
        for (int j = 0; j < kN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[j][e] *= a.scale_log2;
                if (p[e >> 1] < 0 || (!whole && !sees(a, p[e >> 1], slot0 + j * 8 + (lane & 3) * 2 + (e & 1)))) x[j][e] = -INFINITY;
            }
        if (a.logits != nullptr) {
            const int kept = min(C::kRows, a.rows);
            float *to = a.logits + (begin + u) * (int64_t)(kept * kTile);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = wr * 16 + (lane >> 2) + 8 * h;
                if (r < kept) {
#pragma unroll
                    for (int j = 0; j < kN; ++j)
                        *(float2 *)(to + r * kTile + wp * C::kTokens + j * 8 + (lane & 3) * 2) = make_float2(x[j][2 * h], x[j][2 * h + 1]);
                }
            }
        }
        // ---- running maximum and sum ----
        bool scales = false;
        float by[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float top = m[h];
#pragma unroll
            for (int j = 0; j < kN; ++j) top = fmaxf(top, fmaxf(x[j][2 * h], x[j][2 * h + 1]));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const float ref = top == -INFINITY ? 0.0f : top;
            by[h] = exp2_of(m[h] - ref);
            scales |= top != m[h];
            m[h] = top;
            l[h] *= by[h];
#pragma unroll
            for (int j = 0; j < kN; ++j)
#pragma unroll
                for (int e = 2 * h; e < 2 * h + 2; ++e) { x[j][e] = exp2_of(x[j][e] - ref); l[h] += x[j][e]; }
        }
        if (__any_sync(0xffffffffu, scales)) {
#pragma unroll
            for (int i = 0; i < 2 * kSteps; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][e] *= by[e >> 1];
        }
        // ---- the weights' products with the values ----
        bool apart = false;
        if (!whole && now.q.count > 1) {
            // Slots that only some rows see: a weight of zero times an infinite or undefined value is not zero.
            for (int i = lane; i < C::kTokens * C::kDim / 2; i += 32) {
                unsigned w;
                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(values + i / (C::kDim / 2) * C::kPitch + i % (C::kDim / 2) * 4) : "memory");
                const float2 f = Pair<T>::unpack(w);
                apart |= !(fabsf(f.x) <= 3.4028235e38f) || !(fabsf(f.y) <= 3.4028235e38f);
            }
            apart = __any_sync(0xffffffffu, apart);
        }
        if (!apart) {
#pragma unroll
            for (int j = 0; j < kN; j += 2) {
                unsigned pa[4], vb[4];
                pa[0] = Pair<T>::pack(x[j][0], x[j][1]); pa[1] = Pair<T>::pack(x[j][2], x[j][3]);
                pa[2] = Pair<T>::pack(x[j + 1][0], x[j + 1][1]); pa[3] = Pair<T>::pack(x[j + 1][2], x[j + 1][3]);
#pragma unroll
                for (int k = 0; k < kSteps; ++k) {
                    ldsm4t(vb, values + (j * 8 + (lane & 7) + ((lane >> 3) & 1) * 8) * C::kPitch + (2 * k + (lane >> 4)) * 16);
                    mma<T>(acc[2 * k], pa, vb[0], vb[1]);
                    mma<T>(acc[2 * k + 1], pa, vb[2], vb[3]);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < kN; ++j)
                for (int o = 0; o < 8; ++o)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float mine = (o & 1) ? x[j][2 * h + 1] : x[j][2 * h];
                        const float w = __shfl_sync(0xffffffffu, mine, (lane & ~3) | (o >> 1));
                        if (sees(a, p[h], slot0 + j * 8 + o)) {
#pragma unroll
                            for (int i = 0; i < 2 * kSteps; ++i) {
                                unsigned v;
                                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(values + (j * 8 + o) * C::kPitch + i * 16 + (lane & 3) * 4) : "memory");
                                const float2 f = Pair<T>::unpack(v);
                                acc[i][2 * h] = fmaf(w, f.x, acc[i][2 * h]); acc[i][2 * h + 1] = fmaf(w, f.y, acc[i][2 * h + 1]);
                            }
                        }
                    }
        }
        if (more) {
            if (tid < kTile) s_from[stage * kTile + tid] = row_from(page, slot_ahead);
            cursor_next(a, ahead, per);
        }
        const Cursor was = now;
        cursor_next(a, now, per);
        // ---- the piece's end: the warps' parts are joined ----
        if (now.idx == 0 || u == n - 1) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
                l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
                if ((lane & 3) == 0) s_ml[wp * C::kRows + wr * 16 + (lane >> 2) + 8 * h] = make_float2(m[h], l[h]);
            }
            __syncthreads();                             // (and nobody reads the tile any more)
            float sum[2], f[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = wr * 16 + (lane >> 2) + 8 * h;
                float top = -INFINITY;
#pragma unroll
                for (int q = 0; q < kParts; ++q) top = fmaxf(top, s_ml[q * C::kRows + r].x);
                const float ref = top == -INFINITY ? 0.0f : top;
                sum[h] = 0.0f;
#pragma unroll
                for (int q = 0; q < kParts; ++q) { const float2 v = s_ml[q * C::kRows + r]; sum[h] += v.y * exp2_of(v.x - ref); }
                f[h] = exp2_of(m[h] - ref);
                m[h] = top;
            }
#pragma unroll
            for (int i = 0; i < 2 * kSteps; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][e] *= f[e >> 1];
            float4 *const room = (float4 *)(smem + stage * C::kStageBytes);
#pragma unroll
            for (int half = kParts / 2; half > 0; half >>= 1) {
                if (wp >= half && wp < 2 * half) {
#pragma unroll
                    for (int i = 0; i < 2 * kSteps; ++i)
                        room[((wr * half + wp - half) * 2 * kSteps + i) * 32 + lane] = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
                }
                __syncthreads();
                if (wp < half) {
#pragma unroll
                    for (int i = 0; i < 2 * kSteps; ++i) {
                        const float4 o = room[((wr * half + wp) * 2 * kSteps + i) * 32 + lane];
                        acc[i][0] += o.x; acc[i][1] += o.y; acc[i][2] += o.z; acc[i][3] += o.w;
                    }
                }
                __syncthreads();
            }
            // is this all of the item?
            const int first = u - was.idx;               // (the item's first tile, counted from the share's)
            const bool all = first >= 0 && now.idx == 0 && was.idx == was.q.tiles - 1;
            if (wp == 0) {
                const int64_t piece = (item + blockIdx.x) * C::kRows;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int r = wr * 16 + (lane >> 2) + 8 * h, row = first_row + r;
                    if (row >= a.rows) continue;
                    if ((lane & 3) == 0) a.ml[piece + r] = make_float2(m[h], sum[h]);
                    if (all) {
                        const int64_t at = ((int64_t)was.s * a.new_tokens + row / a.group) * a.q_heads + (was.item / a.row_blocks) * a.group + row % a.group;
                        const float inv = 1.0f / sum[h];                   // (sees nothing: zero, whatever the sums hold)
#pragma unroll
                        for (int i = 0; i < 2 * kSteps; ++i)
                            if (i * 8 < a.c.head_dim)
                                *(unsigned *)(a.out + 2 * (at * a.c.head_dim + i * 8 + (lane & 3) * 2)) =
                                    sum[h] == 0.0f ? 0u : Pair<T>::pack(acc[i][2 * h] * inv, acc[i][2 * h + 1] * inv);
                        if (a.lse != nullptr && (lane & 3) == 0) a.lse[at] = sum[h] == 0.0f ? -INFINITY : (m[h] + log2f(sum[h])) * 0.69314718055994531f;
                    } else {
#pragma unroll
                        for (int i = 0; i < 2 * kSteps; ++i)
                            *(float2 *)(a.part + (piece + r) * C::kDim + i * 8 + (lane & 3) * 2) = make_float2(acc[i][2 * h], acc[i][2 * h + 1]);
                    }
                }
            }
            fresh = true;
        }
        stage = stage == kStages - 1 ? 0 : stage + 1;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (bad != 0) raise_status(a.c.status, bad);
}

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
// The pieces of blocks b0 .. b1 joined by `lanes` neighbouring threads (a power of two up to 32); every one has the result.
template <bool kSums>
__device__ __forceinline__ Part part_join(const AttendArgs &a, int64_t item, int b0, int b1, int block_rows, int r, int padded_dim, int d, int lanes)
{
    const int lane = threadIdx.x & (lanes - 1);
    Part p;
    p.top = -INFINITY; p.sum = 0.0f; p.o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int b = b0 + lane; b <= b1; b += lanes) {
        const int64_t piece = (item + b) * block_rows + r;
        const float2 ml = __ldcg(&a.ml[piece]);
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (kSums) o = __ldcg((const float4 *)(a.part + piece * padded_dim + d));
        part_add(p, ml.x, ml.y, o);
    }
    for (int o = lanes / 2; o > 0; o >>= 1) {
        const float top = __shfl_xor_sync(0xffffffffu, p.top, o), sum = __shfl_xor_sync(0xffffffffu, p.sum, o);
        float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (kSums)
            x = make_float4(__shfl_xor_sync(0xffffffffu, p.o.x, o), __shfl_xor_sync(0xffffffffu, p.o.y, o), __shfl_xor_sync(0xffffffffu, p.o.z, o),
                            __shfl_xor_sync(0xffffffffu, p.o.w, o));
        part_add(p, top, sum, x);
    }
    return p;
}
__device__ __forceinline__ int lanes_for(int pieces)
{
    int n = 1;
    while (n < pieces && n < 32) n *= 2;
    return n;
}

// The second kernel.  (1) An item that was cut into pieces is joined by the blocks that made them, each taking a part of its rows and
// dimensions; (2) rows of sequences without tiles are written; (3) weights are booked, the slots of all (sequence, head) shared out anew.
template <typename T>
__global__ void __launch_bounds__(kJoinThreads) k_cache_join(const AttendArgs a, int min_tiles, int padded_dim, int block_rows)
{
    __shared__ float s_lse[1024];
    __shared__ Place s_place[3];
    const int tid = threadIdx.x, per = a.c.kv_heads * a.row_blocks;
    ull ignored = 0;
    const Tally tally = tally_of<kJoinThreads>(a, ignored);
    const Share share = share_of(tally.total, per, gridDim.x, min_tiles);          // the first kernel's
    const int64_t begin = begin_of(share, blockIdx.x), end = begin_of(share, blockIdx.x + 1);
    const Share slots = share_of(tally.total, a.c.kv_heads, gridDim.x, 1);         // of (3)
    const int64_t from = begin_of(slots, blockIdx.x), to = begin_of(slots, blockIdx.x + 1);
    if (begin < end) { place_of(a, tally, begin, per, &s_place[0]); place_of(a, tally, end - 1, per, &s_place[1]); }
    if (a.logits != nullptr && from < to) place_of(a, tally, from, a.c.kv_heads, &s_place[2]);
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");

    // ---- (1): the items of the block's first and last tile (those between are whole) ----
    int64_t done = -1;
    for (int side = 0; side < 2 && begin < end; ++side) {
        const int64_t tile = side == 0 ? begin : end - 1;
        Cursor u;
        cursor_at(a, u, s_place[side], tile);
        const int64_t item = (int64_t)u.s * per + u.item, first = tile - u.idx;
        if (item == done) continue;
        done = item;
        const int b0 = owner_of(first, share), b1 = owner_of(first + u.q.tiles - 1, share), pieces = b1 - b0 + 1;
        if (pieces == 1) continue;
        const int lanes = lanes_for(pieces), teams = kJoinThreads / lanes;
        const int first_row = (u.item % a.row_blocks) * block_rows, rows = min(block_rows, a.rows - first_row);
        const int quads = (a.c.head_dim + 3) / 4, all = rows * quads;
        const int e0 = (int)((int64_t)all * ((int)blockIdx.x - b0) / pieces), e1 = (int)((int64_t)all * ((int)blockIdx.x - b0 + 1) / pieces);
        for (int e = e0; e < e1; e += teams) {           // (all threads take part in the shuffles)
            const int mine = min(e + tid / lanes, e1 - 1), r = mine / quads, d = mine % quads * 4, row = first_row + r;
            const Part p = part_join<true>(a, item, b0, b1, block_rows, r, padded_dim, d, lanes);
            if (e + tid / lanes < e1 && (tid & (lanes - 1)) == 0) {
                const int64_t at = ((int64_t)u.s * a.new_tokens + row / a.group) * a.q_heads + (u.item / a.row_blocks) * a.group + row % a.group;
                const float inv = 1.0f / p.sum;
                uint2 w = make_uint2(Pair<T>::pack(p.o.x * inv, p.o.y * inv), Pair<T>::pack(p.o.z * inv, p.o.w * inv));
                if (p.sum == 0.0f) w = make_uint2(0, 0);
                *(uint2 *)(a.out + 2 * (at * a.c.head_dim + d)) = w;
                if (a.lse != nullptr && d == 0) a.lse[at] = p.sum == 0.0f ? -INFINITY : (p.top + log2f(p.sum)) * 0.69314718055994531f;
            }
        }
    }
    // ---- (2) ----
    for (int s = blockIdx.x; s < a.c.num_seqs; s += gridDim.x) {
        if (seq_of(a, s, ignored).tiles > 0) continue;
        const int64_t rows = (int64_t)a.new_tokens * a.q_heads, n = rows * (a.c.head_dim / 8);
        for (int64_t i = tid; i < n; i += kJoinThreads) ((uint4 *)(a.out + 2 * s * rows * a.c.head_dim))[i] = make_uint4(0, 0, 0, 0);
        if (a.lse != nullptr)
            for (int64_t i = tid; i < rows; i += kJoinThreads) a.lse[s * rows + i] = -INFINITY;
    }
    if (a.logits == nullptr || from >= to) return;

    // ---- (3) ----
    Cursor now;
    cursor_at(a, now, s_place[2], from);
    const int kept = min(block_rows, a.rows);
    int64_t before = s_place[2].before;                  // (tiles of the sequences before, one block of rows)
    ull bad = 0;
    for (int64_t u = from; u < to;) {
        const int n = (int)min((int64_t)(now.q.tiles - now.idx), to - u);          // tiles of this (sequence, head)
        __syncthreads();
        for (int b = 0; b < a.row_blocks; ++b) {
            const int i = now.item * a.row_blocks + b;
            const int64_t first = before * a.row_blocks + (int64_t)i * now.q.tiles;
            const int b0 = owner_of(first, share), b1 = owner_of(first + now.q.tiles - 1, share), lanes = lanes_for(b1 - b0 + 1), teams = kJoinThreads / lanes;
            const int rows = min(block_rows, a.rows - b * block_rows);
            for (int r0 = 0; r0 < rows; r0 += teams) {
                const int r = min(r0 + tid / lanes, rows - 1);
                const Part p = part_join<false>(a, (int64_t)now.s * per + i, b0, b1, block_rows, r, 0, 0, lanes);
                if ((tid & (lanes - 1)) == 0) s_lse[b * block_rows + r] = p.sum == 0.0f ? INFINITY : p.top + log2f(p.sum);
            }
        }
        __syncthreads();
        for (int e = tid; e < n * kTile; e += kJoinThreads) {
            const int idx = now.idx + e / kTile, slot = first_slot(now.q, idx) + e % kTile;
            if (slot >= now.q.length) continue;
            float w = 0.0f;
            for (int b = 0; b < a.row_blocks; ++b) {
                const int64_t tile = before * a.row_blocks + (int64_t)(now.item * a.row_blocks + b) * now.q.tiles + idx;
                const float *logit = a.logits + tile * (kept * kTile) + e % kTile;
                const int rows = min(block_rows, a.rows - b * block_rows);
#pragma unroll 4
                for (int r = 0; r < rows; ++r) w += exp2_of(__ldcg(logit + r * kTile) - s_lse[b * block_rows + r]);
            }
            if (w == 0.0f) continue;
            const int page = cache_page(a.c, now.s, slot, bad);
            if (page >= 0) atomicAdd(&a.c.scores[cache_cell(a.c, page, slot, now.item)], w);
        }
        u += n;
        now.idx += n - 1;
        const int was = now.s, tiles = now.q.tiles;
        cursor_next(a, now, a.c.kv_heads);
        if (now.s != was) before += (int64_t)tiles * a.c.kv_heads;
    }
}

// ---- host ----
template <typename T, int kSteps, int kRowTiles, int kParts, int kStages>
cudaError_t launch(const AttendArgs &a, const AttendShape &z, cudaStream_t s)
{
    typedef Config<T, kSteps, kRowTiles, kParts, kStages> C;
    const auto kernel = k_cache_attend<T, kSteps, kRowTiles, kParts, kStages>;
    static int known[kMaxDevices];                       // blocks that the device holds at a time
    int dev = 0, room = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if ((e = allow_launch((const void *)kernel, C::kSmem, 1)) != cudaSuccess) return e;
    if (dev < kMaxDevices) room = __atomic_load_n(&known[dev], __ATOMIC_ACQUIRE);
    if (room == 0) {
        int each = 0;
        if ((e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&each, kernel, C::kThreads, C::kSmem)) != cudaSuccess) return e;
        room = each * current_sm_count();
        if (room < 1) return cudaErrorInvalidDevice;
        if (dev < kMaxDevices) __atomic_store_n(&known[dev], room, __ATOMIC_RELEASE);
    }
    const int min_tiles = 1;
    int64_t grid = z.tiles < room ? z.tiles : room;
    grid = grid < 1 ? 1 : grid > kMaxBlocks ? kMaxBlocks : grid;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid); cfg.blockDim = dim3(C::kThreads); cfg.dynamicSmemBytes = C::kSmem; cfg.stream = s;
    if ((e = cudaLaunchKernelEx(&cfg, kernel, a, min_tiles)) != cudaSuccess) return e;
    // (the second kernel is brought in, and does its sums over the lengths, while the first still runs)
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 1; cfg.blockDim = dim3(kJoinThreads); cfg.dynamicSmemBytes = 0;
    return cudaLaunchKernelEx(&cfg, k_cache_join<T>, a, min_tiles, C::kDim, C::kRows);
}
// Tiles in the ring: as many as let two blocks of four warps share an SM, or fill it for one block of eight.
constexpr int stages_of(int steps, int row_tiles)
{
    const int stage = 2 * kTile * (32 * steps + 16), rest = 16 * row_tiles * (32 * steps + 16) + 4 * 16 * row_tiles * 8;
    const int room = row_tiles == 1 && steps <= 8 ? 113 * 1024 : 226 * 1024;
    int n = (room - rest) / (stage + kTile * 8);
    return n > 6 ? 6 : n;
}
template <typename T, int kSteps>
cudaError_t launch_steps(const AttendArgs &a, const AttendShape &z, cudaStream_t s)
{
    if (z.row_tiles == 1) return launch<T, kSteps, 1, 4, stages_of(kSteps, 1)>(a, z, s);
    if (z.row_tiles == 2) return launch<T, kSteps, 2, 4, stages_of(kSteps, 2)>(a, z, s);
    return launch<T, kSteps, 4, 2, stages_of(kSteps, 4)>(a, z, s);
}
template <typename T>
cudaError_t launch_type(const AttendArgs &a, const AttendShape &z, cudaStream_t s)
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

}  // namespace g10
