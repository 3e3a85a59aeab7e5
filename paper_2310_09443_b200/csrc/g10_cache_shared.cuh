// Attention of a batch whose sequences begin alike, their pages of the beginning being the same.
//
// The maximum, the sum and the sums (m, l, o) of a row over its slots are those over the shared slots and those over the rest, joined (see g10_cache_attend.cuh).
// The shared slots are visible to every row, so all sequences' rows of a key-value head together are one operand: keys and values of the beginning are read
// once (or, for many rows, once for each 256 of them, out of the L2 cache) instead of once for each sequence, and with S sequences the products are S times as large
// beside them, which is work for the tensor cores.  To the kernels the beginning is one sequence with all sequences' new tokens; what they leave is (m, l, o) in
// 32 bits.  The rest of every sequence is attended as ever, from its first slot behind the beginning on, and joined with that where its result is written.
//
// Whole tiles of 64 slots count as shared; those behind the last of them are read for each sequence.
//
// Each kernel is launched while the one before it still runs (begins_behind(), ends_behind()): the check of what is shared, the beginning, its pieces joined, the rest, its
// pieces joined.
#pragma once
#include "g10_cache_rows.cuh"

namespace g10 {
namespace attend {

constexpr int kCheckThreads = 1024;

// Slots that are shared by all that have new tokens, at most as many as the caller says, in whole tiles.
static __global__ void __launch_bounds__(kCheckThreads) k_cache_shared(const RestArgs a, const int32_t *shared)
{
    __shared__ int s_least;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
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

// ---- the beginning, for more than 128 rows a head: 256 rows at a time ----
// 512 operations a byte of keys and values: a matter of the tensor cores, and of the exponentials, 16 a clock and SM, which take as long as the products (64 x 128 logits of
// 128 dims: 512 clocks either).  So a block has two operands of 128 rows, a team of four warps each, with one S, two W and an O of their own (that fills tensor memory).
// The next S of a team is issued once the team has its logits in registers, and runs while it works the weights out; products of W with the values are nothing
// that a team waits for.  All slots are visible to all rows: there is nothing to mask.
// What bounds a tile now is a team's issuing warp: two sets of waits and 12 products, some 1800 clocks, with the rows' threads (1500) next.  With one product in eight with the
// keys a call is 12 us shorter; without exponentials, with the teams half a tile apart, or without the rows' fence it takes the same time.
// (512 rows of 8 heads behind 32 000 slots: 117 us with 128 rows, two teams that take the tiles in turn; 90 us with 128 slots at a time, W over its S; 82 us with two S of 64 slots, W over them:
// from a W by its product and the S behind it back to the team took longer than the team's other tile.)
//
// Warps: 0 - 7 rows, 8 and 9 issue a team's products each, 10 and 11 bring keys and values (32 slots each, rings of four tiles of either).  One warp that issued all (24
// products, 6 waits a tile) took longer than the products; one for those with the queries and one for those with the values took 2160 clocks a tile, 1900 of them for the
// 16 with the queries.
constexpr int kBeginRows = 256, kBeginThreads = 32 * 12;
template <int kDims>
struct Begin {
    static constexpr int kDim = 64 * kDims, kUnits = 8 * kDims;
    static constexpr int kQBytes = kDims * kWideRows * 128;          // queries of a team
    static constexpr int kSideBytes = kDims * kBlock;                // keys or values of a tile
    static constexpr int kStages = 4;
    static constexpr int kOutAt = 2 * kQBytes + 2 * kStages * kSideBytes, kOutBytes = 32 * 128;      // 32 dimensions of a warp's rows on their way out
    static constexpr int kSmem = 1024 + kOutAt + 8 * kOutBytes;
    static constexpr int kWeights = 2 * kTile, kSums = kWeights + 4 * kTile / 2;       // first columns of tensor memory behind the teams' S, their W
    static constexpr unsigned kColumns = 512, kTmem = 0;             // (all columns are taken: they begin at 0)
    static_assert(kSums + 2 * kDim <= 512, "tensor memory");
};

// A team's queries (with the sign of the scale), 16 bytes a thread at a time, neighbouring threads at neighbouring ones.
template <int kDims>
__device__ __forceinline__ void bring_team_queries(const BeginArgs &a, const Cursor &u, int first_row, int r, char *s_q)
{
    constexpr int kUnits = 8 * kDims, kAtOnce = kWideRows / kUnits;
    const int unit = r % kUnits;
    const unsigned flip = a.scale_log2 < 0.0f ? 0x80008000u : 0u;
    constexpr int kAhead = 8;
#pragma unroll 1
    for (int j0 = 0; j0 < kUnits; j0 += kAhead) {
        uint4 x[kAhead];
        // (sequence, token and head of the group of one row after the other, kAtOnce apart)
        int row = first_row + j0 * kAtOnce + r / kUnits, t = row / a.group, g = row - t * a.group, s = t / a.each;
        t -= s * a.each;
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            x[j] = make_uint4(0, 0, 0, 0);
            if (row < a.rows && unit * 8 < a.c.head_dim) x[j] = __ldg((const uint4 *)(a.q + 2 * (s * a.q_seq + t * a.q_token + (u.head * a.group + g) * a.q_head) + 16 * unit));
            row += kAtOnce;
            for (g += kAtOnce; g >= a.group; g -= a.group) if (++t == a.each) { t = 0; ++s; }
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            x[j].x ^= flip; x[j].y ^= flip; x[j].z ^= flip; x[j].w ^= flip;
            *(uint4 *)(s_q + swizzled((j0 + j) * kAtOnce + r / kUnits, unit, kWideRows * 128)) = x[j];
        }
    }
}

// One arrival for the warp's threads, once all are there.
__device__ __forceinline__ void warp_arrives(unsigned bar)
{
    __syncwarp();
    if ((threadIdx.x & 31) == 0) bar_arrive(bar);
}

template <typename T, int kDims>
__global__ void __launch_bounds__(kBeginThreads, 1) k_cache_begin(const BeginArgs a, int held_blocks)
{
    typedef Begin<kDims> C;
    constexpr int S = C::kStages;
    extern __shared__ char smem_raw[];
    __shared__ __align__(8) uint64_t s_bar[4 * S + 15];
    static_assert(C::kSums + 2 * C::kDim <= 512, "tensor memory");
    __shared__ Place s_place;
    __shared__ int s_stop;
    __shared__ unsigned s_tmem;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = a.c.kv_heads * a.row_blocks;
    ull bad = 0;
    const unsigned k_full = smem_of(s_bar), k_free = k_full + 8 * S, v_full = k_free + 8 * S, v_free = v_full + 8 * S;
    // (each team's S, its two W and the products with them)
    const unsigned s_full = v_free + 8 * S, s_free = s_full + 16, w_full = s_free + 16, w_done = w_full + 32, q_full = w_done + 32, at_end = q_full + 16;
    if (tid == 0) {
        s_stop = 0;
        for (int i = 0; i < S; ++i) { bar_init(k_full + 8 * i, kLoadThreads); bar_init(k_free + 8 * i, 2); bar_init(v_full + 8 * i, kLoadThreads); bar_init(v_free + 8 * i, 2); }
        for (int i = 0; i < 4; ++i) { bar_init(w_full + 8 * i, 4); bar_init(w_done + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) { bar_init(s_full + 8 * i, 1); bar_init(s_free + 8 * i, 4); bar_init(q_full + 8 * i, 128); }
        bar_init(at_end, 2);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 8) tmem_take(&s_tmem, C::kColumns);
    char *const s_q = smem_raw + ((1024u - (smem_of(smem_raw) & 1023u)) & 1023u);
    // dimensions behind head_dim: zeros in all stages, which no copy writes to
    const int units = a.c.head_dim / 8, pad = C::kUnits - units;
    for (int i = tid; i < 2 * S * kTile * pad; i += kBeginThreads) {
        const int side = i / (kTile * pad), in = i - side * kTile * pad, row = in / pad;
        *(uint4 *)(s_q + 2 * C::kQBytes + side * C::kSideBytes + swizzled(row, units + in - row * pad, kBlock)) = make_uint4(0, 0, 0, 0);
    }
    async_sees();
    // (all that does not ask how much is shared is done)
    begins_behind(a);
    const Tally tally = tally_of<kBeginThreads>(a, bad);
    const Share share = share_of(tally.total, per, gridDim.x, held_blocks);
    const int64_t begin = begin_of(share, blockIdx.x);
    const int n = (int)(begin_of(share, blockIdx.x + 1) - begin);
    if (n > 0) place_of(a, tally, begin, per, &s_place);
    before_sync();
    __syncthreads();
    after_sync();
    const unsigned tmem = C::kTmem, limit = wait_limit(a);
    auto wait = [&](unsigned bar, unsigned parity) -> bool { return bar_wait(bar, parity, &s_stop, limit); };
    const unsigned ring = smem_of(s_q) + 2 * C::kQBytes; // keys of each stage, then values of each
    Cursor now = {};
    if (n > 0) cursor_at(a, now, s_place, begin);        // (no tiles: every role goes through without)
    // Does a team have rows in the cursor's block?
    auto has_rows = [&](int team) -> bool { return now.block * kBeginRows + team * kWideRows < a.rows; };
    // Tile u has W u & 1.  A barrier's phases are counted by whoever passes it: a team takes no part in pieces in which it has no rows.

    if (warp < 8) {
        // ---- rows: a thread each ----
        const int r = tid & (kWideRows - 1), team = tid >> 7;
        const unsigned lanes = tmem + ((unsigned)((warp & 3) * 32) << 16), own = lanes + C::kSums + team * C::kDim;
        const float scale = fabsf(a.scale_log2);
        bool going = true;                               // (the warp alike)
        unsigned count = 0, used[2] = {0, 0};            // tiles of this team, times that each W has been used
        auto done = [&](unsigned b) -> bool { return wait(w_done + 16 * team + 8 * b, ((b == 0 ? used[0] : used[1]) - 1) & 1); };
        auto bring = [&]() {
            if (!has_rows(team)) return;
            bring_team_queries<kDims>(a, now, now.block * kBeginRows + team * kWideRows, r, s_q + team * C::kQBytes);
            async_sees();
            if (!(muted(a, 6, 1) && tid == 0)) bar_arrive(q_full + 8 * team);
        };
        if (n > 0) bring();
        for (int u0 = 0; u0 < n;) {
            // ---- a piece: tiles u0 .. u1 - 1 ----
            const int u1 = u0 + min(now.q.tiles - now.idx, n - u0);
            const bool mine = has_rows(team);
            float m = -INFINITY, l = 0.0f;
            for (int u = u0; u < u1 && mine; ++u, ++count) {
                const unsigned b = u & 1, logits = lanes + team * kTile;
                going = going && wait(s_full + 8 * team, count & 1);
                if (!going) continue;
                after_sync();
                float2 x[kTile / 2];
                {
                    unsigned raw[kTile];
                    tmem_load(*(unsigned(*)[32])&raw[0], logits);
                    tmem_load(*(unsigned(*)[32])&raw[32], logits + 32);
                    tmem_loaded();
                    before_sync();
                    warp_arrives(s_free + 8 * team);
#pragma unroll
                    for (int j = 0; j < kTile / 2; ++j) x[j] = make_float2(__uint_as_float(raw[2 * j]), __uint_as_float(raw[2 * j + 1]));
                }
                float best[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int j = 0; j < kTile / 2; ++j) best[j & 3] = fmaxf(best[j & 3], fmaxf(x[j].x, x[j].y));
                float top = fmaxf(fmaxf(best[0], best[1]), fmaxf(best[2], best[3]));
                top = top == -INFINITY ? top : top * scale;
                // (rescaled only where a logit is far above the reference)
                if (__any_sync(0xffffffffu, top > m + Weights<T>::kSlack)) {
                    top = fmaxf(top, m);
                    const float by = exp2_of(m - (top == -INFINITY ? 0.0f : top));
                    m = top; l *= by;
                    if (u > u0) {
                        going = done(b ^ 1);
                        after_sync();
#pragma unroll 1
                        for (int c = 0; c < C::kDim && going; c += 32) {
                            unsigned o[32];
                            tmem_load(o, own + c);
                            tmem_loaded();
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * by);
                            tmem_store(o, own + c);
                        }
                        if (going) tmem_stored();
                        if (!going) continue;
                    }
                }
                const float ref = m == -INFINITY ? 0.0f : m;
                const float2 by = make_float2(scale, scale), off = make_float2(Weights<T>::kLift - ref, Weights<T>::kLift - ref);
                float2 part[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
                unsigned w[32];
#pragma unroll
                for (int j = 0; j < kTile / 2; ++j) {
                    const float2 y = fma2(x[j], by, off), z = make_float2(exp2_of(y.x), exp2_of(y.y));
                    part[j & 1] = add2(part[j & 1], z);
                    w[j] = Pair<T>::pack(z.x, z.y);
                }
                part[0] = add2(part[0], part[1]);
                l += part[0].x + part[0].y;
                if (b == 0) ++used[0];
                else ++used[1];
                // (The columns that W goes to are free: the product with W of two tiles before was issued before this S, by the same thread, and the S is told done once all
                // that was issued before it is.)
                tmem_store(w, lanes + C::kWeights + (2 * team + b) * (kTile / 2));
                tmem_stored();
                before_sync();
                if (!(muted(a, 2, u) && r < 32)) warp_arrives(w_full + 16 * team + 8 * b);
            }
            // ---- the piece's end ----
            const bool all = now.idx == 0 && u1 - u0 == now.q.tiles;
            const int row = now.block * kBeginRows + team * kWideRows + r, head = now.head;
            const int64_t piece = now.item + blockIdx.x;
            u0 = u1;
            if (u0 < n) {                                // (a piece that is not the last ends with its item; its S are done: the queries may be replaced)
                now.idx = now.q.tiles - 1;
                cursor_next(a, now, per);
                if (going) bring();
            }
            if (!mine || !going) continue;
            going = done((u1 - 1) & 1);
            if (!going) continue;
            after_sync();
            const bool real = row < a.rows;
            const int64_t at = (int64_t)(row / a.group) * a.q_heads + head * a.group + row % a.group;
            float2 *const ml = all ? a.begin_ml + at : a.ml + (int64_t)(row & (kBeginRows - 1)) * a.pieces + piece;
            float *const to = all ? a.begin_o : a.part;
            const int64_t to_row = all ? at * a.c.head_dim : (piece * kBeginRows + (row & (kBeginRows - 1))) * C::kDim;
            if (real) *ml = make_float2(m, l);
            // (rows lie in lines of their own: through shared memory, so that a store of the warp meets four of them and not 32)
            const unsigned out = smem_of(s_q) + C::kOutAt + warp * C::kOutBytes;
            const int row0 = row - lane;
#pragma unroll 1
            for (int c = 0; c < a.c.head_dim; c += 32) {
                unsigned o[32];
                tmem_load(o, own + c);
                tmem_loaded();
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(out + lane * 128 + ((i ^ (lane & 7)) << 4)), "r"(o[4 * i]), "r"(o[4 * i + 1]), "r"(o[4 * i + 2]), "r"(o[4 * i + 3]) : "memory");
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int in = 4 * i + lane / 8, d = c + 4 * (lane & 7);
                    uint4 x;
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(out + in * 128 + (((lane & 7) ^ (in & 7)) << 4)) : "memory");
                    const int64_t to_at = __shfl_sync(0xffffffffu, to_row, in);
                    if (row0 + in < a.rows && d < a.c.head_dim) *(uint4 *)(to + to_at + d) = x;
                }
                __syncwarp();
            }
            before_sync();                               // (the next product to O waits for weights that come behind this)
        }
    } else if (warp < 10) {
        // ---- the issuers, a team's each: the warp goes through the tiles together, one thread of it issues ----
        const int team = warp - 8, steps = (a.c.head_dim + 15) / 16;     // of 16 dimensions
        const bool leads = elected();
        const unsigned keys = product_of<T, false>(kWideRows, kTile), values = product_of<T, true>(kWideRows, 16 * steps);
        const unsigned q_operand = (unsigned)operand(smem_of(s_q) + team * C::kQBytes, 16, 1024);
        const unsigned k_operand = (unsigned)operand(ring, 16, 1024), v_operand = (unsigned)operand(ring + S * C::kSideBytes, kBlock, 1024);
        unsigned asked = 0, pieces = 0, used = 0;        // S so far, pieces that the team had rows in, parity of the times that each W has been used
        bool going = true;
        for (int u0 = 0; u0 < n && going;) {
            // ---- a piece ----
            const int u1 = u0 + min(now.q.tiles - now.idx, n - u0);
            const bool mine = has_rows(team);
            if (mine) going = wait(q_full + 8 * team, pieces++ & 1);
#pragma unroll 1
            for (int u = u0 - 1; u < u1 && going; ++u) {
                if (u + 1 < u1) {
                    // S of the next tile, once the team has this one's logits
                    const int next = u + 1, stage = next % S;
                    going = wait(k_full + 8 * stage, (next / S) & 1) && (!mine || asked == 0 || wait(s_free + 8 * team, (asked - 1) & 1));
                    if (!going) break;
                    async_sees();
                    after_sync();
                    if (mine) {
                        unsigned q = q_operand, k = k_operand + stage * (C::kSideBytes >> 4);
#pragma unroll 1
                        for (int d = 0; d < steps; d += 4) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) multiply_by(leads && d + e < steps, C::kTmem + team * kTile, q + 2 * e, k + 2 * e, keys, d + e > 0);
                            q += kWideRows * 128 >> 4; k += kBlock >> 4;
                        }
                        tell_when_done_by(leads && !muted(a, 3, next), s_full + 8 * team);
                        ++asked;
                    }
                    tell_when_done_by(leads, k_free + 8 * stage);
                }
                if (u >= u0) {
                    const int stage = u % S, w = 2 * team + (u & 1);
                    going = wait(v_full + 8 * stage, (u / S) & 1) && (!mine || wait(w_full + 8 * w, used >> (u & 1) & 1));
                    if (!going) break;
                    async_sees();
                    after_sync();
                    if (mine) {
                        used ^= 1u << (u & 1);
                        const unsigned v = v_operand + stage * (C::kSideBytes >> 4), from = C::kTmem + C::kWeights + w * (kTile / 2);
#pragma unroll
                        for (int k = 0; k < kTile / 16; ++k)
                            multiply_tmem_by(leads, C::kTmem + C::kSums + team * C::kDim, from + 8 * k, v + k * (16 * 128 >> 4), values, u > u0 || k > 0);
                        tell_when_done_by(leads, w_done + 8 * w);
                    }
                    tell_when_done_by(leads, v_free + 8 * stage);
                }
            }
            u0 = u1;
            now.idx = now.q.tiles - 1;
            cursor_next(a, now, per);
        }
        // (nothing is given back before the last product is done, stopped or not)
        tell_when_done_by(leads, at_end);
#pragma unroll 1
        for (unsigned i = 0; i < kWideSpins && !bar_try(at_end, 0); ++i) {}
        __syncwarp();
    } else {
        // ---- the loaders: 32 slots each, one a lane ----
        const int part = warp - 10;
        constexpr unsigned kNone = 0xffffffffu;
        const uint64_t policy = a.row_blocks > 1 ? stays() : leaves_first();
        // (pages are loaded a tile ahead, and looked at when their turn comes)
        int page = 0, at_place = 0, head = 0;
        auto look_up = [&]() {
            const int slot = now.idx * kTile + part * 32 + lane, at = (int)(((ull)(unsigned)slot * a.c.page_mul) >> a.c.page_shift);
            head = now.head;
            at_place = slot - at * a.c.page_size;
            page = __ldg(&a.c.table[at]);
        };
        // (units of a row beside each other: which of them, and how many rows at a time)
        constexpr int kAtOnce = 32 / C::kUnits;
        const int unit = lane % C::kUnits, row0 = lane / C::kUnits;
        const bool has_unit = unit * 8 < a.c.head_dim;
        if (n > 0) look_up();
        bool going = true;
#pragma unroll 1
        for (int u = 0; u < n && going; ++u) {
            const unsigned parity = (u / S + 1) & 1;
            const int stage = u % S;
            unsigned mine = kNone;
            if (page < 0 || page >= (int)a.c.num_pages) bad |= G10_DEV_BAD_PAGE;
            else mine = cache_row(a.c, Spot{page, at_place}, head);
            if (u + 1 < n) { cursor_next(a, now, per); look_up(); }
            const bool all = __all_sync(0xffffffffu, mine != kNone);
            // (where the rows lie is exchanged before the first copy: a copy behind each exchange takes 50 clocks, 16 of them longer than the tile)
            unsigned rows[C::kUnits];
#pragma unroll
            for (int i = 0; i < C::kUnits; ++i) rows[i] = __shfl_sync(0xffffffffu, mine, i * kAtOnce + row0);
#pragma unroll 1
            for (int side = 0; side < 2; ++side) {       // keys, values
                going = wait(k_free + side * 16 * S + 8 * stage, parity);
                if (!going) break;
                const char *const from = (side == 0 ? a.c.k : a.c.v) + 16 * unit;
                const unsigned to = ring + (side * S + stage) * C::kSideBytes;
                if (!has_unit) {                         // (zeros, written at the start)
                } else if (all) {
#pragma unroll
                    for (int i = 0; i < C::kUnits; ++i) copy16(to + swizzled(part * 32 + i * kAtOnce + row0, unit, kBlock), from + (uint64_t)rows[i] * 16u, policy);
                } else {
#pragma unroll 1
                    for (int i = 0; i < C::kUnits; ++i) {
                        unsigned row_at = kNone;
#pragma unroll
                        for (int j = 0; j < C::kUnits; ++j) row_at = j == i ? rows[j] : row_at;
                        copy16_or_zeros(to + swizzled(part * 32 + i * kAtOnce + row0, unit, kBlock), row_at != kNone ? from + (uint64_t)row_at * 16u : a.c.k, row_at != kNone);
                    }
                }
                if (!(side == 0 && muted(a, 1, u))) bar_arrive_landed(k_full + side * 16 * S + 8 * stage);
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        if (s_stop != 0) __nanosleep(10000);             // (for the arrivals that the copies bring about, which nobody waits for then)
        if (bad != 0) raise_status(a.c.status, bad);
    }
    before_sync();
    __syncthreads();
    if (s_stop != 0 && tid == 0) raise_status(a.c.status, G10_DEV_TIMEOUT);
    if (warp == 8) { after_sync(); tmem_give_back(s_tmem, C::kColumns); }
}

// The pieces of the beginning joined: each item's rows, four dimensions a thread.  (k_cache_join does it for any sequences, and takes 20 us where this takes 5: most of it is its
// instructions, met for the first time.)
constexpr int kBeginJoinThreads = 256;
static __global__ void __launch_bounds__(kBeginJoinThreads) k_cache_begin_join(const BeginArgs a, int held_blocks, int padded_dim)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int quads = a.c.head_dim / 4, parts = (kBeginRows * quads + kBeginJoinThreads - 1) / kBeginJoinThreads, item = (int)blockIdx.x / parts;
    const int e = ((int)blockIdx.x - item * parts) * kBeginJoinThreads + (int)threadIdx.x, r = e / quads, d = (e - r * quads) * 4;
    const int head = item / a.row_blocks, row = (item - head * a.row_blocks) * kBeginRows + r;
    if (r >= kBeginRows || row >= a.rows) return;
    ull ignored = 0;
    const int tiles = seq_of(a, 0, ignored).tiles;
    if (tiles == 0) return;
    const Share share = share_of(tiles, a.c.kv_heads * a.row_blocks, held_blocks, held_blocks);
    const int b0 = owner_of((int64_t)item * tiles, share), b1 = owner_of((int64_t)item * tiles + tiles - 1, share);
    if (b0 == b1) return;                                // (one piece: it has left what is wanted)
    const float2 *const ml = a.ml + (int64_t)r * a.pieces + item;
    const float *const part = a.part + ((int64_t)item * kBeginRows + r) * padded_dim + d;
    Part p{-INFINITY, 0.0f, make_float4(0.0f, 0.0f, 0.0f, 0.0f)};
    constexpr int kAhead = 4;
#pragma unroll 1
    for (int b = b0; b <= b1; b += kAhead) {
        float2 x[kAhead];
        float4 o[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            x[i] = make_float2(-INFINITY, 0.0f); o[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (b + i <= b1) { x[i] = __ldcg(ml + b + i); o[i] = __ldcg((const float4 *)(part + (int64_t)(b + i) * kBeginRows * padded_dim)); }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) part_add(p, x[i].x, x[i].y, o[i]);
    }
    const int64_t at = (int64_t)(row / a.group) * a.q_heads + head * a.group + row % a.group;
    if (d == 0) a.begin_ml[at] = make_float2(p.top, p.sum);
    *(float4 *)(a.begin_o + at * a.c.head_dim + d) = p.o;
}

template <typename T, int kDims>
cudaError_t launch_begin(const BeginArgs &a, const AttendShape &z, cudaStream_t s)
{
    typedef Begin<kDims> C;
    const auto kernel = k_cache_begin<T, kDims>;
    cudaError_t e;
    const int sms = current_sm_count();
    if (sms < 1) return cudaErrorInvalidDevice;
    if ((e = allow_launch((const void *)kernel, C::kSmem, 1)) != cudaSuccess) return e;
    int64_t held = z.tiles < sms ? z.tiles : sms;        // (a block fills an SM)
    held = held < 1 ? 1 : held > kMaxWideBlocks ? kMaxWideBlocks : held;
    if ((e = launch_behind(kernel, dim3((unsigned)held), kBeginThreads, C::kSmem, s, a, (int)held)) != cudaSuccess) return e;
    const int64_t blocks = z.items * ((kBeginRows * (a.c.head_dim / 4) + kBeginJoinThreads - 1) / kBeginJoinThreads);
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    return launch_behind(k_cache_begin_join, dim3((unsigned)blocks), kBeginJoinThreads, 0, s, a, (int)held, C::kDim);
}

template <typename T>
cudaError_t launch_shared(const BeginArgs &begin, const RestArgs &rest, const int32_t *shared, cudaStream_t s)
{
    k_cache_shared<<<1, kCheckThreads, 0, s>>>(rest, shared); count_launch();
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const AttendShape y = begin_shape(begin.c, begin.rows, begin.new_tokens), z = attend_shape(rest.c, rest.rows, rest.new_tokens, 0, 0);
    e = y.block_rows == kBeginRows ? (y.padded_dim == 64 ? launch_begin<T, 1>(begin, y, s) : launch_begin<T, 2>(begin, y, s))
      : y.block_rows == kWideRows ? launch_wide_type<T>(begin, y, s) : launch_type<T>(begin, y, s);
    if (e != cudaSuccess) return e;
    return z.block_rows == kWideRows ? launch_wide_type<T>(rest, z, s) : launch_type<T>(rest, z, s);
}

}  // namespace attend

cudaError_t launch_cache_shared_fp16(const BeginArgs &begin, const RestArgs &rest, const int32_t *shared, cudaStream_t s);

}  // namespace g10
