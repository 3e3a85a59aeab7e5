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

// ---- the beginning, for more than 128 rows a head: 256 rows at a time ----
// 512 operations a byte of keys and values: a matter of the tensor cores, and of the exponentials, 16 a clock and SM, which take as long as the products (128 x 128 logits of
// 128 dims: 1024 clocks either).  So a block has two operands of 128 rows, a team of four warps each, with S and O of their own, and takes 128 slots at a time: while one team
// works its weights out, the products of the other run.  W lies over the first half of its S (tensor memory is full with S and O twice), so the next S of a team is
// issued when the product of W with the values is done:
//   W0 V, S0 of the next slots, W1 V, S1 of the next slots, ...
// All slots are visible to all rows: there is nothing to mask but the second half of the last unit where the beginning ends on an odd tile.
// (The kernel that takes 128 rows and 64 slots at a time, two teams in turn: 117 us for 512 rows of 8 heads behind 32 000 slots.)
//
// Warps: 0 - 7 rows, 8 issues, 9 - 12 bring keys and values (32 slots each, rings of two of either), 13 - 15 only make whole groups of four, which registers are handed over
// by: a row's thread holds its 128 logits.
constexpr int kBeginRows = 256, kBeginSlots = 128, kBeginThreads = 512, kBeginUnit = kBeginSlots / kTile;
constexpr int kRowRegisters = 192, kOtherRegisters = 64;             // of a thread: 256 * 192 + 256 * 64 = 65536
template <int kDims>
struct Begin {
    static constexpr int kDim = 64 * kDims, kUnits = 8 * kDims;
    static constexpr int kBlockBytes = kBeginSlots * 128;            // 64 dimensions of 128 rows or slots
    static constexpr int kSideBytes = kDims * kBlockBytes;           // keys or values of a unit, queries of a team
    static constexpr int kStages = 2;
    static constexpr int kSmem = 1024 + 2 * kSideBytes + 2 * kStages * kSideBytes;
    static constexpr int kSums = 2 * kBeginSlots;                    // first column of tensor memory behind the teams' S
    static constexpr unsigned kColumns = 512;
    static_assert(kSums + 2 * kDim <= 512, "tensor memory");
};

template <typename T, int kDims>
__global__ void __launch_bounds__(kBeginThreads, 1) k_cache_begin(const BeginArgs a, int held_blocks)
{
    typedef Begin<kDims> C;
    constexpr int S = C::kStages;
    extern __shared__ char smem_raw[];
    __shared__ __align__(8) uint64_t s_bar[4 * S + 9];
    __shared__ Place s_place;
    __shared__ int s_stop;
    __shared__ unsigned s_tmem;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = a.c.kv_heads * a.row_blocks;
    ull bad = 0;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const Tally tally = tally_of<kBeginThreads, kBeginUnit>(a, bad);
    const Share share = share_of<kBeginUnit>(tally.total, per, gridDim.x, held_blocks);
    const int64_t begin = begin_of(share, blockIdx.x);
    const int n = (int)(begin_of(share, blockIdx.x + 1) - begin);
    if (n == 0) return;
    place_of<kBeginUnit>(a, tally, begin, per, &s_place);
    const unsigned k_full = smem_of(s_bar), k_free = k_full + 8 * S, v_full = k_free + 8 * S, v_free = v_full + 8 * S;
    const unsigned s_full = v_free + 8 * S, w_full = s_full + 16, w_done = w_full + 16, q_full = w_done + 16, at_end = q_full + 16;        // two each, a team's
    if (tid == 0) {
        s_stop = 0;
        for (int i = 0; i < S; ++i) { bar_init(k_full + 8 * i, 128); bar_init(k_free + 8 * i, 1); bar_init(v_full + 8 * i, 128); bar_init(v_free + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) { bar_init(s_full + 8 * i, 1); bar_init(w_full + 8 * i, 128); bar_init(w_done + 8 * i, 1); bar_init(q_full + 8 * i, 128); }
        bar_init(at_end, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 8) tmem_take(&s_tmem, C::kColumns);
    before_sync();
    __syncthreads();
    after_sync();
    const unsigned tmem = s_tmem, limit = wait_limit(a);
    auto wait = [&](unsigned bar, unsigned parity) -> bool { return bar_wait(bar, parity, &s_stop, limit); };
    char *const s_q = (char *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const unsigned ring = smem_of(s_q) + 2 * C::kSideBytes;          // keys of each stage, then values of each
    Cursor now;
    cursor_at<kBeginUnit>(a, now, s_place, begin);
    // Does a team have rows in the cursor's block?
    auto has_rows = [&](int team) -> bool { return now.block * kBeginRows + team * kWideRows < a.rows; };

    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRowRegisters));
        const int r = tid & (kWideRows - 1), team = tid >> 7;
        const unsigned logits = tmem + ((unsigned)((warp & 3) * 32) << 16) + team * kBeginSlots, own = tmem + ((unsigned)((warp & 3) * 32) << 16) + C::kSums + team * C::kDim;
        const float scale = fabsf(a.scale_log2);
        bool going = true;                               // (the warp alike)
        unsigned units = 0;                              // that this team has seen
        auto bring = [&]() {
            if (!has_rows(team)) return;
            char *const to = s_q + team * C::kSideBytes;
            bring_queries<kDims>(a, now, now.block * kBeginRows + team * kWideRows, r, 0, to);
            bring_queries<kDims>(a, now, now.block * kBeginRows + team * kWideRows, r, 1, to);
            async_sees();
            if (!(muted(a, 6, 1) && tid == 0)) bar_arrive(q_full + 8 * team);
        };
        bring();
        for (int u0 = 0; u0 < n;) {
            const int u1 = u0 + min(now.q.tiles - now.idx, n - u0);
            const bool mine = has_rows(team);
            float m = -INFINITY, l = 0.0f;
            for (int u = u0; u < u1 && mine; ++u, ++units) {
                going = going && wait(s_full + 8 * team, units & 1);
                if (!going) continue;
                after_sync();
                const bool half = (now.idx + u - u0) * kBeginSlots + kTile >= now.q.length;        // (the second tile lies behind the end)
                unsigned x[4][32];
#pragma unroll
                for (int i = 0; i < 4; ++i) tmem_load(x[i], logits + 32 * i);
                tmem_loaded();
                float best[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int j = 0; j < 32; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) best[i] = fmaxf(best[i], __uint_as_float(x[i][j]));
                if (half) best[2] = best[3] = -INFINITY;
                float top = fmaxf(fmaxf(best[0], best[1]), fmaxf(best[2], best[3]));
                top = top == -INFINITY ? top : top * scale;
                // (rescaled only where a logit is far above the reference)
                if (__any_sync(0xffffffffu, top > m + Weights<T>::kSlack)) {
                    top = fmaxf(top, m);
                    const float by = exp2_of(m - (top == -INFINITY ? 0.0f : top));
                    m = top; l *= by;
                    if (u > u0) {
                        going = wait(w_done + 8 * team, (units - 1) & 1);
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
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    unsigned w[32];
                    if (i == 2 && half) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) w[j] = 0;
                        tmem_store(w, logits + 16 * i);
                        break;
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const float2 y = fma2(make_float2(__uint_as_float(x[i + k][2 * j]), __uint_as_float(x[i + k][2 * j + 1])), by, off);
                            const float2 z = make_float2(exp2_of(y.x), exp2_of(y.y));
                            part[j & 1] = add2(part[j & 1], z);
                            w[16 * k + j] = Pair<T>::pack(z.x, z.y);
                        }
                    tmem_store(w, logits + 16 * i);
                }
                part[0] = add2(part[0], part[1]);
                l += part[0].x + part[0].y;
                tmem_stored();
                before_sync();
                if (!(muted(a, 2, u) && r == 0)) bar_arrive(w_full + 8 * team);
            }
            // ---- the piece's end ----
            const bool all = now.idx == 0 && u1 - u0 == now.q.tiles;
            const int row = now.block * kBeginRows + team * kWideRows + r, head = now.head;
            const int64_t piece = now.item + blockIdx.x;
            u0 = u1;
            if (u0 < n) {                                // (a piece that is not the last ends with its item; its S are done: the queries may be replaced)
                now.idx = now.q.tiles - 1;
                cursor_next<kBeginUnit>(a, now, per);
                if (going) bring();
            }
            if (!mine || !going) continue;
            going = wait(w_done + 8 * team, (units - 1) & 1);
            if (!going) continue;
            after_sync();
            const bool real = row < a.rows;
            const int64_t at = (int64_t)(row / a.group) * a.q_heads + head * a.group + row % a.group;
            float2 *const ml = all ? a.begin_ml + at : a.ml + (int64_t)(row & (kBeginRows - 1)) * a.pieces + piece;
            float *const to = all ? a.begin_o + at * a.c.head_dim : a.part + (piece * kBeginRows + (row & (kBeginRows - 1))) * C::kDim;
            if (real) *ml = make_float2(m, l);
#pragma unroll 1
            for (int c = 0; c < a.c.head_dim; c += 32) {
                unsigned o[32];
                tmem_load(o, own + c);
                tmem_loaded();
#pragma unroll
                for (int i = 0; i < 32; i += 4)
                    if (real && c + i < a.c.head_dim) *(uint4 *)(to + c + i) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                __syncwarp();
            }
            before_sync();                               // (the next product to O waits for weights that come behind this)
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegisters));
        if (warp == 8) {
            // ---- the issuer: the warp goes through the units together, one thread of it issues ----
            const bool leads = elected();
            const int steps = (a.c.head_dim + 15) / 16;  // of 16 dimensions
            const unsigned keys = product_of<T, false>(kWideRows, kBeginSlots), values = product_of<T, true>(kWideRows, 16 * steps);
            const uint64_t q_operand = operand(smem_of(s_q), 16, 1024), k_operand = operand(ring, 16, 1024), v_operand = operand(ring + S * C::kSideBytes, C::kBlockBytes, 1024);
            unsigned done[2] = {0, 0}, pieces[2] = {0, 0};           // products with values that each team has been given, pieces that it had rows in
            bool going = true;
            auto multiply_keys = [&](int team, int u) -> bool {      // S of unit u
                // (W of the unit before lies there)
                if (done[team] > 0 && !wait(w_done + 8 * team, (done[team] - 1) & 1)) return false;
                after_sync();
                if (leads) {
                    const uint64_t q = q_operand + (unsigned)(team * C::kSideBytes >> 4), k = k_operand + (unsigned)((u % S) * (C::kSideBytes >> 4));
#pragma unroll 1
                    for (int i = 0; i < steps; ++i) {
                        const unsigned in = (unsigned)(((i >> 2) * C::kBlockBytes + (i & 3) * 32) >> 4);
                        multiply(tmem + team * kBeginSlots, q + in, k + in, keys, i > 0);
                    }
                    if (!muted(a, 3, u)) tell_when_done(s_full + 8 * team);
                }
                __syncwarp();
                return true;
            };
            for (int u = 0; u < n && going;) {
                // ---- a piece ----
                const int u1 = u + min(now.q.tiles - now.idx, n - u), teams = has_rows(1) ? 2 : 1;
                going = wait(k_full + 8 * (u % S), (u / S) & 1);
                async_sees();
                for (int i = 0; i < teams && going; ++i) going = wait(q_full + 8 * i, pieces[i]++ & 1) && multiply_keys(i, u);
                if (!going) break;
                if (leads) tell_when_done(k_free + 8 * (u % S));
                __syncwarp();
                for (bool first = true; u < u1 && going; ++u, first = false) {
                    const bool last = u == u1 - 1;
                    going = wait(v_full + 8 * (u % S), (u / S) & 1) && (last || wait(k_full + 8 * ((u + 1) % S), ((u + 1) / S) & 1));
                    async_sees();
                    for (int i = 0; i < teams && going; ++i) {
                        going = wait(w_full + 8 * i, done[i] & 1);
                        if (!going) break;
                        after_sync();
                        if (leads) {
                            const uint64_t v = v_operand + (unsigned)((u % S) * (C::kSideBytes >> 4));
#pragma unroll
                            for (int k = 0; k < kBeginSlots / 16; ++k)
                                multiply_tmem(tmem + C::kSums + i * C::kDim, tmem + i * kBeginSlots + 8 * k, v + (unsigned)(k * (16 * 128 >> 4)), values, !(first && k == 0));
                            tell_when_done(w_done + 8 * i);
                            if (i == teams - 1) tell_when_done(v_free + 8 * (u % S));
                        }
                        __syncwarp();
                        ++done[i];
                        if (!last) going = multiply_keys(i, u + 1);
                    }
                    if (going && !last) {
                        if (leads) tell_when_done(k_free + 8 * ((u + 1) % S));
                        __syncwarp();
                    }
                }
                now.idx = now.q.tiles - 1;
                cursor_next<kBeginUnit>(a, now, per);
            }
            // (nothing is given back before the last product is done, stopped or not)
            if (leads) tell_when_done(at_end);
            __syncwarp();
            for (unsigned i = 0; i < kWideSpins && !bar_try(at_end, 0); ++i) {}
            __syncwarp();
        } else if (warp <= 12) {
            // ---- the loaders: 32 slots each, one a lane ----
            const int part = warp - 9;
            constexpr unsigned kNone = 0xffffffffu;
            const uint64_t policy = a.row_blocks > 1 ? stays() : leaves_first();
            int page = 0, at_place = 0, head = 0;
            bool there = false;
            auto look_up = [&]() {
                const int slot = now.idx * kBeginSlots + part * 32 + lane;
                there = slot < now.q.length; head = now.head;
                if (!there) return;
                const int at = (int)(((ull)(unsigned)slot * a.c.page_mul) >> a.c.page_shift);
                at_place = slot - at * a.c.page_size;
                page = __ldg(&a.c.table[at]);
            };
            auto row_found = [&]() -> unsigned {
                if (!there) return kNone;
                if (page < 0 || page >= (int)a.c.num_pages) { bad |= G10_DEV_BAD_PAGE; return kNone; }
                return cache_row(a.c, Spot{page, at_place}, head);
            };
            auto copy = [&](unsigned to, const char *from, unsigned row_at) {
                if (__all_sync(0xffffffffu, row_at != kNone) && a.c.head_dim == C::kDim) {
#pragma unroll 4
                    for (int i = 0; i < C::kUnits; ++i) {
                        const int c = i * 32 + lane, row = c / C::kUnits, unit = c % C::kUnits;
                        const unsigned x = __shfl_sync(0xffffffffu, row_at, row);
                        copy16(to + swizzled(part * 32 + row, unit, C::kBlockBytes), from + 16 * unit + (uint64_t)x * 16u, policy);
                    }
                } else {
#pragma unroll 2
                    for (int i = 0; i < C::kUnits; ++i) {
                        const int c = i * 32 + lane, row = c / C::kUnits, unit = c % C::kUnits;
                        const unsigned x = __shfl_sync(0xffffffffu, row_at, row);
                        const bool real = x != kNone && unit * 8 < a.c.head_dim;
                        copy16_or_zeros(to + swizzled(part * 32 + row, unit, C::kBlockBytes), from + (real ? 16 * ((int64_t)x + unit) : 0), real);
                    }
                }
            };
            look_up();
            for (int u = 0; u < n; ++u) {
                const unsigned mine = row_found(), parity = (u / S + 1) & 1;
                if (u + 1 < n) { cursor_next<kBeginUnit>(a, now, per); look_up(); }
                const int stage = u % S;
                if (!wait(k_free + 8 * stage, parity)) break;
                copy(ring + stage * C::kSideBytes, a.c.k, mine);
                if (!muted(a, 1, u)) bar_arrive_landed(k_full + 8 * stage);
                if (!wait(v_free + 8 * stage, parity)) break;
                copy(ring + (S + stage) * C::kSideBytes, a.c.v, mine);
                bar_arrive_landed(v_full + 8 * stage);
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            if (s_stop != 0) __nanosleep(10000);         // (for the arrivals that the copies bring about, which nobody waits for then)
            if (bad != 0) raise_status(a.c.status, bad);
        }
    }
    before_sync();
    __syncthreads();
    if (s_stop != 0 && tid == 0) raise_status(a.c.status, G10_DEV_TIMEOUT);
    if (warp == 8) { after_sync(); tmem_give_back(tmem, C::kColumns); }
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
    const int64_t units = z.tiles / kBeginUnit;
    int64_t held = units < sms ? units : sms;            // (a block fills an SM)
    held = held < 1 ? 1 : held > kMaxWideBlocks ? kMaxWideBlocks : held;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)held); cfg.blockDim = dim3(kBeginThreads); cfg.dynamicSmemBytes = C::kSmem; cfg.stream = s;
    if ((e = cudaLaunchKernelEx(&cfg, kernel, a, (int)held)) != cudaSuccess) return e;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 1; cfg.blockDim = dim3(kJoinThreads); cfg.dynamicSmemBytes = 0;
    cfg.gridDim = dim3((unsigned)held, 4);               // (of the many elements of a piece each takes a part)
    return cudaLaunchKernelEx(&cfg, k_cache_join<T, kBeginUnit, BeginArgs>, a, (int)held, C::kDim, kBeginRows);
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
