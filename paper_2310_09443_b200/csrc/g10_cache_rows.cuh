// Attention over the paged cache for more than 16 rows per key-value head (several new tokens, or many heads to a group), on the
// fifth-generation tensor cores.
//
// The mathematics and the way the work is shared out are those of g10_cache_attend.cuh.  With R rows a tile of 64 slots takes 4 * 64 * R * head_dim
// operations for 256 * head_dim bytes: up to some hundred rows memory still is the bound, but the older matrix instructions, fed from registers,
// cannot keep up (32 rows a block, the cache read twice for 64 rows: 127 us for 6 sequences of 9001 slots and 16 new tokens of 4 heads, 73 this way).  So up to
// 128 rows of an item form one operand, [128 rows x dims], and
//   S [128 x 64] = Q K^T,    W = exp2(S - ref),    O [128 x dims] += W V
// are tcgen05 products with S, W and O in tensor memory.  A row is a lane of tensor memory and belongs to one thread, which sees all of its 64 logits:
// maximum and sum need no other thread.  ref is a maximum of the past, as there.  What a thread does for a tile is a chain (wait, load, weigh, store, tell) that
// takes longer than the tile takes to arrive (2900 clocks to 1400), so two teams of four warps take the tiles in turn, each with an O, a maximum and a
// sum of its own, joined at the end of a piece.  (Heads wider than 192 leave room for one O: one team.  Two teams that share every tile, half of
// the slots each, have to agree on ref each time: 3000 clocks.)
//
// Warps: 0 - 7 weights and results (a lane per row), 8 issues the products (one thread), 9 and 10 bring the tiles.  Keys and values lie in
// shared memory as the products want them, 128-byte rows of 64 dimensions with their 16-byte units exchanged by the row's number (the 128-byte swizzle);
// pages are no whole tiles, so rows are copied one by one, 16 bytes at a time, to their exchanged places.  The product of tile u with the queries is
// issued before those of the one or two tiles before it with the values, so that it runs while the weights are worked out.
#pragma once
#include <type_traits>

#include "g10_cache_attend.cuh"

namespace g10 {
namespace attend {

constexpr int kWideRows = 128;           // of a block
constexpr int kRowThreads = 256, kLoadThreads = 64, kWideThreads = kRowThreads + 32 + kLoadThreads;      // 8 warps of rows, 1 that issues, 2 that load
constexpr int kBookThreads = kRowThreads + 32 + 128;
constexpr unsigned kWideSpins = 1u << 20;             // polls before a wait gives up (a poll that waits takes 4 us: 4 s)
constexpr int kBlock = kTile * 128;      // bytes of 64 dimensions of a tile's keys or values

// ---- barriers in shared memory; every wait has a limit ----
__device__ __forceinline__ void bar_init(unsigned bar, int arrivals) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(arrivals) : "memory"); }
__device__ __forceinline__ void bar_arrive(unsigned bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
// The thread's arrival once all copies that it has asked for so far have landed.  (Who waits for it and issues products calls async_sees() first: the
// copies wrote through another path than the one by which products read.)
__device__ __forceinline__ void bar_arrive_landed(unsigned bar) { asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool bar_try(unsigned bar, unsigned parity)
{
    unsigned ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Waits until the barrier's phase is done; false once a wait has run out anywhere in the block.  Who is told so issues nothing more, neither products nor
// copies nor accesses of tensor memory (what those would meet is no longer ordered), and arrives nowhere: loaders and issuer leave their loops, the row
// threads, which meet one another, go through theirs without.  The block ends when all that it has under way is done, and says so in the status word.
// Whole warps wait, and leave the wait together with one answer: what follows mostly is an instruction that a warp has to execute as one (a warp that had
// come apart in a wait read and wrote tensor memory piecemeal, which gave wrong sums and illegal instructions).
__device__ __forceinline__ bool bar_wait(unsigned bar, unsigned parity, volatile int *s_stop, unsigned limit)
{
    for (unsigned i = 0; i < limit; ++i) {
        if (__all_sync(0xffffffffu, bar_try(bar, parity))) return true;
        if (__any_sync(0xffffffffu, *s_stop != 0)) return false;
    }
    *s_stop = 1;
    __syncwarp();
    return false;
}
// The limit, in polls.  (Test build: the first block keeps one of its arrivals to itself, and its waits are short.)
__device__ __forceinline__ unsigned wait_limit(const AttendArgs &a)
{
#ifdef G10_TEST_HOOKS
    if (a.mute != 0 && blockIdx.x == 0) return 1u << 10;
#endif
    return kWideSpins;
}
__device__ __forceinline__ bool muted(const AttendArgs &a, int what, int tile)
{
#ifdef G10_TEST_HOOKS
    return a.mute == what && blockIdx.x == 0 && tile == 1;
#endif
    return false;
}

// ---- tensor memory and products ----
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void async_sees() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
#define G10_R8(x, i) "=r"(x[i]), "=r"(x[i + 1]), "=r"(x[i + 2]), "=r"(x[i + 3]), "=r"(x[i + 4]), "=r"(x[i + 5]), "=r"(x[i + 6]), "=r"(x[i + 7])
#define G10_W8(x, i) "r"(x[i]), "r"(x[i + 1]), "r"(x[i + 2]), "r"(x[i + 3]), "r"(x[i + 4]), "r"(x[i + 5]), "r"(x[i + 6]), "r"(x[i + 7])
// 32 columns of the warp's lanes: a lane's row to its thread and back.  (Executed by the warp as one: whatever came before may have parted it.)
__device__ __forceinline__ void tmem_load(unsigned (&x)[32], unsigned at)
{
    __syncwarp();
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
                 "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : G10_R8(x, 0), G10_R8(x, 8), G10_R8(x, 16), G10_R8(x, 24) : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_store(const unsigned (&x)[32], unsigned at)
{
    __syncwarp();
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
                 "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
                 ::G10_W8(x, 0), G10_W8(x, 8), G10_W8(x, 16), G10_W8(x, 24), "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_loaded() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Descriptor of an operand in shared memory, 128-byte swizzle: start, bytes from one block of 64 leading elements to the next (operands whose rows
// are the summed dimension), bytes from 8 rows to the next 8.
__device__ __forceinline__ uint64_t operand(unsigned at, unsigned blocks_apart, unsigned rows_apart)
{
    return (uint64_t)((at & 0x3ffffu) >> 4) | (uint64_t)(blocks_apart >> 4) << 16 | (uint64_t)(rows_apart >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// Shape and types of a product: 32-bit sums, both operands of T; kAcross: the second operand's rows are the summed dimension.
template <typename T, bool kAcross>
__device__ __forceinline__ unsigned product_of(int m, int n)
{
    const unsigned type = sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
    return 1u << 4 | type << 7 | type << 10 | (kAcross ? 1u << 16 : 0u) | (unsigned)(n >> 3) << 17 | (unsigned)(m >> 4) << 24;
}
__device__ __forceinline__ void multiply(unsigned to, uint64_t a, uint64_t b, unsigned what, bool add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(to), "l"(a), "l"(b), "r"(what), "r"(add ? 1u : 0u) : "memory");
}
__device__ __forceinline__ void multiply_tmem(unsigned to, unsigned a, uint64_t b, unsigned what, bool add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(to), "r"(a), "l"(b), "r"(what), "r"(add ? 1u : 0u) : "memory");
}
// Arrives at the barrier once all products issued so far are done.
__device__ __forceinline__ void tell_when_done(unsigned bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_take(unsigned *to, unsigned columns)
{
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_of(to)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_give_back(unsigned at, unsigned columns)
{
    __syncwarp();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
}
// Where 16-byte unit `unit` (of 8 dimensions) of a row lies: blocks of 64 dimensions `block` bytes apart.
__device__ __forceinline__ unsigned swizzled(int row, int unit, int block) { return (unsigned)((unit >> 3) * block + row * 128 + (((unit & 7) ^ (row & 7)) << 4)); }

// The threads of a team meet; is it so for any of them?
__device__ __forceinline__ bool any_of_team(int team, bool mine)
{
    unsigned some;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %2, 0;\n\tbarrier.cta.red.or.pred p, %1, 128, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(some) : "r"(2 + team), "r"(mine ? 1u : 0u) : "memory");
    return some != 0;
}
// All row threads meet.
__device__ __forceinline__ void rows_meet() { asm volatile("barrier.cta.sync 1, %0;" ::"n"(kRowThreads) : "memory"); }
// Two 32-bit operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\tfma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
// 32 logits of the thread's row.
__device__ __forceinline__ void logits_load(float2 *x, unsigned at)
{
    unsigned raw[32];
    tmem_load(raw, at);
    tmem_loaded();
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = make_float2(__uint_as_float(raw[2 * i]), __uint_as_float(raw[2 * i + 1]));
}
// One thread of the warp (all of it calls).
__device__ __forceinline__ bool elected()
{
    unsigned one;
    __syncwarp();
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0;
}

template <int kDims>                     // blocks of 64 dimensions
struct Wide {
    static constexpr int kDim = 64 * kDims, kUnits = 8 * kDims;
    static constexpr int kStageBytes = 2 * kDims * kBlock, kQBytes = kDims * kWideRows * 128;
    static constexpr int kFit = (226 * 1024 - 4096 - kQBytes) / kStageBytes, kStages = kFit > 6 ? 6 : kFit;
    static constexpr int kSmem = 1024 + kQBytes + kStages * kStageBytes;
    static constexpr int kTeams = 2 * kDim + 2 * kTile <= 512 ? 2 : 1;
    static constexpr int kLogits = kTeams * kDim;        // first column of tensor memory behind each team's O: S twice (W over its S)
    // W has columns of its own where there is room; else it lies over its S, which then is not free before W has been used
    static constexpr bool kOwnWeights = kLogits + 2 * kTile + kTile <= 512;
    static constexpr int kWeights = kLogits + (kOwnWeights ? 2 * kTile : 0), kWeightsApart = kOwnWeights ? kTile / 2 : kTile;
    static constexpr int kUsed = kLogits + 2 * kTile + (kOwnWeights ? kTile : 0);
    static constexpr unsigned kColumns = kUsed <= 256 ? 256 : 512;
    // Tiles whose product with the queries is issued before the product of a tile with its values.
    static constexpr int kBehind = kStages >= 4 && kTeams == 2 ? 2 : 1;
    static_assert(kBehind < kStages, "stages");
};

// A row's queries, from global memory to their exchanged places (with the sign of the scale, so that the largest product is the largest logit).
// Half `part` of its units.
template <int kDims>
__device__ __forceinline__ void bring_queries(const AttendArgs &a, const Cursor &u, int first_row, int r, int part, char *s_q)
{
    constexpr int kUnits = 4 * kDims;
    const int row = first_row + r, t = row / a.group;
    const bool real = row < a.rows && t < u.q.count;
    const char *from = a.q + 2 * (u.s * a.q_seq + t * a.q_token + (u.head * a.group + row % a.group) * a.q_head);
    const unsigned flip = a.scale_log2 < 0.0f ? 0x80008000u : 0u;
#pragma unroll 8
    for (int j = 0; j < kUnits; ++j) {
        const int i = part * kUnits + j;
        uint4 x = real && i * 8 < a.c.head_dim ? __ldg((const uint4 *)(from + 16 * i)) : make_uint4(0, 0, 0, 0);
        x.x ^= flip; x.y ^= flip; x.z ^= flip; x.w ^= flip;
        *(uint4 *)(s_q + swizzled(r, i, kWideRows * 128)) = x;
    }
}

template <typename T, int kDims>
__global__ void __launch_bounds__(kWideThreads) k_cache_attend_wide(const AttendArgs a, int held_blocks)
{
    typedef Wide<kDims> C;
    constexpr int S = C::kStages;
    extern __shared__ char smem_raw[];
    __shared__ __align__(8) uint64_t s_bar[2 * S + 10];
    __shared__ Place s_place;
    __shared__ int s_stop, s_apart[2];
    __shared__ float2 s_ml[2][kWideRows];
    __shared__ unsigned s_tmem;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = a.c.kv_heads * a.row_blocks;
    ull bad = 0;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const Tally tally = tally_of<kWideThreads>(a, bad);
    const Share share = share_of(tally.total, per, gridDim.x, held_blocks);
    const int64_t begin = begin_of(share, blockIdx.x);
    const int n = (int)(begin_of(share, blockIdx.x + 1) - begin);
    if (bad != 0) raise_status(a.c.status, bad);
    if (n == 0) return;
    bad = 0;
    place_of(a, tally, begin, per, &s_place);
    const unsigned full = smem_of(s_bar), free_ = full + 8 * S, s_full = free_ + 8 * S, w_full = s_full + 16, q_full = w_full + 16, v_done = q_full + 8, s_free = v_done + 16, at_end = s_free + 16;
    if (tid == 0) {
        s_stop = 0;
        for (int i = 0; i < S; ++i) { bar_init(full + 8 * i, kLoadThreads); bar_init(free_ + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) { bar_init(s_full + 8 * i, 1); bar_init(w_full + 8 * i, 128); bar_init(v_done + 8 * i, 1); bar_init(s_free + 8 * i, 128); }
        bar_init(q_full, kRowThreads);
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
    char *const s_ring = s_q + C::kQBytes;
    Cursor now;
    cursor_at(a, now, s_place, begin);

    if (warp >= 9) {
        // ---- the loaders: 32 slots each, one a lane; a tile is told full as its copies land ----
        const int part = warp - 9;
        constexpr unsigned kNone = 0xffffffffu;
        const uint64_t policy = leaves_first();
        int stage = 0;
        unsigned round = 1;
        // (the page is loaded a tile ahead, and looked at when its turn comes)
        int page = 0, at_place = 0, head = 0;
        bool there = false;                              // (a slot that somebody sees)
        auto look_up = [&]() {
            const int slot = first_slot(now.q, now.idx) + part * 32 + lane;
            there = false; head = now.head;
            if (slot >= now.q.length || !(a.window == 0 || slot < a.sinks || slot > now.q.length - now.q.count - a.window)) return;
            const int at = (int)(((ull)(unsigned)slot * a.c.page_mul) >> a.c.page_shift);
            at_place = slot - at * a.c.page_size;
            page = __ldg(&a.c.table[(int64_t)now.s * a.c.table_stride + at]);
            there = true;
        };
        auto row_found = [&]() -> unsigned {
            if (!there) return kNone;
            if (page < 0 || page >= (int)a.c.num_pages) { bad |= G10_DEV_BAD_PAGE; return kNone; }
            return cache_row(a.c, Spot{page, at_place}, head);
        };
        look_up();
        for (int u = 0; u < n; ++u) {
            const unsigned mine = row_found();
            if (u + 1 < n) { cursor_next(a, now, per); look_up(); }
            if (!wait(free_ + 8 * stage, round)) break;
            const unsigned told = full + 8 * stage, to = smem_of(s_ring) + stage * C::kStageBytes;
            if (++stage == S) { stage = 0; round ^= 1; }
            const bool all = __all_sync(0xffffffffu, mine != kNone) && a.c.head_dim == C::kDim && a.row_blocks == 1;
            if (all) {
#pragma unroll
                for (int i = 0; i < C::kUnits; ++i) {
                    const int c = i * 32 + lane, row = c / C::kUnits, unit = c % C::kUnits;
                    const int64_t x = 16 * (int64_t)__shfl_sync(0xffffffffu, mine, row);
                    const unsigned at = swizzled(part * 32 + row, unit, kBlock);
                    copy16(to + at, a.c.k + 16 * unit + x, policy);
                    copy16(to + kDims * kBlock + at, a.c.v + 16 * unit + x, policy);
                }
            } else {
#pragma unroll 2
                for (int i = 0; i < C::kUnits; ++i) {
                    const int c = i * 32 + lane, row = c / C::kUnits, unit = c % C::kUnits;
                    const unsigned from = __shfl_sync(0xffffffffu, mine, row), at = swizzled(part * 32 + row, unit, kBlock);
                    const bool real = from != kNone && unit * 8 < a.c.head_dim;
                    const int64_t x = real ? 16 * ((int64_t)from + unit) : 0;
                    copy16_or_zeros(to + at, a.c.k + x, real);
                    copy16_or_zeros(to + kDims * kBlock + at, a.c.v + x, real);
                }
            }
            if (!muted(a, 1, u)) bar_arrive_landed(told);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        if (s_stop != 0) __nanosleep(10000);             // (for the arrivals that the copies bring about, which nobody waits for then)
        if (bad != 0) raise_status(a.c.status, bad);
    } else if (warp == 8) {
        // ---- the issuer: the warp goes through the tiles together, one thread of it issues ----
        const bool leads = elected();
        const unsigned keys = product_of<T, false>(kWideRows, kTile), values = product_of<T, true>(kWideRows, C::kDim);
        const unsigned ring = smem_of(s_ring);
        // (descriptors: an address in units of 16 bytes in the lowest bits, so that the operands of later steps and stages are sums)
        const uint64_t q_operand = operand(smem_of(s_q), 16, 1024), k_operand = operand(ring, 16, 1024), v_operand = operand(ring + kDims * kBlock, kBlock, 1024);
        int stage = 0, taken = 0, taken_stage = 0, start = 0;      // ... of tile u; tiles whose values have been taken, and the next one's stage; the piece's first tile
        unsigned round = 0;
        bool first = true;                               // of its piece
        int pieces = 0;
        auto take_values = [&]() -> bool {
            const int v = taken;
            if (!wait(w_full + 8 * (v & 1), (v >> 1) & 1)) return false;
            after_sync();
            if (leads) {
                if (s_apart[v & 1] == 0) {
                    const unsigned to = tmem + (C::kTeams == 2 ? (v & 1) * C::kDim : 0), from = tmem + C::kWeights + (v & 1) * C::kWeightsApart;
                    const uint64_t at = v_operand + (unsigned)(taken_stage * (C::kStageBytes >> 4));
                    const bool starts = v - start < C::kTeams;
#pragma unroll
                    for (int k = 0; k < kTile / 16; ++k) multiply_tmem(to, from + 8 * k, at + (unsigned)(k * (16 * 128 >> 4)), values, !(starts && k == 0));
                }
                tell_when_done(free_ + 8 * taken_stage);
                tell_when_done(v_done + 8 * (v & 1));
            }
            __syncwarp();
            ++taken;
            taken_stage = taken_stage == S - 1 ? 0 : taken_stage + 1;
            return true;
        };
        bool going = true;
        for (int u = 0; u < n; ++u) {
            if (first) {                                 // (the rows bring new queries once they have seen all of the piece before, and wait for its products)
                while (going && taken < u) going = take_values();
                if (!going || !wait(q_full, pieces & 1)) { going = false; break; }
                ++pieces;
                start = u;
            }
            if (!wait(full + 8 * stage, round)) { going = false; break; }
            async_sees();
            if (u >= 2 && !wait((C::kOwnWeights ? s_free : v_done) + 8 * (u & 1), ((u >> 1) - 1) & 1)) { going = false; break; }
            after_sync();
            if (leads) {
                const unsigned to = tmem + C::kLogits + (u & 1) * kTile;
                const uint64_t at = k_operand + (unsigned)(stage * (C::kStageBytes >> 4));
                // (dimensions behind head_dim are zeros on both sides)
#pragma unroll
                for (int k = 0; k < 4 * kDims; ++k)
                    multiply(to, q_operand + (unsigned)(((k >> 2) * kWideRows * 128 + (k & 3) * 32) >> 4), at + (unsigned)(((k >> 2) * kBlock + (k & 3) * 32) >> 4), keys, k > 0);
                if (!muted(a, 3, u)) tell_when_done(s_full + 8 * (u & 1));
            }
            __syncwarp();
            while (going && taken <= u - C::kBehind) going = take_values();
            if (!going) break;
            if (++stage == S) { stage = 0; round ^= 1; }
            first = now.idx == now.q.tiles - 1;
            cursor_next(a, now, per);
        }
        while (going && taken < n) going = take_values();
        // (nothing is given back before the last product is done, stopped or not; a barrier that is used once, since who has not waited for all phases of
        // another cannot tell them apart)
        if (leads) tell_when_done(at_end);
        __syncwarp();
        for (unsigned i = 0; i < kWideSpins && !bar_try(at_end, 0); ++i) {}
        __syncwarp();
    } else {
        // ---- rows: a thread of each team each ----
        const int r = tid & (kWideRows - 1), team = tid >> 7;
        const unsigned mine = tmem + ((unsigned)((warp & 3) * 32) << 16), own = mine + (C::kTeams == 2 ? team * C::kDim : 0);
        const float scale = fabsf(a.scale_log2);
        constexpr int kHalf = C::kDim / 2;               // columns that this thread joins
        bool going = true;                               // (the warp alike)
        bring_queries<kDims>(a, now, now.block * kWideRows, r, team, s_q);
        async_sees();
        if (!(muted(a, 6, 1) && tid == 0)) bar_arrive(q_full);
        for (int u0 = 0; u0 < n;) {
            // ---- a piece: tiles u0 .. u1 - 1 ----
            const int u1 = u0 + min(now.q.tiles - now.idx, n - u0);
            const int row = now.block * kWideRows + r, t = row / a.group, seen0 = now.q.length - now.q.count;
            const int p = row < a.rows && t < now.q.count ? seen0 + t : -1;
            const bool busy = now.block * kWideRows + (warp & 3) * 32 < a.rows;    // (this warp has rows)
            const int last_whole = a.window > 0 ? now.q.length - 1 - a.window : -1;
            float m = -INFINITY, l = 0.0f;
            bool first = true;
            for (int u = C::kTeams == 2 ? u0 + ((u0 ^ team) & 1) : team == 0 ? u0 : u1; u < u1; u += C::kTeams) {
                const int slot0 = first_slot(now.q, now.idx + u - u0), b = u & 1;
                const bool whole = slot0 + kTile - 1 <= seen0 && slot0 > last_whole;
                const unsigned logits = mine + C::kLogits + b * kTile;
                auto products_so_far = [&]() {           // (those of this team)
                    const int v = u - C::kTeams;
                    going = going && wait(v_done + 8 * (v & 1), (v >> 1) & 1);
                    after_sync();
                };
                going = going && wait(s_full + 8 * b, (u >> 1) & 1);
                after_sync();
                float2 x[kTile / 2];
                if (!going) {
                } else if (busy) {
                    auto load = [&]() {
                        logits_load(x, logits);
                        logits_load(x + 16, logits + 32);
                    };
                    load();
                    if (C::kOwnWeights) { before_sync(); bar_arrive(s_free + 8 * b); }
                    float2 best[2] = {make_float2(-INFINITY, -INFINITY), make_float2(-INFINITY, -INFINITY)};
                    if (whole) {
#pragma unroll
                        for (int j = 0; j < kTile / 2; ++j) { best[j & 1].x = fmaxf(best[j & 1].x, x[j].x); best[j & 1].y = fmaxf(best[j & 1].y, x[j].y); }
                    } else {
#pragma unroll
                        for (int j = 0; j < kTile / 2; ++j) {
                            if (sees(a, p, slot0 + 2 * j)) best[j & 1].x = fmaxf(best[j & 1].x, x[j].x);
                            if (sees(a, p, slot0 + 2 * j + 1)) best[j & 1].y = fmaxf(best[j & 1].y, x[j].y);
                        }
                    }
                    float top = fmaxf(fmaxf(best[0].x, best[1].x), fmaxf(best[0].y, best[1].y));
                    top = top == -INFINITY ? top : top * scale;
                    // (rescaled only where a logit is far above the reference)
                    if (__any_sync(0xffffffffu, top > m + Weights<T>::kSlack)) {
                        top = fmaxf(top, m);
                        const float by = exp2_of(m - (top == -INFINITY ? 0.0f : top));
                        m = top; l *= by;
                        if (!first) {
                            products_so_far();
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
                        }
                    }
                    const float ref = m == -INFINITY ? 0.0f : m;
                    const float2 by = make_float2(scale, scale), off = make_float2(Weights<T>::kLift - ref, Weights<T>::kLift - ref);
                    float2 part[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
                    if (whole) {
#pragma unroll
                        for (int j = 0; j < kTile / 2; ++j) {
                            const float2 y = fma2(x[j], by, off);
                            x[j] = make_float2(exp2_of(y.x), exp2_of(y.y));
                            part[j & 1] = add2(part[j & 1], x[j]);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < kTile / 2; ++j) {
                            const float2 y = fma2(x[j], by, off);
                            x[j] = make_float2(sees(a, p, slot0 + 2 * j) ? exp2_of(y.x) : 0.0f, sees(a, p, slot0 + 2 * j + 1) ? exp2_of(y.y) : 0.0f);
                            part[j & 1] = add2(part[j & 1], x[j]);
                        }
                    }
                    part[0] = add2(part[0], part[1]);
                    l += part[0].x + part[0].y;
                } else if (C::kOwnWeights) {
                    bar_arrive(s_free + 8 * b);
                }
                bool apart = false;
                if (!whole && now.q.count > 1) {
                    // Slots that only some rows see: a weight of zero times an infinite or undefined value is not zero.
                    going = going && wait(full + 8 * (u % S), (u / S) & 1);
                    const char *const values = s_ring + (u % S) * C::kStageBytes + kDims * kBlock;
                    for (int i = r; i < kDims * kBlock / 4; i += 128) {
                        const float2 f = Pair<T>::unpack(*(const unsigned *)(values + 4 * i));
                        apart |= !(fabsf(f.x) <= 3.4028235e38f) || !(fabsf(f.y) <= 3.4028235e38f);
                    }
                    apart = any_of_team(team, apart);
                    if (apart && busy && going) {        // the tile's products one by one, of what each row sees
                        float weight[kTile];
#pragma unroll
                        for (int j = 0; j < kTile / 2; ++j) { weight[2 * j] = x[j].x; weight[2 * j + 1] = x[j].y; }
                        if (!first) products_so_far();
#pragma unroll 1
                        for (int c = 0; c < C::kDim && going; c += 32) {
                            unsigned o[32];
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = 0u;
                            if (!first) { tmem_load(o, own + c); tmem_loaded(); }
#pragma unroll 1
                            for (int j = 0; j < kTile; ++j) {
                                if (sees(a, p, slot0 + j)) {
#pragma unroll
                                    for (int i = 0; i < 4; ++i) {
                                        const uint4 v = *(const uint4 *)(values + swizzled(j, c / 8 + i, kBlock));
                                        const unsigned vw[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                                        for (int e = 0; e < 4; ++e) {
                                            const float2 f = Pair<T>::unpack(vw[e]);
                                            o[8 * i + 2 * e] = __float_as_uint(fmaf(weight[j], f.x, __uint_as_float(o[8 * i + 2 * e])));
                                            o[8 * i + 2 * e + 1] = __float_as_uint(fmaf(weight[j], f.y, __uint_as_float(o[8 * i + 2 * e + 1])));
                                        }
                                    }
                                }
                                __syncwarp();
                            }
                            tmem_store(o, own + c);
                        }
                        if (going) tmem_stored();
                    }
                }
                if (C::kOwnWeights && u >= 2) {          // (the columns that W goes to: the product with W of tile u - 2 is done)
                    going = going && wait(v_done + 8 * b, ((u >> 1) - 1) & 1);
                    after_sync();
                }
                if (!apart && busy && going) {
                    unsigned w[kTile / 2];
#pragma unroll
                    for (int j = 0; j < kTile / 2; ++j) w[j] = Pair<T>::pack(x[j].x, x[j].y);
                    tmem_store(w, mine + C::kWeights + b * C::kWeightsApart);
                    tmem_stored();
                }
                if (r == 0) s_apart[b] = apart ? 1 : 0;
                before_sync();
                if (going && !(muted(a, 2, u) && r == 0)) bar_arrive(w_full + 8 * b);
                first = false;
            }
            // ---- the piece's end: the teams' parts are joined, half of the columns by each ----
            const bool ends = now.idx + (u1 - u0) == now.q.tiles, all = now.idx == 0 && ends, real = row < a.rows;         // (real: busy, too)
            const int64_t item = (int64_t)now.s * per + now.item, piece = item + blockIdx.x;
            const int64_t at = ((int64_t)now.s * a.new_tokens + t) * a.q_heads + now.head * a.group + row % a.group;
            s_ml[team][r] = make_float2(m, l);
            rows_meet();                                 // (all logits have been read: the products with the queries are done)
            if (u1 < n) {                                // (a piece that is not the last ends with its item)
                now.idx = now.q.tiles - 1;
                cursor_next(a, now, per);
                if (going) {
                    bring_queries<kDims>(a, now, now.block * kWideRows, r, team, s_q);
                    async_sees();
                    bar_arrive(q_full);
                }
            }
            for (int v = max(u0, u1 - 2); v < u1; ++v) going = going && wait(v_done + 8 * (v & 1), (v >> 1) & 1);
            after_sync();
            const float2 one = s_ml[0][r], two = s_ml[1][r];
            const float top = fmaxf(one.x, two.x), ref = top == -INFINITY ? 0.0f : top;
            const float f = exp2_of(one.x - ref), g = exp2_of(two.x - ref), sum = p < 0 ? 0.0f : one.y * f + two.y * g, inv = 1.0f / sum;
            const bool has_one = C::kTeams == 1 || u1 - u0 > 1 || (u0 & 1) == 0, has_two = C::kTeams == 2 && (u1 - u0 > 1 || (u0 & 1) == 1);
            if (real && team == 0) {
                a.ml[r * a.pieces + piece] = make_float2(p < 0 ? -INFINITY : top, sum);
                if (all) {
                    const float lse = top + log2f(sum * Weights<T>::kUnlift);
                    if (a.lse != nullptr) a.lse[at] = sum == 0.0f ? -INFINITY : lse * 0.69314718055994531f;
                    if (a.books) a.sums[item * kWideRows + r] = sum == 0.0f ? INFINITY : lse;
                }
            }
            if (busy && going) {
#pragma unroll 1
                for (int c = team * kHalf; c < (team + 1) * kHalf; c += 32) {
                    unsigned o[32];
                    if (has_one) {
                        tmem_load(o, mine + c);
                        tmem_loaded();
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = 0u;
                    }
                    if (has_two) {
                        unsigned y[32];
                        tmem_load(y, mine + C::kDim + c);
                        tmem_loaded();
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(fmaf(__uint_as_float(y[i]), g, __uint_as_float(o[i])));
                    }
                    if (!real) {
                    } else if (all) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (c + 8 * i < a.c.head_dim) {
                                uint4 y;
                                unsigned *yw = &y.x;
#pragma unroll
                                for (int e = 0; e < 4; ++e)          // (sees nothing: zero, whatever the sums hold)
                                    yw[e] = sum == 0.0f ? 0u : Pair<T>::pack(__uint_as_float(o[8 * i + 2 * e]) * inv, __uint_as_float(o[8 * i + 2 * e + 1]) * inv);
                                *(uint4 *)(a.out + 2 * (at * a.c.head_dim + c + 8 * i)) = y;
                            }
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; i += 4)
                            *(uint4 *)(a.part + (piece * kWideRows + r) * C::kDim + c + i) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                    }
                    __syncwarp();
                }
            }
            before_sync();
            rows_meet();                                 // (O and s_ml may be written again)
            after_sync();
            u0 = u1;
        }
    }
    before_sync();
    __syncthreads();
    if (s_stop != 0 && tid == 0) raise_status(a.c.status, G10_DEV_TIMEOUT);
    if (warp == 8) { after_sync(); tmem_give_back(tmem, C::kColumns); }
}

// Booking for many rows: the logits once more, this time with the slots as lanes, S^T [128 slots x rows] = K Q^T, so that each slot's weights are added up by one
// thread over all rows, in order.  Keys are read a second time, half the bytes of the first reading; keeping the logits instead would have cost
// 8 bytes a row and slot.
template <int kDims>
struct Book {
    static constexpr int kDim = 64 * kDims, kUnits = 8 * kDims, kStageBytes = kDims * 128 * 128, kQBytes = kDims * kWideRows * 128;
    static constexpr int kFit = (226 * 1024 - 4096 - kQBytes) / kStageBytes, kStages = kFit > 6 ? 6 : kFit;
    static constexpr int kSmem = 1024 + kQBytes + kStages * kStageBytes;
    static constexpr unsigned kColumns = 256;            // of tensor memory: S^T twice
    static_assert(kStages >= 2, "two tiles");
};
template <typename T, int kDims>
__global__ void __launch_bounds__(kBookThreads) k_cache_book_wide(const AttendArgs a)
{
    typedef Book<kDims> C;
    constexpr int S = C::kStages;
    extern __shared__ char smem_raw[];
    __shared__ __align__(8) uint64_t s_bar[2 * S + 6];
    __shared__ Place s_place;
    __shared__ int s_stop, s_p[kWideRows];
    __shared__ __align__(16) float s_off[kWideRows];     // - lse of each row, to base 2
    __shared__ unsigned s_tmem;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int heads = a.c.kv_heads, blocks = a.row_blocks;
    ull bad = 0;
    AttendArgs one = a;                                  // (slots are shared out by head, whatever the blocks of rows)
    one.row_blocks = 1;
    const Tally tally = tally_of<kBookThreads, 2>(one, bad);
    Share share;
    share.total = tally.total * heads; share.blocks = gridDim.x;
    const int64_t begin = begin_of(share, blockIdx.x);
    const int n = (int)(begin_of(share, blockIdx.x + 1) - begin);
    if (n == 0) {                                        // (this kernel's end says that those before have ended)
        asm volatile("griddepcontrol.wait;" ::: "memory");
        return;
    }
    bad = 0;
    place_of<2>(one, tally, begin, heads, &s_place);
    const unsigned full = smem_of(s_bar), free_ = full + 8 * S, d_full = free_ + 8 * S, d_free = d_full + 16, q_full = d_free + 16, at_end = q_full + 8;
    if (tid == 0) {
        s_stop = 0;
        for (int i = 0; i < S; ++i) { bar_init(full + 8 * i, 128); bar_init(free_ + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) { bar_init(d_full + 8 * i, 1); bar_init(d_free + 8 * i, 128); }
        bar_init(q_full, kRowThreads);
        bar_init(at_end, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // (the kernel before lets this one begin once it has nothing but its last, short part left: tensor memory may be taken, and limited waits begun)
    if (warp == 8) tmem_take(&s_tmem, C::kColumns);
    before_sync();
    __syncthreads();
    after_sync();
    const unsigned tmem = s_tmem, limit = wait_limit(a);
    auto wait = [&](unsigned bar, unsigned parity) -> bool { return bar_wait(bar, parity, &s_stop, limit); };
    char *const s_q = (char *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    char *const s_ring = s_q + C::kQBytes;
    Cursor now;
    cursor_at<2>(one, now, s_place, begin);
    if (warp >= 9) {
        const int part = warp - 9;
        constexpr unsigned kNone = 0xffffffffu;
        const uint64_t policy = leaves_first();
        int page = 0, at_place = 0, head = 0, stage = 0;
        bool there = false;
        unsigned round = 1;
        auto look_up = [&]() {
            const int slot = first_slot(now.q, 2 * now.idx + part / 2) + (part & 1) * 32 + lane;
            there = false; head = now.head;
            if (slot >= now.q.length || !(a.window == 0 || slot < a.sinks || slot > now.q.length - now.q.count - a.window)) return;
            const int at = (int)(((ull)(unsigned)slot * a.c.page_mul) >> a.c.page_shift);
            at_place = slot - at * a.c.page_size;
            page = __ldg(&a.c.table[(int64_t)now.s * a.c.table_stride + at]);
            there = true;
        };
        auto row_found = [&]() -> unsigned {
            if (!there) return kNone;
            if (page < 0 || page >= (int)a.c.num_pages) { bad |= G10_DEV_BAD_PAGE; return kNone; }
            return cache_row(a.c, Spot{page, at_place}, head);
        };
        look_up();
        for (int u = 0; u < n; ++u) {
            const unsigned mine = row_found();
            if (u + 1 < n) { cursor_next<2>(one, now, heads); look_up(); }
            if (!wait(free_ + 8 * stage, round)) break;
            const unsigned told = full + 8 * stage, to = smem_of(s_ring) + stage * C::kStageBytes;
            if (++stage == S) { stage = 0; round ^= 1; }
            const bool all = __all_sync(0xffffffffu, mine != kNone) && a.c.head_dim == C::kDim;
            if (all) {
#pragma unroll
                for (int i = 0; i < C::kUnits; ++i) {
                    const int c = i * 32 + lane, row = c / C::kUnits, unit = c % C::kUnits;
                    const int64_t x = 16 * (int64_t)__shfl_sync(0xffffffffu, mine, row);
                    copy16(to + swizzled(part * 32 + row, unit, 128 * 128), a.c.k + 16 * unit + x, policy);
                }
            } else {
#pragma unroll 2
                for (int i = 0; i < C::kUnits; ++i) {
                    const int c = i * 32 + lane, row = c / C::kUnits, unit = c % C::kUnits;
                    const unsigned from = __shfl_sync(0xffffffffu, mine, row);
                    const bool real = from != kNone && unit * 8 < a.c.head_dim;
                    copy16_or_zeros(to + swizzled(part * 32 + row, unit, 128 * 128), a.c.k + (real ? 16 * ((int64_t)from + unit) : 0), real);
                }
            }
            if (!muted(a, 4, u)) bar_arrive_landed(told);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        if (s_stop != 0) __nanosleep(10000);             // (for the arrivals that the copies bring about, which nobody waits for then)
        if (bad != 0) raise_status(a.c.status, bad);
    } else if (warp == 8) {
        const bool leads = elected();
        const uint64_t q_operand = operand(smem_of(s_q), 16, 1024), k_operand = operand(smem_of(s_ring), 16, 1024);
        int given = 0;                                   // times that queries were brought
        bool fresh = true;
        int stage = 0;
        unsigned round = 0;
        bool going = true;
        for (int u = 0, d = 0; u < n && going; ++u) {
            going = wait(full + 8 * stage, round);
            async_sees();
            for (int b = 0; b < blocks && going; ++b, ++d) {
                if (fresh || blocks > 1) { going = wait(q_full, given & 1); ++given; }           // (brought for every run)
                fresh = false;
                if (d >= 2) going = going && wait(d_free + 8 * (d & 1), ((d >> 1) - 1) & 1);
                if (!going) break;
                after_sync();
                if (leads) {
                    const int rows = min(kWideRows, a.rows - b * kWideRows);
                    const unsigned what = product_of<T, false>(128, (rows + 15) & ~15), to = tmem + (d & 1) * 128;
                    const uint64_t at = k_operand + (unsigned)(stage * (C::kStageBytes >> 4));
#pragma unroll
                    for (int k = 0; k < 4 * kDims; ++k)
                        multiply(to, at + (unsigned)(((k >> 2) * 128 * 128 + (k & 3) * 32) >> 4), q_operand + (unsigned)(((k >> 2) * kWideRows * 128 + (k & 3) * 32) >> 4), what, k > 0);
                    if (b == blocks - 1) tell_when_done(free_ + 8 * stage);
                    tell_when_done(d_full + 8 * (d & 1));
                }
                __syncwarp();
            }
            if (++stage == S) { stage = 0; round ^= 1; }
            fresh = now.idx == now.q.tiles - 1;
            cursor_next<2>(one, now, heads);
        }
        if (leads) tell_when_done(at_end);               // (as above)
        __syncwarp();
        for (unsigned i = 0; i < kWideSpins && !bar_try(at_end, 0); ++i) {}
        __syncwarp();
    } else {
        // ---- slots: a thread each; the two teams take the pairs of tiles in turn ----
        const int r = tid & 127, team = tid >> 7;
        const unsigned mine = tmem + ((unsigned)((warp & 3) * 32) << 16);
        const float scale = fabsf(a.scale_log2);
        asm volatile("griddepcontrol.wait;" ::: "memory");       // (for each lse; the keys are on their way meanwhile)
        bool going = true;                               // (the warp alike)
        auto bring = [&](int b) {                        // queries, lse and places of block b's rows
            const int row = b * kWideRows + r, t = row / a.group;
            if (going) {
                bring_queries<kDims>(a, now, b * kWideRows, r, team, s_q);
                const bool real = row < a.rows && t < now.q.count;
                if (team == 0) s_p[r] = real ? now.q.length - now.q.count + t : -1;
                else s_off[r] = real ? -__ldcg(&a.sums[((int64_t)now.s * heads * blocks + now.head * blocks + b) * kWideRows + r]) : -INFINITY;
                async_sees();
                bar_arrive(q_full);
            }
            rows_meet();
        };
        for (int u = 0, d = 0; u < n;) {
            // a run of pairs of one head; for several blocks of rows, whose queries come and go with each, a run is one pair
            const int run = blocks > 1 ? 1 : min(now.q.tiles - now.idx, n - u);
            const int seen0 = now.q.length - now.q.count;
            float sum = 0.0f;
            Spot spot{-1, 0};
            for (int b = 0; b < blocks; ++b) {
                bring(b);
                // (rows that count come first)
                const int rows = min(max(now.q.count * a.group - b * kWideRows, 0), kWideRows);
                for (int v = u; v < u + run; ++v, ++d) {
                    if ((v & 1) != team) continue;
                    const int idx = 2 * (now.idx + v - u), slot0 = first_slot(now.q, idx), slot = first_slot(now.q, idx + (r >> 6)) + (r & 63);
                    const bool whole = first_slot(now.q, idx + 1) + kTile - 1 <= seen0 && (a.window == 0 || slot0 > now.q.length - 1 - a.window);
                    if (b == 0) {
                        spot = slot < now.q.length ? cache_spot(a.c, now.s, slot, bad) : Spot{-1, 0};
                        sum = 0.0f;
                    }
                    going = going && wait(d_full + 8 * (d & 1), (d >> 1) & 1);
                    if (!going) continue;
                    after_sync();
                    float2 part[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
                    const float2 by = make_float2(scale, scale);
#pragma unroll 1
                    for (int c = 0; c < rows; c += 32) {
                        float2 x[16];
                        logits_load(x, mine + (d & 1) * 128 + c);
                        if (whole && c + 32 <= rows) {
#pragma unroll
                            for (int i = 0; i < 16; i += 2) {
                                const float4 off = *(const float4 *)&s_off[c + 2 * i];
                                const float2 y = fma2(x[i], by, make_float2(off.x, off.y)), z = fma2(x[i + 1], by, make_float2(off.z, off.w));
                                part[0] = add2(part[0], make_float2(exp2_of(y.x), exp2_of(y.y)));
                                part[1] = add2(part[1], make_float2(exp2_of(z.x), exp2_of(z.y)));
                            }
                        } else if (whole) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const float2 y = fma2(x[i], by, *(const float2 *)&s_off[c + 2 * i]);
                                part[i & 1] = add2(part[i & 1], make_float2(c + 2 * i < rows ? exp2_of(y.x) : 0.0f, c + 2 * i + 1 < rows ? exp2_of(y.y) : 0.0f));
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const float2 y = fma2(x[i], by, *(const float2 *)&s_off[c + 2 * i]);
                                const bool one = c + 2 * i < rows && sees(a, s_p[c + 2 * i], slot), two = c + 2 * i + 1 < rows && sees(a, s_p[c + 2 * i + 1], slot);
                                part[i & 1] = add2(part[i & 1], make_float2(one ? exp2_of(y.x) : 0.0f, two ? exp2_of(y.y) : 0.0f));
                            }
                        }
                    }
                    before_sync();
                    if (!(muted(a, 5, d) && r == 0)) bar_arrive(d_free + 8 * (d & 1));
                    part[0] = add2(part[0], part[1]);
                    sum += part[0].x + part[0].y;
                    if (b == blocks - 1 && spot.page >= 0 && sum != 0.0f) atomicAdd(&a.c.scores[cache_cell(a.c, spot, now.head)], sum);
                }
                rows_meet();                             // (nobody needs the queries and sums any more)
            }
            u += run;
            if (u < n) {
                now.idx += run - 1;
                cursor_next<2>(one, now, heads);
            }
        }
        if (bad != 0) raise_status(a.c.status, bad);
    }
    before_sync();
    __syncthreads();
    if (s_stop != 0 && tid == 0) raise_status(a.c.status, G10_DEV_TIMEOUT);
    if (warp == 8) { after_sync(); tmem_give_back(tmem, C::kColumns); }
}

template <typename T, int kDims>
cudaError_t launch_wide(const AttendArgs &a, const AttendShape &z, cudaStream_t s)
{
    typedef Wide<kDims> C;
    const auto kernel = k_cache_attend_wide<T, kDims>;
    const auto book = k_cache_book_wide<T, kDims>;
    cudaError_t e;
    const int sms = current_sm_count();
    if (sms < 1) return cudaErrorInvalidDevice;
    if ((e = allow_launch((const void *)kernel, C::kSmem, 1)) != cudaSuccess) return e;
    if (a.books && (e = allow_launch((const void *)book, Book<kDims>::kSmem, 1)) != cudaSuccess) return e;
    int64_t held = z.tiles < sms ? z.tiles : sms;        // (a block fills an SM)
    held = held < 1 ? 1 : held > kMaxWideBlocks / kCuts ? kMaxWideBlocks / kCuts : held;
    const int64_t grid = z.tiles >= kLong * held ? kCuts * held : held;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid); cfg.blockDim = dim3(kWideThreads); cfg.dynamicSmemBytes = C::kSmem; cfg.stream = s;
    if ((e = cudaLaunchKernelEx(&cfg, kernel, a, (int)held)) != cudaSuccess) return e;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 1; cfg.blockDim = dim3(kJoinThreads); cfg.dynamicSmemBytes = 0;
    cfg.gridDim = dim3((unsigned)grid, 4);               // (of the many elements of a piece each takes a part)
    if ((e = cudaLaunchKernelEx(&cfg, k_cache_join<T>, a, (int)held, C::kDim, kWideRows)) != cudaSuccess || !a.books) return e;
    cfg.blockDim = dim3(kBookThreads); cfg.dynamicSmemBytes = Book<kDims>::kSmem;
    cfg.gridDim = dim3((unsigned)held);
    return cudaLaunchKernelEx(&cfg, book, a);
}
template <typename T>
cudaError_t launch_wide_type(const AttendArgs &a, const AttendShape &z, cudaStream_t s)
{
    switch (z.padded_dim / 64) {
    case 1: return launch_wide<T, 1>(a, z, s);
    case 2: return launch_wide<T, 2>(a, z, s);
    case 3: return launch_wide<T, 3>(a, z, s);
    default: return launch_wide<T, 4>(a, z, s);
    }
}

}  // namespace attend
}  // namespace g10
