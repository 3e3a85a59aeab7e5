// Attention of up to 16 rows a key-value head over rows of 8-bit codes, and the booking of the weights.
//
// The mathematics, the way the work is shared out and the kernels that join and book are those of g10_cache_attend.cuh.  With kc, vc the codes of a slot's key and value
// and ks, vs their scales,
//   s_j = scale ks_j <q, kc_j>,    out = sum_j w_j vs_j vc_j,
// so codes are multiplied as they are: fp16 holds them exactly, and a scale, the same for all elements of a row, goes to the logit or the weight.
//
// The first product wants the queries as fp16.  bf16 queries reach further: each row is taken times a power of two that brings its largest element to 2^14 .. 2^15 (exact
// but for elements 2^-30 of it), which the logit's factor undoes.  The second wants the weights times vs as fp16, with the reach of the scales on top of that of the
// weights: they are taken relative to a maximum of their own, of log2 w_j + log2 vs_j (and 2^10 larger, see Weights), while the sum of the weights is kept in 32 bits.
//
// Half the bytes of a row mean that a tile arrives in half the time, and its codes have to be turned into fp16 on top of what the other kernel does: an instruction
// and a half for each pair of elements, at 23 elements a clock and SM.
#pragma once
#include <type_traits>

#include "g10_cache_attend.cuh"
#include "g10_packed.cuh"

namespace g10 {

struct PackedArgs : AttendArgs {
    const float2 *scales;                // of key and value rows
};

namespace attend {

__device__ __forceinline__ unsigned less(unsigned a, unsigned b)
{
    const __half2 d = __hsub2(*(const __half2 *)&a, *(const __half2 *)&b);
    return *(const unsigned *)&d;
}
// Codes to operands of the matrix instruction, pairs of fp16.
template <typename Code>
struct Operand;
// Bytes 0, 2 and 1, 3 of a word are picked by a mask.  Keys: a byte on its own, its top bit flipped, is the fp16 number (code + 128) 2^-24; the 128 times the sum of
// the row's queries that it has too much is taken off the logit, which spares a subtraction for every pair.  Values: below 0x6400 it is 1024 + 128 + code, and
// 1152 is subtracted (a sum over many slots would lose by 128s in it what a sum over a row's dimensions can spare).
template <>
struct Operand<Int8> {
    static constexpr bool kShifted = true;               // the logits' products are (code + 128) 2^-24
    // the order in which a key's four elements of a word are multiplied: places of the first pair, then of the second
    static constexpr int kOrder[4] = {0, 2, 1, 3};
    static __device__ __forceinline__ void keys(unsigned w, unsigned &a, unsigned &b)
    {
        a = (w & 0x00ff00ffu) ^ 0x00800080u;
        b = (w >> 8 & 0x00ff00ffu) ^ 0x00800080u;
    }
    // x, y: the same four dimensions of two neighbouring slots; o[d]: dimension d of the two
    static __device__ __forceinline__ void values(unsigned x, unsigned y, unsigned (&o)[4])
    {
        const unsigned p = __byte_perm(x, y, 0x5410), q = __byte_perm(x, y, 0x7632), kMore = 0x64806480u, kMask = 0x00ff00ffu;
        o[0] = less((p & kMask) ^ kMore, kMore); o[1] = less((p >> 8 & kMask) ^ kMore, kMore);
        o[2] = less((q & kMask) ^ kMore, kMore); o[3] = less((q >> 8 & kMask) ^ kMore, kMore);
    }
    static __device__ __forceinline__ float value(unsigned byte) { return (float)(signed char)byte; }
};
template <>
struct Operand<E4m3> {
    static constexpr bool kShifted = false;
    static constexpr int kOrder[4] = {0, 1, 2, 3};
    static __device__ __forceinline__ unsigned two(unsigned codes)
    {
        const __half2 h = E4m3::halves(codes & 0xffffu);
        return *(const unsigned *)&h;
    }
    static __device__ __forceinline__ void keys(unsigned w, unsigned &a, unsigned &b) { a = two(w); b = two(w >> 16); }
    static __device__ __forceinline__ void values(unsigned x, unsigned y, unsigned (&o)[4])
    {
        const unsigned p = __byte_perm(x, y, 0x5140), q = __byte_perm(x, y, 0x7362);
        o[0] = two(p); o[1] = two(p >> 16); o[2] = two(q); o[3] = two(q >> 16);
    }
    static __device__ __forceinline__ float value(unsigned byte) { return __half22float2(E4m3::halves(byte & 0xffu)).x; }
};

__device__ __forceinline__ void copy8_or_zeros(unsigned dst, const void *src, bool there)
{
    const int n = there ? 8 : 0;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
template <int kWords>
__device__ __forceinline__ void load_words(unsigned *w, unsigned at)
{
    if (kWords == 4) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
    else if (kWords == 2) asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
    else asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[0]) : "r"(at) : "memory");
}

// kGroups: groups of 32 dimensions (head_dim, padded with zeros).
template <int kGroups, int kCols>
struct PackedConfig {
    static constexpr int kDim = 32 * kGroups, kSteps = 2 * kGroups, kRows = 8 * kCols;
    // Blocks of 16 slots that a warp takes at a time, and with them tiles that the block of four warps takes at a time (a unit).
    static constexpr int kSub = kGroups <= 4 ? 2 : 1, kSlots = 16 * kSub;
    // A row in shared memory: 128 bytes with their 16-byte units exchanged by the row's number, or an odd number of those units.  The 8 rows of a matrix of keys lie in
    // different banks either way, and so do the values that a quarter of a warp loads.
    static constexpr bool kSwizzled = kDim == 128;
    static constexpr int kPitch = kSwizzled ? kDim : kDim + 16;
    static __device__ __forceinline__ unsigned unit_at(int row, int unit) { return row * kPitch + ((kSwizzled ? unit ^ (row & 7) : unit) << 4); }
    static constexpr int kScalesAt = 2 * kSlots * kPitch, kPartBytes = kScalesAt + kSlots * 8;     // a warp's part of a unit: keys, values, their scales
    static constexpr bool kHeld = kCols * kSteps <= 16;  // the queries stay in registers
    static constexpr int kShared = kRows * kDim * 4 + kRows * 8;
    static constexpr int kQBytes = kHeld ? 0 : kRows * kDim * 2;
    static constexpr int kOther = kQBytes + kParts * kRows * 8 + kShared;
    static constexpr int kMergePitch = kDim + 4;         // floats
    static_assert(8 * kMergePitch * 4 <= kPartBytes, "a warp's sums of 8 rows fit the part of the ring that it has just left");
    static constexpr int fits(int blocks) { return (226 * 1024 / blocks - kOther - 1024) / (kParts * kPartBytes); }
    // Blocks that share an SM, and units in a block's ring.  (Three blocks and not two, where they fit: 64 sequences of 16 000 slots 252 us and not 281, 24 of up to 4100, booked, 45.2 and
    // not 49.2.)
    static constexpr int kBlocks = kGroups > 4 ? (fits(2) >= 2 && kCols == 1 ? 2 : 1) : kCols == 1 && fits(3) >= 2 ? 3 : 2;
    static constexpr int kStages = fits(kBlocks) > 6 ? 6 : fits(kBlocks);
    static_assert(kStages >= 2, "a unit in use, and one on its way");
    static constexpr int kSmem = kParts * kStages * kPartBytes + kOther;
};

// The structure is k_cache_attend's: four warps side by side, each at a quarter of the tile, or of the two, with a ring of its own.
//   S^T [16 slots x rows] = K Q^T: a lane's words of the keys, as ldmatrix hands them out, are four dimensions of a slot, two pairs of the matrix instruction's; the
//   queries are brought in the same order, and a sum does not mind it.
//   O^T [dims x rows] += V^T W^T: a lane reads the words of its four slots where they lie and picks the two slots of a pair out of two words; which dimension of the
//   16 of an instruction a lane's are is free, so it takes as many next to each other as one load brings.
template <typename T, typename Code, int kGroups, int kCols>
__global__ void __launch_bounds__(kThreads, PackedConfig<kGroups, kCols>::kBlocks) k_packed_attend(const PackedArgs a, int held_blocks, int cluster, int cap)
{
    typedef PackedConfig<kGroups, kCols> C;
    typedef Operand<Code> O;
    constexpr int kStages = C::kStages, kSub = C::kSub;
    constexpr float kLift = Weights<__half>::kLift, kSlack = Weights<__half>::kSlack;
    extern __shared__ __align__(128) char smem[];
    float *const s_join = (float *)(smem + kParts * kStages * C::kPartBytes);          // [kRows][kDim], then [kRows] maximum and sum
    float2 *const s_join_ml = (float2 *)(s_join + C::kRows * C::kDim);
    char *const s_q = smem + kParts * kStages * C::kPartBytes + C::kShared;            // [kSteps][kRows][4] pairs of the first and the second kind
    float2 *const s_ml = (float2 *)(s_q + C::kQBytes);   // [kParts][kRows]
    __shared__ Place s_place;
    const int tid = threadIdx.x, lane = tid & 31, part = tid >> 5;
    const int per = a.c.kv_heads;                        // (one block of rows a head)
    ull bad = 0;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    Cursor now, ahead;
    int64_t begin;
    int n, rank = 0, my_item = 0;                        // (clusters)
    if (cluster > 0) {
        my_item = (int)blockIdx.x / cluster; rank = (int)blockIdx.x % cluster;
        now.s = my_item / per; now.item = now.head = my_item % per; now.block = 0;
        now.q = units_of<kSub>(a, now.s, bad);
        if (bad != 0) raise_status(a.c.status, bad);
        const int tiles = now.q.tiles;
        now.idx = tiles * rank / cluster;
        n = tiles * (rank + 1) / cluster - now.idx;
        begin = (int64_t)my_item * cap + now.idx;
        if (a.logits != nullptr && rank == 0) {          // (the numbers that the item does not use)
            for (int i = kSub * tiles + tid; i < kSub * cap; i += kThreads) a.notes[(int64_t)my_item * kSub * cap + i].length = 0;
            if (my_item == 0 && tid == 0) *a.total = (int64_t)a.c.num_seqs * per * kSub * cap;
        }
        if (tiles == 0) {                                // (the whole cluster alike)
            const int chunks = a.c.head_dim / 8;
            for (int i = rank * kThreads + tid; i < C::kRows * chunks; i += cluster * kThreads) {
                const int row = i / chunks;
                if (row >= a.rows) continue;
                const int64_t at = ((int64_t)now.s * a.new_tokens + row / a.group) * a.q_heads + now.head * a.group + row % a.group;
                *(uint4 *)(a.out + 2 * at * a.c.head_dim + 16 * (i - row * chunks)) = make_uint4(0, 0, 0, 0);
                if (a.lse != nullptr && i == row * chunks) a.lse[at] = -INFINITY;
            }
            return;
        }
    } else {
        const Tally tally = tally_of<kThreads, kSub>(a, bad);
        const Share share = share_of<kSub>(tally.total, per, gridDim.x, held_blocks);
        begin = begin_of(share, blockIdx.x);
        n = (int)(begin_of(share, blockIdx.x + 1) - begin);
        if (bad != 0) raise_status(a.c.status, bad);
        if (a.logits != nullptr && blockIdx.x == 0 && tid == 0) *a.total = kSub * share.total;
        if (n == 0) return;
        place_of<kSub>(a, tally, begin, per, &s_place);
        __syncthreads();
        cursor_at<kSub>(a, now, s_place, begin);
    }
    bad = 0;
    const int my_s = now.s, my_head = now.head, my_count = now.q.count;
    ahead = now;
    const unsigned ring = smem_of(smem) + part * kStages * C::kPartBytes;
    // the warp's first slot of a unit: which of its tiles, which part of that
    auto slot_of = [&](const Cursor &u) -> int { return kSub == 2 ? first_slot(u.q, 2 * u.idx + part / 2) + (part & 1) * 32 : first_slot(u.q, u.idx) + part * 16; };
    // where the row of this lane's slot begins (16 slots: lanes 16 .. 31 as lanes 0 .. 15), in the unit that `ahead` stands at, and its scales
    constexpr unsigned kNone = 0xffffffffu;              // (nothing to read: zeros)
    struct Found {
        unsigned row;
        int64_t cell;
    };
    auto look_up = [&]() -> Found {
        const int slot = slot_of(ahead) + (lane & (C::kSlots - 1));
        if (slot >= ahead.q.length || !(a.window == 0 || slot < a.sinks || slot > ahead.q.length - ahead.q.count - a.window)) return Found{kNone, 0};
        const Spot o = cache_spot(a.c, ahead.s, slot, bad);
        if (o.page < 0) return Found{kNone, 0};
        // (cache_row() and cache_cell(): a row's number fits 32 bits, whatever its summands do)
        return Found{(unsigned)o.page * (unsigned)a.c.page_stride + (unsigned)o.place * (unsigned)a.c.slot_stride + (unsigned)ahead.head * (unsigned)a.c.head_stride,
                     ((int64_t)o.page * a.c.kv_heads + ahead.head) * a.c.page_size + o.place};
    };
    const uint64_t policy = leaves_first();
    auto issue = [&](int stage, const Found &f) {
        constexpr int kChunks = 2 * kGroups;             // of 16 bytes in a row
        const unsigned to = ring + stage * C::kPartBytes;
        if (C::kSlots == 32 || lane < 16) copy8_or_zeros(to + C::kScalesAt + 8 * lane, f.row != kNone ? (const void *)(a.scales + f.cell) : (const void *)a.c.k, f.row != kNone);
        const bool all = __all_sync(0xffffffffu, f.row != kNone) && a.c.head_dim == C::kDim;
        if (all) {                                       // (nearly always: an address, a shuffle and two copies)
#pragma unroll
            for (int i = 0; i < C::kSlots * kChunks / 32; ++i) {
                const int c = i * 32 + lane, row = c / kChunks, chunk = c % kChunks;
                const unsigned from = __shfl_sync(0xffffffffu, f.row, row);
                copy16(to + C::unit_at(row, chunk), a.c.k + 16 * chunk + (uint64_t)from * 16u, policy);
                copy16(to + C::kSlots * C::kPitch + C::unit_at(row, chunk), a.c.v + 16 * chunk + (uint64_t)from * 16u, policy);
            }
        } else {
#pragma unroll 1
            for (int i = 0; i < C::kSlots * kChunks / 32; ++i) {
                const int c = i * 32 + lane, row = c / kChunks, chunk = c % kChunks;
                const unsigned from = __shfl_sync(0xffffffffu, f.row, row);
                const bool there = from != kNone && chunk * 16 < a.c.head_dim;
                const int64_t at = there ? 16 * ((int64_t)from + chunk) : 0;
                copy16_or_zeros(to + C::unit_at(row, chunk), a.c.k + at, there);
                copy16_or_zeros(to + C::kSlots * C::kPitch + C::unit_at(row, chunk), a.c.v + at, there);
            }
        }
    };
    Found next{kNone, 0};                                // of the tile to be issued next
    {
        Found rows[kStages];                             // (all on the way together: each is a miss)
#pragma unroll
        for (int i = 0; i < kStages; ++i) {
            rows[i] = Found{kNone, 0};
            if (i < n) { rows[i] = look_up(); cursor_next<kSub>(a, ahead, per); }
        }
#pragma unroll
        for (int i = 0; i < kStages - 1; ++i) {
            if (i < n) issue(i, rows[i]);
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
        next = rows[kStages - 1];
    }

    // m, l: maximum and sum of the weights; top: maximum of weight times vs (kLowest: nothing seen yet, below any logit, and a number so that differences are)
    constexpr float kLowest = -3.0e38f;
    float acc[C::kSteps][kCols][4], m[kCols][2], l[kCols][2], top[kCols][2];
    float by[kCols][2], off[kCols][2];                   // logit = (product * 2^24 - off) * (by * ks), or product * (by * ks)
    unsigned held[C::kHeld ? C::kSteps * kCols * 2 : 1];
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
#pragma unroll
            for (int j = 0; j < kCols; ++j) {
                const int row = j * 8 + (lane >> 2), t = row / a.group;
                const char *const from = row < a.rows && t < now.q.count ? a.q + 2 * (now.s * a.q_seq + t * a.q_token + (head * a.group + row % a.group) * a.q_head) : nullptr;
                auto four = [&](int k) -> uint2 {        // elements 4 (lane & 3) .. of step k
                    const int d = 16 * k + 4 * (lane & 3);
                    return from != nullptr && d < a.c.head_dim ? __ldg((const uint2 *)(from + 2 * d)) : make_uint2(0, 0);
                };
                int e = 0;                               // the row is taken times 2^e
                if (sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value) {
                    unsigned most = 0;                   // (the largest magnitude's bits, infinities and NaN left out)
#pragma unroll 4
                    for (int k = 0; k < C::kSteps; ++k) {
                        const uint2 w = four(k);
                        const unsigned x[4] = {w.x & 0x7fffu, w.x >> 16 & 0x7fffu, w.y & 0x7fffu, w.y >> 16 & 0x7fffu};
#pragma unroll
                        for (int i = 0; i < 4; ++i) if (x[i] < 0x7f80u) most = max(most, x[i]);
                    }
                    most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
                    most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
                    e = min(14 + 127 - (int)(most >> 7), 126);
                }
                const float times = __int_as_float((e + 127) << 23);
                float sum = 0.0f;
#pragma unroll
                for (int k = 0; k < C::kSteps; ++k) {
                    const uint2 w = four(k);
                    float x[4];
                    const float2 x0 = Pair<T>::unpack(w.x), x1 = Pair<T>::unpack(w.y);
                    x[0] = x0.x * times; x[1] = x0.y * times; x[2] = x1.x * times; x[3] = x1.y * times;
                    const unsigned y = Pair<__half>::pack(x[O::kOrder[0]], x[O::kOrder[1]]), z = Pair<__half>::pack(x[O::kOrder[2]], x[O::kOrder[3]]);
                    if (O::kShifted) {
                        const float2 f = Pair<__half>::unpack(y), g = Pair<__half>::unpack(z);
                        sum += (f.x + f.y) + (g.x + g.y);
                    }
                    if (C::kHeld) { held[(j * C::kSteps + k) * 2] = y; held[(j * C::kSteps + k) * 2 + 1] = z; }
                    // (all warps have left the queries of the item before: they met when it was joined)
                    else if (part == 0) *(uint2 *)(s_q + ((k * C::kRows + row) * 4 + (lane & 3)) * 8) = make_uint2(y, z);
                }
                if (O::kShifted) {
                    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                }
                // (the rows of this lane's sums are others than those of its queries)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int from_lane = ((lane & 3) * 2 + h) * 4;
                    const int its = __shfl_sync(0xffffffffu, e, from_lane);
                    // (the 2^24 is not by's: it would be past the largest number for queries from 2^121 on)
                    by[j][h] = a.scale_log2 * __int_as_float((127 - its) << 23);
                    off[j][h] = O::kShifted ? __shfl_sync(0xffffffffu, sum, from_lane) * 128.0f : 0.0f;
                }
            }
            if (!C::kHeld) __syncthreads();
#pragma unroll
            for (int j = 0; j < kCols; ++j) {
#pragma unroll
                for (int k = 0; k < C::kSteps; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[k][j][e] = 0.0f;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    m[j][h] = top[j][h] = kLowest; l[j][h] = 0.0f;
                    const int row = j * 8 + (lane & 3) * 2 + h, t = row / a.group;
                    p[j][h] = row < a.rows && t < now.q.count ? now.q.length - now.q.count + t : -1;
                }
            }
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
        __syncwarp();
        if (u + kStages - 1 < n) issue(stage == 0 ? kStages - 1 : stage - 1, next);
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (u + kStages < n) { next = look_up(); cursor_next<kSub>(a, ahead, per); }

        // ---- S^T ----
        const unsigned keys = ring + stage * C::kPartBytes, values = keys + C::kSlots * C::kPitch;
        unsigned kw[kSub][4];
        float x[kSub][kCols][4];
#pragma unroll
        for (int b = 0; b < kSub; ++b)
#pragma unroll
            for (int j = 0; j < kCols; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[b][j][e] = 0.0f;
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int k = 2 * g + i;
                uint2 qb[kCols];
#pragma unroll
                for (int j = 0; j < kCols; ++j)
                    qb[j] = C::kHeld ? make_uint2(held[(j * C::kSteps + k) * 2 * C::kHeld], held[((j * C::kSteps + k) * 2 + 1) * C::kHeld])
                                     : *(const uint2 *)(s_q + ((k * C::kRows + j * 8 + (lane >> 2)) * 4 + (lane & 3)) * 8);
#pragma unroll
                for (int b = 0; b < kSub; ++b) {
                    // words of slots lane / 4 and 8 more; dimensions 32 g + 4 (lane & 3) .. and 16 more
                    if (i == 0) ldsm4(kw[b], keys + C::unit_at(16 * b + (lane & 15), 2 * g + (lane >> 4)));
                    unsigned ka[4];
                    O::keys(kw[b][2 * i], ka[0], ka[2]);
                    O::keys(kw[b][2 * i + 1], ka[1], ka[3]);
#pragma unroll
                    for (int j = 0; j < kCols; ++j) mma<__half>(x[b][j], ka, qb[j].x, qb[j].y);
                }
            }
        // ---- what each row sees ----
        const int slot0 = slot_of(now), seen0 = now.q.length - now.q.count;
        const bool whole = slot0 + C::kSlots - 1 <= seen0 && (a.window == 0 || slot0 > now.q.length - 1 - a.window);
        float more[kSub][2];                             // logarithms of the values' scales, of slots lane / 4 and 8 more
#pragma unroll
        for (int b = 0; b < kSub; ++b) {
            float2 scales[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(scales[i].x), "=f"(scales[i].y) : "r"(keys + C::kScalesAt + 8 * (16 * b + (lane >> 2) + 8 * i)) : "memory");
                more[b][i] = log2_of(scales[i].y);
            }
#pragma unroll
            for (int j = 0; j < kCols; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[b][j][e] = (O::kShifted ? fmaf(x[b][j][e], 16777216.0f, -off[j][e & 1]) : x[b][j][e]) * (by[j][e & 1] * scales[e >> 1].x);
                    if (!whole && !sees(a, p[j][e & 1], slot0 + 16 * b + (lane >> 2) + (e >> 1) * 8)) x[b][j][e] = -INFINITY;
                }
        }
        if (a.logits != nullptr) {
            const int64_t tile = (begin + u) * kSub + (kSub == 2 ? part / 2 : 0);
            const int in_tile = kSub == 2 ? (part & 1) * 32 : part * 16;
            if (in_tile == 0 && lane == 0) *(int4 *)&a.notes[tile] = make_int4(now.s, now.head, slot0, now.q.length);
#pragma unroll
            for (int b = 0; b < kSub; ++b) {
                float *const to = a.logits + tile * (int64_t)(logit_pitch * kTile) + (in_tile + 16 * b + (lane >> 2)) * logit_pitch;
#pragma unroll
                for (int j = 0; j < kCols; ++j) {
                    const int r = j * 8 + (lane & 3) * 2;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float2 w = make_float2(p[j][0] < 0 ? -INFINITY : x[b][j][2 * e], p[j][1] < 0 ? -INFINITY : x[b][j][2 * e + 1]);
                        float *const at = to + e * 8 * logit_pitch + r;
                        if (logit_pitch > 1) { if (r < logit_pitch) *(float2 *)at = w; }
                        else if (r == 0) *at = w.x;
                    }
                }
            }
        }
        // ---- weights ----
        float y[kSub][kCols][4];                         // with the value's scale (an unseen slot's may be anything)
        bool over = false;
#pragma unroll
        for (int b = 0; b < kSub; ++b)
#pragma unroll
            for (int j = 0; j < kCols; ++j) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y[b][j][e] = x[b][j][e] + more[b][e >> 1];
                    if (!whole) y[b][j][e] = x[b][j][e] == -INFINITY ? -INFINITY : y[b][j][e];
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) over |= fmaxf(fmaxf(x[b][j][h], x[b][j][h + 2]) - m[j][h], fmaxf(y[b][j][h], y[b][j][h + 2]) - top[j][h]) > kSlack;
            }
        if (__any_sync(0xffffffffu, over)) {
#pragma unroll
            for (int j = 0; j < kCols; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float best = m[j][h], most = top[j][h];
#pragma unroll
                    for (int b = 0; b < kSub; ++b) {
                        best = fmaxf(best, fmaxf(x[b][j][h], x[b][j][h + 2]));
                        most = fmaxf(most, fmaxf(y[b][j][h], y[b][j][h + 2]));
                    }
#pragma unroll
                    for (int o = 4; o < 32; o *= 2) {
                        best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, o));
                        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
                    }
                    l[j][h] *= exp2_of(m[j][h] - best);
                    const float less_now = exp2_of(top[j][h] - most);
                    m[j][h] = best; top[j][h] = most;
#pragma unroll
                    for (int k = 0; k < C::kSteps; ++k) { acc[k][j][h] *= less_now; acc[k][j][h + 2] *= less_now; }
                }
        }
#pragma unroll
        for (int b = 0; b < kSub; ++b)
#pragma unroll
            for (int j = 0; j < kCols; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float most = top[j][h] - kLift;
                    l[j][h] += exp2_of(x[b][j][h] - m[j][h]) + exp2_of(x[b][j][h + 2] - m[j][h]);
                    x[b][j][h] = exp2_of(y[b][j][h] - most); x[b][j][h + 2] = exp2_of(y[b][j][h + 2] - most);
                }
        // ---- O^T ----
        __syncwarp();                                    // (a warp executes what follows as one)
        bool apart = false;
        if (std::is_same<Code, E4m3>::value && !whole && now.q.count > 1) {
            // Slots that only some rows see: a weight of zero times a code that is no number is none.
            for (int i = lane; i < C::kSlots * C::kDim / 16; i += 32) {
                unsigned w[4];
                load_words<4>(w, values + C::unit_at(i / (C::kDim / 16), i % (C::kDim / 16)));
#pragma unroll
                for (int e = 0; e < 4; ++e) apart |= __vcmpeq4(w[e] & 0x7f7f7f7fu, 0x7f7f7f7fu) != 0;
            }
            apart = __any_sync(0xffffffffu, apart);
        }
        const int c = lane & 3, r = lane >> 2;
        // where bytes `at` .. of a slot's values lie
        auto value_at = [&](int slot, int at) -> unsigned { return values + C::unit_at(slot, at >> 4) + (at & 15); };
        // words words_ of the lane's slots from dimension `base` + 4 words_ (lane / 4) on: steps k0 .. of the sums
        auto values_of = [&](auto words_, int base, int k0, int b, const unsigned (&wb)[kCols][2]) {
            constexpr int kWords = decltype(words_)::value;
            unsigned w[4][kWords];                       // slots 2 c, 2 c + 1, 2 c + 8, 2 c + 9
#pragma unroll
            for (int i = 0; i < 4; ++i) load_words<kWords>(w[i], value_at(16 * b + 2 * c + (i & 1) + (i >> 1) * 8, base + 4 * kWords * r));
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                unsigned lo[4], hi[4];
                O::values(w[0][i], w[1][i], lo);
                O::values(w[2][i], w[3][i], hi);
                const unsigned va[2][4] = {{lo[0], lo[1], hi[0], hi[1]}, {lo[2], lo[3], hi[2], hi[3]}};
#pragma unroll
                for (int z = 0; z < 2; ++z)
#pragma unroll
                    for (int j = 0; j < kCols; ++j) mma<__half>(acc[k0 + 2 * i + z][j], va[z], wb[j][0], wb[j][1]);
            }
        };
        // the dimension that step k's sums 0 and 1 belong to (2 and 3: the next one)
        auto dim_of = [&](int k) -> int {
            const int whole16 = kGroups / 4 * 8;         // steps of the blocks of 128 dimensions
            if (k < whole16) return k / 8 * 128 + 16 * r + 2 * (k % 8);
            if (kGroups % 4 >= 2 && k < whole16 + 4) return whole16 * 16 + 8 * r + 2 * (k - whole16);
            return (whole16 + kGroups % 4 / 2 * 4) * 16 + 4 * r + 2 * (k - whole16 - kGroups % 4 / 2 * 4);
        };
        if (!apart) {
#pragma unroll
            for (int b = 0; b < kSub; ++b) {
                unsigned wb[kCols][2];
#pragma unroll
                for (int j = 0; j < kCols; ++j)
#pragma unroll
                    for (int e = 0; e < 2; ++e) wb[j][e] = turned8x8(Pair<__half>::pack(x[b][j][2 * e], x[b][j][2 * e + 1]));
#pragma unroll
                for (int q = 0; q < kGroups / 4; ++q) values_of(std::integral_constant<int, 4>(), 128 * q, 8 * q, b, wb);
                if (kGroups % 4 >= 2) values_of(std::integral_constant<int, 2>(), kGroups / 4 * 128, kGroups / 4 * 8, b, wb);
                if (kGroups % 2 == 1) values_of(std::integral_constant<int, 1>(), (kGroups - 1) * 32, (kGroups - 1) * 2, b, wb);
            }
        } else {
#pragma unroll
            for (int b = 0; b < kSub; ++b)
                for (int o = 0; o < 16; ++o)
#pragma unroll
                    for (int j = 0; j < kCols; ++j) {
                        float w[2];
                        bool in[2];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            w[h] = __shfl_sync(0xffffffffu, o < 8 ? x[b][j][h] : x[b][j][h + 2], (o & 7) * 4 + c);
                            in[h] = sees(a, p[j][h], slot0 + 16 * b + o);
                        }
#pragma unroll
                        for (int k = 0; k < C::kSteps; ++k) {
                            unsigned short v;
                            asm volatile("ld.shared.b16 %0, [%1];" : "=h"(v) : "r"(value_at(16 * b + o, dim_of(k))) : "memory");
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const float f = O::value((unsigned)v >> (8 * e));
#pragma unroll
                                for (int h = 0; h < 2; ++h) if (in[h]) acc[k][j][2 * e + h] = fmaf(w[h], f, acc[k][j][2 * e + h]);
                            }
                        }
                    }
        }
        if (now.idx == now.q.tiles - 1 || u == n - 1) {
            // ---- the piece's end: the parts are joined, eight rows at a time, each warp's sums in the part of its ring that it is done with ----
            __syncwarp();
#pragma unroll
            for (int j = 0; j < kCols; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int o = 4; o < 32; o *= 2) l[j][h] += __shfl_xor_sync(0xffffffffu, l[j][h], o);
                    l[j][h] /= Weights<T>::kUnlift;      // (what joins expects sums as the other kernel leaves them)
                    // (padding has seen nothing, whatever its weights were; a row without a number among its logits keeps a sum that is none)
                    const float2 ml = p[j][h] < 0 ? make_float2(-INFINITY, 0.0f) : m[j][h] == kLowest ? make_float2(-INFINITY, l[j][h] - l[j][h]) : make_float2(m[j][h], l[j][h]);
                    if (lane < 4) s_ml[part * C::kRows + j * 8 + lane * 2 + h] = ml;
                }
            float *const room = (float *)(smem + stage * C::kPartBytes);
            constexpr int kApart = kStages * C::kPartBytes / 4;      // floats from one warp's to the next's
            // is this all of the item?
            const bool all = u >= now.idx && now.idx == now.q.tiles - 1;
            const int64_t piece = item + blockIdx.x;
#pragma unroll
            for (int j = 0; j < kCols; ++j) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // from the maximum of weight times vs to that of the weights (no value yet: no sums)
                    const float back = top[j][h] == kLowest ? 1.0f : exp2_of(top[j][h] - m[j][h] - kLift + Weights<T>::kLift);
#pragma unroll
                    for (int k = 0; k < C::kSteps; k += 2)
                        *(float4 *)&room[part * kApart + (c * 2 + h) * C::kMergePitch + dim_of(k)] =
                            make_float4(acc[k][j][h] * back, acc[k][j][h + 2] * back, acc[k + 1][j][h] * back, acc[k + 1][j][h + 2] * back);
                }
                __syncthreads();
                for (int i = tid; i < 8 * (C::kDim / 4); i += kThreads) {
                    const int in = i / (C::kDim / 4), row = j * 8 + in, d = i % (C::kDim / 4) * 4;
                    if (row >= a.rows) continue;
                    float best = -INFINITY, sum = 0.0f;
#pragma unroll
                    for (int q = 0; q < kParts; ++q) best = fmaxf(best, s_ml[q * C::kRows + row].x);
                    const float ref = best == -INFINITY ? 0.0f : best;
                    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                    for (int q = 0; q < kParts; ++q) {
                        const float2 ml = s_ml[q * C::kRows + row];
                        const float f = exp2_of(ml.x - ref);
                        const float4 v = *(const float4 *)&room[q * kApart + in * C::kMergePitch + d];
                        sum = fmaf(ml.y, f, sum);
                        o.x = fmaf(v.x, f, o.x); o.y = fmaf(v.y, f, o.y); o.z = fmaf(v.z, f, o.z); o.w = fmaf(v.w, f, o.w);
                    }
                    if (cluster > 0) {
                        if (d == 0) s_join_ml[row] = make_float2(best, sum);
                        *(float4 *)(s_join + row * C::kDim + d) = o;
                        continue;
                    }
                    if (d == 0) a.ml[row * a.pieces + piece] = make_float2(best, sum);
                    if (!all) {
                        *(float4 *)(a.part + (piece * C::kRows + row) * C::kDim + d) = o;
                    } else if (d < a.c.head_dim) {
                        const int64_t at = ((int64_t)now.s * a.new_tokens + row / a.group) * a.q_heads + now.head * a.group + row % a.group;
                        give<T>(a, at, d, row / a.group < now.q.count, best, sum, o, item * C::kRows + row);
                    }
                }
                __syncthreads();                         // (the ring may be written again)
            }
            fresh = true;
        }
        stage = stage == kStages - 1 ? 0 : stage + 1;
        cursor_next<kSub>(a, now, per);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (bad != 0) raise_status(a.c.status, bad);
    if (cluster > 0) {
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

// ---- host ----
template <typename T, typename Code, int kGroups, int kCols>
cudaError_t launch_packed(const PackedArgs &a, const AttendShape &z, cudaStream_t s)
{
    typedef PackedConfig<kGroups, kCols> C;
    static int known[kMaxDevices], most_known[kMaxDevices];
    return launch_few<T, C::kRows, C::kDim, C::kSub, AttendArgs>(k_packed_attend<T, Code, kGroups, kCols>, C::kSmem, known, most_known, a, z, s);
}
template <typename T, typename Code, int kGroups>
cudaError_t launch_packed_rows(const PackedArgs &a, const AttendShape &z, cudaStream_t s)
{
    return z.block_rows == 8 ? launch_packed<T, Code, kGroups, 1>(a, z, s) : launch_packed<T, Code, kGroups, 2>(a, z, s);
}
template <typename T, typename Code>
cudaError_t launch_packed_type(const PackedArgs &a, const AttendShape &z, cudaStream_t s)
{
    switch (z.padded_dim / 32) {
    case 2: return launch_packed_rows<T, Code, 2>(a, z, s);
    case 3: return launch_packed_rows<T, Code, 3>(a, z, s);
    case 4: return launch_packed_rows<T, Code, 4>(a, z, s);
    case 6: return launch_packed_rows<T, Code, 6>(a, z, s);
    default: return launch_packed_rows<T, Code, 8>(a, z, s);
    }
}

}  // namespace attend

cudaError_t launch_packed_bf16_int8(const PackedArgs &a, const AttendShape &z, cudaStream_t s);
cudaError_t launch_packed_bf16_e4m3(const PackedArgs &a, const AttendShape &z, cudaStream_t s);
cudaError_t launch_packed_fp16_int8(const PackedArgs &a, const AttendShape &z, cudaStream_t s);
cudaError_t launch_packed_fp16_e4m3(const PackedArgs &a, const AttendShape &z, cudaStream_t s);

}  // namespace g10
