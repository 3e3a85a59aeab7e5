// Writing new tokens to the key-value cache: norm of queries and keys per head, position rotation, write to the pages (as they are, or in 8 bits), one
// pass.
#include <type_traits>

#include "g10_packed.cuh"

namespace g10 {
namespace {

constexpr int kAppendThreads = 128;

// A row (one head of one token) is held by kLanes threads, 8 elements each.  Rows of a token: its query heads, its key heads, its
// value heads; a team of kLanes threads takes kEach of them, every kTeams-th, and asks for all before it looks at the first.  Everything is read once and
// written once; the 8 values stay in registers between norm, rotation and rounding, and only the partners of half-split pairs go
// through shared memory.  The rotation's 8 cosines and sines are the same for all rows of a team: loaded once, 16 bytes at a time where the
// tables and rotary_dim allow it.  A block takes `run` tokens of a sequence, one after the other: what is the same for all of them (addresses,
// lengths, weights) is worked out once, since for prompts the instructions, not the traffic, are what takes the time.
// With a Code, rows of keys and values go out as 8-bit codes: the row's threads find its largest element while it is still in their registers.  (Five blocks an SM instead of six, for the
// registers: 3 prompts up to 4097 tokens of 48 heads of 64 take 30.5 instead of 33 us; 22.8 as they are.)
enum { kNone, kSplit, kPairs, kAny };    // rotation: none, half-split or interleaved pairs in whole 16-byte units, whatever else

template <typename T, typename Code, int kLanes, int kEach, int kTurn>
__global__ void __launch_bounds__(kAppendThreads, std::is_void<Code>::value ? 6 : 5) k_cache_append(const AppendArgs a, int shares, int runs, int run)
{
    constexpr int kTeams = kAppendThreads / kLanes;
    constexpr bool kPacked = !std::is_void<Code>::value;
    __shared__ __align__(16) float s_x[kAppendThreads * 8];
    const CacheView &c = a.c;
    const int lane = threadIdx.x % kLanes, team = threadIdx.x / kLanes;
    const int rows = a.q_heads + 2 * c.kv_heads;
    const unsigned place = blockIdx.x / (unsigned)shares;          // which run of which sequence
    const int share = (int)(blockIdx.x - place * (unsigned)shares);
    const int s = (int)(place / (unsigned)runs), t0 = (int)(place - (unsigned)s * (unsigned)runs) * run;
    const int d0 = lane * 8, half = a.rotary / 2;
    const bool mine = d0 < c.head_dim;
    const bool turned = kTurn != kNone && d0 < a.rotary;
    // the thread's rows: where they come from and go to, token 0 of the sequence and slot 0 of page 0
    const char *from[kEach];
    char *to[kEach];
    uint4 u[kEach];
    const int64_t q_from = 2 * (s * a.q_seq + d0), k_from = 2 * (s * a.k_seq + d0), v_from = 2 * (s * a.v_seq + d0);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int row = (share * kEach + i) * kTeams + team;
        from[i] = nullptr; to[i] = nullptr;
        u[i] = make_uint4(0, 0, 0, 0);
        if (!mine || row >= rows) continue;
        const bool is_q = row < a.q_heads, is_k = row < a.q_heads + c.kv_heads;
        const int head = is_q ? row : is_k ? row - a.q_heads : row - a.q_heads - c.kv_heads;
        from[i] = is_q ? a.q + q_from + 2 * head * a.q_head : is_k ? a.k + k_from + 2 * head * a.k_head : a.v + v_from + 2 * head * a.v_head;
        to[i] = is_q ? a.q_out + 2 * (((int64_t)s * a.new_tokens * a.q_heads + head) * c.head_dim + d0)
                     : const_cast<char *>(is_k ? c.k : c.v) + 16 * head * c.head_stride + (kPacked ? 1 : 2) * d0;
        // (those of padding too: what they hold is not used)
        u[i] = __ldg((const uint4 *)(from[i] + 2 * (int64_t)t0 * (is_q ? a.q_token : is_k ? a.k_token : a.v_token)));
    }
    ull bad = 0;
    const int seen = __ldg(&c.seen[s]);
    const int length = cache_length(c, s, bad), count = cache_count(a.counts, s, a.new_tokens, length, bad);
    const uint4 qw = a.q_weight != nullptr && mine ? __ldg((const uint4 *)(a.q_weight + 2 * d0)) : make_uint4(0, 0, 0, 0);
    const uint4 kw = a.k_weight != nullptr && mine ? __ldg((const uint4 *)(a.k_weight + 2 * d0)) : make_uint4(0, 0, 0, 0);
    float *const mate = s_x + team * kLanes * 8;
    const int t1 = min(a.new_tokens, t0 + run);
#pragma unroll 1
    for (int t = t0; t < min(t1, count); ++t) {
        const int64_t position = (int64_t)seen - count + t;
        const Spot spot = cache_spot(c, s, length - count + t, bad);
        const bool turns = turned && position >= 0 && position < a.table_rows;
        if (kTurn != kNone && (position < 0 || position >= a.table_rows)) bad |= G10_DEV_BAD_POSITION;
        if (t > t0) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int row = (share * kEach + i) * kTeams + team;
                if (from[i] != nullptr) u[i] = __ldg((const uint4 *)(from[i] + 2 * (int64_t)t * (row < a.q_heads ? a.q_token : row < a.q_heads + c.kv_heads ? a.k_token : a.v_token)));
            }
        }
        float co[8], si[8];                              // (the first of a pair takes its partner with a minus)
        if (turns) {
            const float *const cos_row = a.cos_table + position * half, *const sin_row = a.sin_table + position * half;
            if (kTurn == kPairs) {
                const float4 x = __ldg((const float4 *)(cos_row + d0 / 2)), y = __ldg((const float4 *)(sin_row + d0 / 2));
                co[0] = co[1] = x.x; co[2] = co[3] = x.y; co[4] = co[5] = x.z; co[6] = co[7] = x.w;
                si[0] = -y.x; si[1] = y.x; si[2] = -y.y; si[3] = y.y; si[4] = -y.z; si[5] = y.z; si[6] = -y.w; si[7] = y.w;
            } else if (kTurn == kSplit) {
                const int j = d0 < half ? d0 : d0 - half;
                *(float4 *)&co[0] = __ldg((const float4 *)(cos_row + j)); *(float4 *)&co[4] = __ldg((const float4 *)(cos_row + j + 4));
                *(float4 *)&si[0] = __ldg((const float4 *)(sin_row + j)); *(float4 *)&si[4] = __ldg((const float4 *)(sin_row + j + 4));
                if (d0 < half) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) si[e] = -si[e];
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int d = d0 + e, j = a.interleaved ? d >> 1 : (d < half ? d : d - half);
                    co[e] = 1.0f; si[e] = 0.0f;
                    if (d < a.rotary) {
                        co[e] = __ldg(&cos_row[j]); si[e] = __ldg(&sin_row[j]);
                        if (a.interleaved ? (e & 1) == 0 : d < half) si[e] = -si[e];
                    }
                }
            }
        }
        const int64_t q_at = 2 * (int64_t)t * a.q_heads * c.head_dim, kv_at = 16 * ((int64_t)spot.page * c.page_stride + (int64_t)spot.place * c.slot_stride);
        const int64_t cell = ((int64_t)spot.page * c.kv_heads) * c.page_size + spot.place;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int row = (share * kEach + i) * kTeams + team;
            const bool is_q = row < a.q_heads, is_k = !is_q && row < a.q_heads + c.kv_heads;
            unsigned *w = &u[i].x;
            float x[8];
            if (kPacked || __any_sync(0xffffffffu, is_q || is_k)) {      // (some row of the warp has arithmetic to do)
#pragma unroll
                for (int e = 0; e < 4; ++e) { const float2 p = Pair<T>::unpack(w[e]); x[2 * e] = p.x; x[2 * e + 1] = p.y; }
                if (a.q_weight != nullptr || a.k_weight != nullptr) {
                    float sum = 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum = fmaf(x[e], x[e], sum);
#pragma unroll
                    for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                    const float r = rsqrtf(fmaf(sum, a.inv_dim, a.eps));
                    if (is_q ? a.q_weight != nullptr : a.k_weight != nullptr && (!kPacked || is_k)) {
                        const unsigned g[4] = {is_q ? qw.x : kw.x, is_q ? qw.y : kw.y, is_q ? qw.z : kw.z, is_q ? qw.w : kw.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) { const float2 p = Pair<T>::unpack(g[e]); x[2 * e] *= r * p.x; x[2 * e + 1] *= r * p.y; }
                    }
                }
                if (kTurn == kPairs || (kTurn == kAny && a.interleaved)) {
                    if (turns && (!kPacked || is_q || is_k)) {
#pragma unroll
                        for (int e = 0; e < 8; e += 2) {
                            const float y = fmaf(x[e], co[e], x[e + 1] * si[e]), z = fmaf(x[e + 1], co[e + 1], x[e] * si[e + 1]);
                            if (kTurn == kPairs || d0 + e < a.rotary) { x[e] = y; x[e + 1] = z; }
                        }
                    }
                } else if (kTurn != kNone) {
                    __syncwarp();
                    *(float4 *)&mate[d0] = make_float4(x[0], x[1], x[2], x[3]); *(float4 *)&mate[d0 + 4] = make_float4(x[4], x[5], x[6], x[7]);
                    __syncwarp();
                    if (turns && (!kPacked || is_q || is_k)) {
                        if (kTurn == kSplit) {
                            const float *const other = &mate[d0 < half ? d0 + half : d0 - half];
                            const float4 y = *(const float4 *)other, z = *(const float4 *)(other + 4);
                            x[0] = fmaf(x[0], co[0], y.x * si[0]); x[1] = fmaf(x[1], co[1], y.y * si[1]); x[2] = fmaf(x[2], co[2], y.z * si[2]); x[3] = fmaf(x[3], co[3], y.w * si[3]);
                            x[4] = fmaf(x[4], co[4], z.x * si[4]); x[5] = fmaf(x[5], co[5], z.y * si[5]); x[6] = fmaf(x[6], co[6], z.z * si[6]); x[7] = fmaf(x[7], co[7], z.w * si[7]);
                        } else {
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const int d = d0 + e;
                                if (d < a.rotary) x[e] = fmaf(x[e], co[e], mate[d < half ? d + half : d - half] * si[e]);
                            }
                        }
                    }
                }
                if (kPacked ? is_q : is_q || is_k) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = Pair<T>::pack(x[2 * e], x[2 * e + 1]);
                }
            }
            if constexpr (kPacked) {
                // (as unsigned numbers the magnitudes are in order, infinities and NaN above all others)
                unsigned top = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
#pragma unroll
                for (int o = kLanes / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
                if (!is_q && to[i] != nullptr && spot.page >= 0) {
                    float scale;
                    *(uint2 *)(to[i] + kv_at) = packed_row<Code>(x, top, scale);
                    if (lane == 0) {
                        const int head = row - a.q_heads - (is_k ? 0 : c.kv_heads);
                        a.scales[2 * (cell + (int64_t)head * c.page_size) + (is_k ? 0 : 1)] = scale;
                    }
                }
            }
            if (kPacked && !is_q) {
            } else if (to[i] != nullptr && (is_q || spot.page >= 0)) *(uint4 *)(to[i] + (is_q ? q_at : kv_at)) = u[i];
            if (is_k && spot.page >= 0 && lane == 0) {
                const int64_t at = cell + (int64_t)(row - a.q_heads) * c.page_size;
                if (c.scores != nullptr) c.scores[at] = 0.0f;
                if (c.positions != nullptr) c.positions[at] = (int32_t)position;
            }
        }
    }
    // padding: its queries are zero, the cache has no room for it
    for (int t = max(t0, count); t < t1; ++t)
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if ((share * kEach + i) * kTeams + team < a.q_heads && mine) *(uint4 *)(to[i] + 2 * (int64_t)t * a.q_heads * c.head_dim) = make_uint4(0, 0, 0, 0);
    if (bad != 0 && threadIdx.x == 0) raise_status(c.status, bad);
}

template <typename T, typename Code, int kLanes, int kEach>
cudaError_t launch(const AppendArgs &a, int shares, cudaStream_t s)
{
    const int half = a.rotary / 2;
    const bool wide = (((uintptr_t)a.cos_table | (uintptr_t)a.sin_table) & 15u) == 0 && half % (a.interleaved ? 4 : 8) == 0;
    // (runs of up to 8 tokens, as long as there are 8 blocks for every SM: one token a block takes 41 us where eight take 23)
    int run = 1;
    while (run < 8 && run < a.new_tokens && (int64_t)a.c.num_seqs * ((a.new_tokens + 2 * run - 1) / (2 * run)) * shares >= 148 * 8) run *= 2;
    const int runs = (a.new_tokens + run - 1) / run;
    const int64_t blocks = (int64_t)a.c.num_seqs * runs * shares;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    const auto kernel = half == 0 ? k_cache_append<T, Code, kLanes, kEach, kNone> : !wide ? k_cache_append<T, Code, kLanes, kEach, kAny>
                      : a.interleaved ? k_cache_append<T, Code, kLanes, kEach, kPairs> : k_cache_append<T, Code, kLanes, kEach, kSplit>;
    kernel<<<(unsigned)blocks, kAppendThreads, 0, s>>>(a, shares, runs, run); count_launch();
    return cudaGetLastError();
}
template <typename T, typename Code, int kLanes>
cudaError_t launch_lanes(const AppendArgs &a, cudaStream_t s)
{
    constexpr int kTeams = kAppendThreads / kLanes;
    const int rows = a.q_heads + 2 * a.c.kv_heads;
    const int64_t tokens = (int64_t)a.c.num_seqs * a.new_tokens;
    auto shares = [&](int each) { return (rows + kTeams * each - 1) / (kTeams * each); };
    // (several rows a thread once there are blocks enough for all SMs all the same: fewer look-ups and rotations for each)
    if (tokens * shares(4) >= 148 * 16 && rows > 2 * kTeams) return launch<T, Code, kLanes, 4>(a, shares(4), s);
    if (tokens * shares(2) >= 148 * 16 && rows > kTeams) return launch<T, Code, kLanes, 2>(a, shares(2), s);
    return launch<T, Code, kLanes, 1>(a, shares(1), s);
}

template <typename T, typename Code>
cudaError_t launch_type(const AppendArgs &a, cudaStream_t s)
{
    const int lanes = (a.c.head_dim + 7) / 8;
    return lanes <= 8 ? launch_lanes<T, Code, 8>(a, s) : lanes <= 16 ? launch_lanes<T, Code, 16>(a, s) : launch_lanes<T, Code, 32>(a, s);
}

}  // namespace

cudaError_t launch_cache_append(const AppendArgs &a, int dtype, cudaStream_t s)
{
    return dtype == G10_BF16 ? launch_type<__nv_bfloat16, void>(a, s) : launch_type<__half, void>(a, s);
}
cudaError_t launch_packed_append(const AppendArgs &a, int dtype, int code, cudaStream_t s)
{
    if (code == G10_INT8) return dtype == G10_BF16 ? launch_type<__nv_bfloat16, Int8>(a, s) : launch_type<__half, Int8>(a, s);
    return dtype == G10_BF16 ? launch_type<__nv_bfloat16, E4m3>(a, s) : launch_type<__half, E4m3>(a, s);
}

}  // namespace g10
