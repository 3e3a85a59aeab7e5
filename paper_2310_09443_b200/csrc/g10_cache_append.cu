// Writing new tokens to the key-value cache: norm of queries and keys per head, position rotation, write to the pages, one pass.
#include "g10_cache.cuh"

namespace g10 {
namespace {

constexpr int kAppendThreads = 128;

// A row (one head of one token) is held by kLanes threads, 8 elements each.  Rows of a token: its query heads, its key heads, its
// value heads; a team of kLanes threads takes kEach of them, every kTeams-th, and asks for all before it looks at the first.  Everything is read once and
// written once; the 8 values stay in registers between norm, rotation and rounding, and only the partners of half-split pairs go
// through shared memory.  The rotation's 8 cosines and sines are the same for all rows of a team: loaded once, 16 bytes at a time (kWide:
// tables and rotary_dim allow it).  A block takes `run` tokens of a sequence, one after the other: what is the same for all of them (addresses,
// lengths, weights) is worked out once, since for prompts the instructions, not the traffic, are what takes the time.
template <typename T, int kLanes, int kEach, bool kWide>
__global__ void __launch_bounds__(kAppendThreads) k_cache_append(const AppendArgs a, int shares, int runs, int run)
{
    constexpr int kTeams = kAppendThreads / kLanes;
    __shared__ __align__(16) float s_x[kAppendThreads * 8];
    const CacheView &c = a.c;
    const int lane = threadIdx.x % kLanes, team = threadIdx.x / kLanes;
    const int rows = a.q_heads + 2 * c.kv_heads;
    const unsigned place = blockIdx.x / (unsigned)shares;          // which run of which sequence
    const int share = (int)(blockIdx.x - place * (unsigned)shares);
    const int s = (int)(place / (unsigned)runs), t0 = (int)(place - (unsigned)s * (unsigned)runs) * run;
    const int d0 = lane * 8, half = a.rotary / 2;
    const bool mine = d0 < c.head_dim;
    // the thread's rows: where they come from, token t0
    const char *from[kEach];
    uint4 u[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int row = (share * kEach + i) * kTeams + team;
        from[i] = nullptr;
        if (row < a.q_heads) from[i] = a.q + 2 * (s * a.q_seq + t0 * a.q_token + row * a.q_head + d0);
        else if (row < a.q_heads + c.kv_heads) from[i] = a.k + 2 * (s * a.k_seq + t0 * a.k_token + (row - a.q_heads) * a.k_head + d0);
        else if (row < rows) from[i] = a.v + 2 * (s * a.v_seq + t0 * a.v_token + (row - a.q_heads - c.kv_heads) * a.v_head + d0);
        if (!mine) from[i] = nullptr;
        // (those of padding too: what they hold is not used)
        u[i] = from[i] != nullptr ? __ldg((const uint4 *)from[i]) : make_uint4(0, 0, 0, 0);
    }
    ull bad = 0;
    const int seen = __ldg(&c.seen[s]);
    const int length = cache_length(c, s, bad), count = cache_count(a.counts, s, a.new_tokens, length, bad);
    float qw[8], kw[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const char *const weight = h == 0 ? a.q_weight : a.k_weight;
        float *const to = h == 0 ? qw : kw;
        if (weight != nullptr && mine) {
            const uint4 g = __ldg((const uint4 *)(weight + 2 * d0));
            const unsigned gw[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) { const float2 p = Pair<T>::unpack(gw[e]); to[2 * e] = p.x; to[2 * e + 1] = p.y; }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) to[e] = 1.0f;
        }
    }
    float *const mate = s_x + team * kLanes * 8;
    const int t1 = min(a.new_tokens, t0 + run);
#pragma unroll 1
    for (int t = t0; t < min(t1, count); ++t) {
        const int64_t position = (int64_t)seen - count + t;
        const Spot spot = cache_spot(c, s, length - count + t, bad);
        if (t > t0) {
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                if (from[i] != nullptr) {
                    const int row = (share * kEach + i) * kTeams + team;
                    from[i] += 2 * (row < a.q_heads ? a.q_token : row < a.q_heads + c.kv_heads ? a.k_token : a.v_token);
                    u[i] = __ldg((const uint4 *)from[i]);
                }
        }
        float co[8], si[8];
        const bool turns = a.rotary > 0 && position >= 0 && position < a.table_rows;
        if (a.rotary > 0 && !turns) bad |= G10_DEV_BAD_POSITION;
#pragma unroll
        for (int e = 0; e < 8; ++e) { co[e] = 1.0f; si[e] = 0.0f; }
        if (turns && d0 < a.rotary) {
            const float *const cos_row = a.cos_table + position * half, *const sin_row = a.sin_table + position * half;
            if (kWide) {
                if (a.interleaved) {
                    const float4 x = __ldg((const float4 *)(cos_row + d0 / 2)), y = __ldg((const float4 *)(sin_row + d0 / 2));
                    co[0] = co[1] = x.x; co[2] = co[3] = x.y; co[4] = co[5] = x.z; co[6] = co[7] = x.w;
                    si[0] = si[1] = y.x; si[2] = si[3] = y.y; si[4] = si[5] = y.z; si[6] = si[7] = y.w;
                } else {
                    const int j = d0 < half ? d0 : d0 - half;
                    *(float4 *)&co[0] = __ldg((const float4 *)(cos_row + j)); *(float4 *)&co[4] = __ldg((const float4 *)(cos_row + j + 4));
                    *(float4 *)&si[0] = __ldg((const float4 *)(sin_row + j)); *(float4 *)&si[4] = __ldg((const float4 *)(sin_row + j + 4));
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int d = d0 + e, j = a.interleaved ? d >> 1 : (d < half ? d : d - half);
                    if (d < a.rotary) { co[e] = __ldg(&cos_row[j]); si[e] = __ldg(&sin_row[j]); }
                }
            }
        }
        // (the first of a pair takes its partner with a minus)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (a.interleaved ? (e & 1) == 0 : d0 + e < half) si[e] = -si[e];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int row = (share * kEach + i) * kTeams + team;
            const bool is_q = row < a.q_heads, is_k = !is_q && row < a.q_heads + c.kv_heads, is_v = !is_q && !is_k && row < rows;
            const int head = is_q ? row : is_k ? row - a.q_heads : row - a.q_heads - c.kv_heads;
            unsigned *w = &u[i].x;
            if (__any_sync(0xffffffffu, is_q || is_k)) {       // (some row of the warp has arithmetic to do)
                float x[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) { const float2 p = Pair<T>::unpack(w[e]); x[2 * e] = p.x; x[2 * e + 1] = p.y; }
                if (a.q_weight != nullptr || a.k_weight != nullptr) {
                    float sum = 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum = fmaf(x[e], x[e], sum);
#pragma unroll
                    for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                    const float r = rsqrtf(fmaf(sum, a.inv_dim, a.eps));
                    if (is_q ? a.q_weight != nullptr : a.k_weight != nullptr)
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] *= r * (is_q ? qw[e] : kw[e]);
                }
                if (a.rotary > 0) {
                    float other[8];
                    if (a.interleaved) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) other[e] = x[e ^ 1];
                    } else {
                        __syncwarp();
                        *(float4 *)&mate[d0] = make_float4(x[0], x[1], x[2], x[3]); *(float4 *)&mate[d0 + 4] = make_float4(x[4], x[5], x[6], x[7]);
                        __syncwarp();
                        if (kWide) {
                            const int at = d0 >= a.rotary ? d0 : d0 < half ? d0 + half : d0 - half;
                            *(float4 *)&other[0] = *(const float4 *)&mate[at]; *(float4 *)&other[4] = *(const float4 *)&mate[at + 4];
                        } else {
#pragma unroll
                            for (int e = 0; e < 8; ++e) { const int d = d0 + e; other[e] = d >= a.rotary ? 0.0f : mate[d < half ? d + half : d - half]; }
                        }
                    }
                    if (kWide) {
                        if (d0 < a.rotary)
#pragma unroll
                            for (int e = 0; e < 8; ++e) x[e] = fmaf(x[e], co[e], other[e] * si[e]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) if (d0 + e < a.rotary) x[e] = fmaf(x[e], co[e], other[e] * si[e]);
                    }
                }
                if (is_q || is_k) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = Pair<T>::pack(x[2 * e], x[2 * e + 1]);
                }
            }
            if (is_q && mine) *(uint4 *)(a.q_out + 2 * ((((int64_t)s * a.new_tokens + t) * a.q_heads + head) * c.head_dim + d0)) = u[i];
            if ((is_k || is_v) && spot.page >= 0) {
                if (mine) *(uint4 *)(const_cast<char *>(is_k ? c.k : c.v) + 16 * (int64_t)cache_row(c, spot, head) + 2 * d0) = u[i];
                if (is_k && lane == 0) {
                    const int64_t cell = cache_cell(c, spot, head);
                    if (c.scores != nullptr) c.scores[cell] = 0.0f;
                    if (c.positions != nullptr) c.positions[cell] = (int32_t)position;
                }
            }
        }
    }
    // padding: its queries are zero, the cache has no room for it
    for (int t = max(t0, count); t < t1; ++t)
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int row = (share * kEach + i) * kTeams + team;
            if (row < a.q_heads && mine) *(uint4 *)(a.q_out + 2 * ((((int64_t)s * a.new_tokens + t) * a.q_heads + row) * c.head_dim + d0)) = make_uint4(0, 0, 0, 0);
        }
    if (bad != 0 && threadIdx.x == 0) raise_status(c.status, bad);
}

template <typename T, int kLanes, int kEach>
cudaError_t launch(const AppendArgs &a, int shares, cudaStream_t s)
{
    const int half = a.rotary / 2;
    const bool wide = (((uintptr_t)a.cos_table | (uintptr_t)a.sin_table) & 15u) == 0 && half % (a.interleaved ? 4 : 8) == 0;
    // (runs of up to 8 tokens, as long as there are 16 blocks for every SM: 31 us with one token a block, for 12 291 of which 4120 count)
    int run = 1;
    while (run < 8 && run < a.new_tokens && (int64_t)a.c.num_seqs * ((a.new_tokens + 2 * run - 1) / (2 * run)) * shares >= 148 * 16) run *= 2;
    const int runs = (a.new_tokens + run - 1) / run;
    const int64_t blocks = (int64_t)a.c.num_seqs * runs * shares;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    if (wide) k_cache_append<T, kLanes, kEach, true><<<(unsigned)blocks, kAppendThreads, 0, s>>>(a, shares, runs, run);
    else k_cache_append<T, kLanes, kEach, false><<<(unsigned)blocks, kAppendThreads, 0, s>>>(a, shares, runs, run);
    count_launch();
    return cudaGetLastError();
}
template <typename T, int kLanes>
cudaError_t launch_lanes(const AppendArgs &a, cudaStream_t s)
{
    constexpr int kTeams = kAppendThreads / kLanes;
    const int rows = a.q_heads + 2 * a.c.kv_heads;
    const int64_t tokens = (int64_t)a.c.num_seqs * a.new_tokens;
    auto shares = [&](int each) { return (rows + kTeams * each - 1) / (kTeams * each); };
    // (several rows a thread once there are blocks enough for all SMs all the same: fewer look-ups and rotations for each)
    if (tokens * shares(4) >= 148 * 16 && rows > 2 * kTeams) return launch<T, kLanes, 4>(a, shares(4), s);
    if (tokens * shares(2) >= 148 * 16 && rows > kTeams) return launch<T, kLanes, 2>(a, shares(2), s);
    return launch<T, kLanes, 1>(a, shares(1), s);
}

}  // namespace

cudaError_t launch_cache_append(const AppendArgs &a, int dtype, cudaStream_t s)
{
    const int lanes = (a.c.head_dim + 7) / 8;
    if (dtype == G10_BF16) return lanes <= 8 ? launch_lanes<__nv_bfloat16, 8>(a, s) : lanes <= 16 ? launch_lanes<__nv_bfloat16, 16>(a, s) : launch_lanes<__nv_bfloat16, 32>(a, s);
    return lanes <= 8 ? launch_lanes<__half, 8>(a, s) : lanes <= 16 ? launch_lanes<__half, 16>(a, s) : launch_lanes<__half, 32>(a, s);
}

}  // namespace g10
