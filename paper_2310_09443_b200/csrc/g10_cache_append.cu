// Writing new tokens to the key-value cache: norm of queries and keys per head, position rotation, write to the pages, one pass.
#include "g10_cache.cuh"

namespace g10 {
namespace {

constexpr int kAppendThreads = 128;

// A row (one head of one token) is held by kLanes threads, 8 elements each.  Rows of a token: its query heads, its key heads, its
// value heads.  Everything is read once and written once; the 8 values stay in registers between norm, rotation and rounding, and only
// the partners of half-split pairs go through shared memory.
template <typename T, int kLanes>
__global__ void __launch_bounds__(kAppendThreads) k_cache_append(const AppendArgs a, int rows_each)
{
    constexpr int kGroups = kAppendThreads / kLanes;
    __shared__ float s_x[kAppendThreads * 8];
    const CacheView &c = a.c;
    const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
    const int rows = a.q_heads + 2 * c.kv_heads;
    const int shares = (rows + kGroups * rows_each - 1) / (kGroups * rows_each);
    const int64_t item = blockIdx.x;
    const int share = (int)(item % shares);
    const int64_t token = item / shares;
    const int s = (int)(token / a.new_tokens), t = (int)(token % a.new_tokens);
    ull bad = 0;
    const int length = cache_length(c, s, bad), count = cache_count(a.counts, s, a.new_tokens, length, bad);
    const bool counts = t < count;
    const int slot = length - count + t;
    Spot spot{-1, 0};
    int64_t position = 0;
    if (counts) {
        spot = cache_spot(c, s, slot, bad);
        position = (int64_t)__ldg(&c.seen[s]) - count + t;
    }
    const int d0 = lane * 8, half = a.rotary / 2;
    const bool mine = d0 < c.head_dim;
    // the rotation of this thread's 8 dimensions: the same for every head of the token
    float co[8], si[8];
    const bool turns = counts && a.rotary > 0 && position >= 0 && position < a.table_rows;
    if (counts && a.rotary > 0 && !turns) bad |= G10_DEV_BAD_POSITION;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int d = d0 + e;
        co[e] = 1.0f; si[e] = 0.0f;
        if (turns && d < a.rotary) {
            const int64_t at = position * half + (a.interleaved ? d >> 1 : (d < half ? d : d - half));
            co[e] = __ldg(&a.cos_table[at]); si[e] = __ldg(&a.sin_table[at]);
        }
    }
    float *mate = s_x + group * kLanes * 8;
    for (int i = 0; i < rows_each; ++i) {
        const int row = (share * rows_each + i) * kGroups + group;
        const bool is_q = row < a.q_heads, is_k = !is_q && row < a.q_heads + c.kv_heads, is_v = !is_q && !is_k && row < rows;
        const int head = is_q ? row : is_k ? row - a.q_heads : row - a.q_heads - c.kv_heads;
        const char *from = nullptr;
        char *to = nullptr;
        if (is_q) {
            from = a.q + 2 * (s * a.q_seq + t * a.q_token + head * a.q_head);
            to = a.q_out + 2 * ((token * a.q_heads + head) * c.head_dim);
        } else if (is_k || is_v) {
            from = is_k ? a.k + 2 * (s * a.k_seq + t * a.k_token + head * a.k_head) : a.v + 2 * (s * a.v_seq + t * a.v_token + head * a.v_head);
            if (spot.page >= 0) to = const_cast<char *>(is_k ? c.k : c.v) + 16 * (int64_t)cache_row(c, spot, head);
        }
        uint4 u = make_uint4(0, 0, 0, 0);
        if (counts && from != nullptr && mine) u = *(const uint4 *)(from + 2 * d0);
        if (__syncthreads_or(is_q || is_k)) {                  // (some row of the block has arithmetic to do)
            float x[8];
            unsigned *w = &u.x;
#pragma unroll
            for (int e = 0; e < 4; ++e) { const float2 p = Pair<T>::unpack(w[e]); x[2 * e] = p.x; x[2 * e + 1] = p.y; }
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(x[e], x[e], sum);
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            const char *weight = is_q ? a.q_weight : is_k ? a.k_weight : nullptr;
            if (weight != nullptr) {
                const float r = rsqrtf(sum / (float)c.head_dim + a.eps);
                const uint4 g = mine ? *(const uint4 *)(weight + 2 * d0) : make_uint4(0, 0, 0, 0);
                const unsigned *gw = &g.x;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 p = Pair<T>::unpack(gw[e]);
                    x[2 * e] = x[2 * e] * r * p.x; x[2 * e + 1] = x[2 * e + 1] * r * p.y;
                }
            }
            if (a.rotary > 0) {
                float y[8];
                if (a.interleaved) {
#pragma unroll
                    for (int e = 0; e < 8; e += 2) { y[e] = x[e] * co[e] - x[e + 1] * si[e]; y[e + 1] = x[e + 1] * co[e + 1] + x[e] * si[e + 1]; }
                } else {
                    __syncwarp();
#pragma unroll
                    for (int e = 0; e < 8; ++e) mate[d0 + e] = x[e];
                    __syncwarp();
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int d = d0 + e;
                        const bool low = d < half;
                        const float other = d < a.rotary ? mate[low ? d + half : d - half] : 0.0f;
                        y[e] = low ? x[e] * co[e] - other * si[e] : x[e] * co[e] + other * si[e];
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = y[e];
            }
            if (is_q || is_k) {
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = Pair<T>::pack(x[2 * e], x[2 * e + 1]);
            }
        }
        if (to != nullptr && mine) {
            if (!counts) u = make_uint4(0, 0, 0, 0);           // (a padding token's query: zero)
            if (counts || is_q) *(uint4 *)(to + 2 * d0) = u;
        }
        if (is_k && spot.page >= 0 && counts && lane == 0) {
            const int64_t cell = cache_cell(c, spot, head);
            if (c.scores != nullptr) c.scores[cell] = 0.0f;
            if (c.positions != nullptr) c.positions[cell] = (int32_t)position;
        }
    }
    if (bad != 0 && threadIdx.x == 0) raise_status(c.status, bad);
}

template <typename T, int kLanes>
cudaError_t launch(const AppendArgs &a, cudaStream_t s)
{
    constexpr int kGroups = kAppendThreads / kLanes;
    const int rows = a.q_heads + 2 * a.c.kv_heads;
    const int64_t tokens = (int64_t)a.c.num_seqs * a.new_tokens;
    int each = 1;
    while (each < 8 && kGroups * each < rows && tokens * ((rows + 2 * kGroups * each - 1) / (2 * kGroups * each)) >= 148 * 16) each *= 2;
    const int64_t blocks = tokens * ((rows + kGroups * each - 1) / (kGroups * each));
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    k_cache_append<T, kLanes><<<(unsigned)blocks, kAppendThreads, 0, s>>>(a, each); count_launch();
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_cache_append(const AppendArgs &a, int dtype, cudaStream_t s)
{
    const int lanes = (a.c.head_dim + 7) / 8;
    if (dtype == G10_BF16) return lanes <= 8 ? launch<__nv_bfloat16, 8>(a, s) : lanes <= 16 ? launch<__nv_bfloat16, 16>(a, s) : launch<__nv_bfloat16, 32>(a, s);
    return lanes <= 8 ? launch<__half, 8>(a, s) : lanes <= 16 ? launch<__half, 16>(a, s) : launch<__half, 32>(a, s);
}

}  // namespace g10
