// Reading rows of 8-bit codes back.
#include "g10_packed.cuh"

namespace g10 {
namespace {

constexpr int kReadThreads = 256, kEach = 4;

__device__ __forceinline__ void store32(void *to, const uint4 &x, const uint4 &y)
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w), "r"(y.x), "r"(y.y), "r"(y.z), "r"(y.w) : "memory");
}

// Pure traffic: head_dim codes and a scale in, 2 * head_dim bytes out for each row.  A thread takes 16 codes of key and value of a (token, head), always the same place of
// the same head, and goes through the block's tokens, kEach of them at a time: what it works out for a token is the slot's page.  A token's units (16 codes each) are `per`
// threads' or, where they are more than a block has, blockIdx.y's part of them; a block takes `run` tokens of a sequence, kReadThreads / per at a time.
template <typename T, typename Code, bool kWhole>        // kWhole: outputs may be written 32 bytes at a time
__global__ void __launch_bounds__(kReadThreads) k_packed_read(const ReadArgs a, int runs, int run, int per)
{
    const CacheView &c = a.c;
    // (tokens' numbers have no sign: a block's last ones, and those that a thread looks ahead at, may lie behind 2^31)
    const int s = (int)(blockIdx.x / (unsigned)runs);
    const unsigned t0 = (blockIdx.x - (unsigned)s * (unsigned)runs) * (unsigned)run, t1 = min((unsigned)a.tokens, t0 + (unsigned)run);
    const unsigned team = threadIdx.x / (unsigned)per, teams = kReadThreads / (unsigned)per;
    const int chunks = c.head_dim / 16, unit = (int)blockIdx.y * per + (int)(threadIdx.x - team * (unsigned)per);
    const int head = unit / chunks, chunk = unit - head * chunks;
    if (team >= teams || head >= c.kv_heads) return;
    ull bad = 0;
    const int length = cache_length(c, s, bad);
    const int64_t start = a.starts != nullptr ? __ldg(&a.starts[s]) : 0;
    char *const k_to = a.k + 2 * (s * a.k_seq + head * a.k_head + 16 * chunk), *const v_to = a.v + 2 * (s * a.v_seq + head * a.v_head + 16 * chunk);
#pragma unroll 1
    for (unsigned t = t0 + team; t < t1; t += kEach * teams) {
        uint4 x[kEach], y[kEach];
        float2 scale[kEach];
        Spot spot[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int64_t slot = start + t + j * teams;
            spot[j] = Spot{-1, 0};
            if (t + j * teams < t1 && slot >= 0 && slot < length) spot[j] = cache_spot(c, s, (int)slot, bad);
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            x[j] = y[j] = make_uint4(0, 0, 0, 0); scale[j] = make_float2(0.0f, 0.0f);
            if (spot[j].page < 0) continue;
            const int64_t at = 16 * ((int64_t)cache_row(c, spot[j], head) + chunk);
            if (a.k != nullptr) x[j] = __ldg((const uint4 *)(c.k + at));
            if (a.v != nullptr) y[j] = __ldg((const uint4 *)(c.v + at));
            scale[j] = __ldg(&a.scales[cache_cell(c, spot[j], head)]);
        }
        auto put = [](char *to, const uint4 &u, float by) {
            const unsigned w[4] = {u.x, u.y, u.z, u.w};
            uint4 o[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float4 p = Code::unpack(w[2 * h]), q = Code::unpack(w[2 * h + 1]);
                o[h] = make_uint4(Pair<T>::pack(p.x * by, p.y * by), Pair<T>::pack(p.z * by, p.w * by), Pair<T>::pack(q.x * by, q.y * by), Pair<T>::pack(q.z * by, q.w * by));
            }
            if (kWhole) store32(to, o[0], o[1]);
            else { *(uint4 *)to = o[0]; *(uint4 *)(to + 16) = o[1]; }
        };
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (t + j * teams < t1) {
                if (a.k != nullptr) put(k_to + 2 * (int64_t)(t + j * teams) * a.k_token, x[j], scale[j].x);
                if (a.v != nullptr) put(v_to + 2 * (int64_t)(t + j * teams) * a.v_token, y[j], scale[j].y);
            }
    }
    if (bad != 0) raise_status(c.status, bad);
}

template <typename T, typename Code>
cudaError_t launch(const ReadArgs &a, cudaStream_t s)
{
    const int units = a.c.kv_heads * (a.c.head_dim / 16), per = units < kReadThreads ? units : kReadThreads, teams = kReadThreads / per;
    const unsigned parts = (unsigned)((units + per - 1) / per);
    // (runs of kEach tokens a thread, or as many more as leave 16 blocks for every SM)
    int64_t run = (int64_t)kEach * teams;
    while (run < 64 * teams && run < a.tokens && (int64_t)a.c.num_seqs * ((a.tokens + 2 * run - 1) / (2 * run)) * parts >= 148 * 16) run *= 2;
    const int64_t runs = (a.tokens + run - 1) / run, blocks = a.c.num_seqs * runs;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    const bool whole = (((uintptr_t)a.k | (uintptr_t)a.v) & 31u) == 0 && ((a.k_seq | a.k_token | a.k_head | a.v_seq | a.v_token | a.v_head) & 15) == 0;
    const auto kernel = whole ? k_packed_read<T, Code, true> : k_packed_read<T, Code, false>;
    kernel<<<dim3((unsigned)blocks, parts), kReadThreads, 0, s>>>(a, (int)runs, (int)run, per); count_launch();
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_packed_read(const ReadArgs &a, int dtype, int code, cudaStream_t s)
{
    if (code == G10_INT8) return dtype == G10_BF16 ? launch<__nv_bfloat16, Int8>(a, s) : launch<__half, Int8>(a, s);
    return dtype == G10_BF16 ? launch<__nv_bfloat16, E4m3>(a, s) : launch<__half, E4m3>(a, s);
}

}  // namespace g10
