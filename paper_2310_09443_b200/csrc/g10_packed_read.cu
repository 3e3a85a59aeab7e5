// Reading rows of 8-bit codes back.
#include "g10_packed.cuh"

namespace g10 {
namespace {

constexpr int kReadThreads = 256, kEach = 4;

// Pure traffic: head_dim codes and a scale in, 2 * head_dim bytes out for each row.  A thread takes 8 codes (8 bytes in, 16 out: a warp's accesses lie side by side
// in both directions) of key and value of a (token, head), kEach of those at a time.  A block takes `run` tokens of a sequence.
template <typename T, typename Code>
__global__ void __launch_bounds__(kReadThreads) k_packed_read(const ReadArgs a, int runs, int run, unsigned unit_mul)
{
    const CacheView &c = a.c;
    const int s = (int)(blockIdx.x / (unsigned)runs), t0 = (int)(blockIdx.x - (unsigned)s * (unsigned)runs) * run;
    ull bad = 0;
    const int length = cache_length(c, s, bad);
    const int64_t start = a.starts != nullptr ? __ldg(&a.starts[s]) : 0;
    const unsigned units = (unsigned)c.head_dim / 8, all = units * (unsigned)c.kv_heads;         // of a row, of a token: 8 codes each
    const unsigned n = (unsigned)min(run, a.tokens - t0) * all;
#pragma unroll 1
    for (unsigned i0 = threadIdx.x; i0 < n; i0 += kReadThreads * kEach) {
        uint2 x[kEach], y[kEach];
        float2 scale[kEach];
        int64_t k_at[kEach], v_at[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const unsigned i = i0 + j * kReadThreads;
            x[j] = y[j] = make_uint2(0, 0); scale[j] = make_float2(0.0f, 0.0f); k_at[j] = v_at[j] = 0;
            if (i >= n) continue;
            const unsigned row = (unsigned)(((ull)i * unit_mul) >> 32), t = row / (unsigned)c.kv_heads, head = row - t * (unsigned)c.kv_heads, unit = i - row * units;
            k_at[j] = 2 * (s * a.k_seq + (int64_t)(t0 + (int)t) * a.k_token + head * a.k_head + 8 * unit);
            v_at[j] = 2 * (s * a.v_seq + (int64_t)(t0 + (int)t) * a.v_token + head * a.v_head + 8 * unit);
            const int64_t slot = start + t0 + (int)t;
            if (slot < 0 || slot >= length) continue;
            const Spot spot = cache_spot(c, s, (int)slot, bad);
            if (spot.page < 0) continue;
            const int64_t at = 16 * (int64_t)cache_row(c, spot, (int)head) + 8 * unit;
            if (a.k != nullptr) x[j] = __ldg((const uint2 *)(c.k + at));
            if (a.v != nullptr) y[j] = __ldg((const uint2 *)(c.v + at));
            scale[j] = __ldg(&a.scales[cache_cell(c, spot, (int)head)]);
        }
        auto values = [](uint2 u, float by) -> uint4 {
            const float4 p = Code::unpack(u.x), q = Code::unpack(u.y);
            return make_uint4(Pair<T>::pack(p.x * by, p.y * by), Pair<T>::pack(p.z * by, p.w * by), Pair<T>::pack(q.x * by, q.y * by), Pair<T>::pack(q.z * by, q.w * by));
        };
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (i0 + j * kReadThreads < n) {
                if (a.k != nullptr) *(uint4 *)(a.k + k_at[j]) = values(x[j], scale[j].x);
                if (a.v != nullptr) *(uint4 *)(a.v + v_at[j]) = values(y[j], scale[j].y);
            }
    }
    if (bad != 0) raise_status(c.status, bad);
}

template <typename T, typename Code>
cudaError_t launch(const ReadArgs &a, cudaStream_t s)
{
    // (a block does not look beyond 2^32 / units units, for which the product below finds the row exactly; runs are as long as leave 8 blocks for every SM)
    const unsigned units = (unsigned)a.c.head_dim / 8, all = units * (unsigned)a.c.kv_heads;
    int run = (int)((kReadThreads * kEach + all - 1) / all);
    while (run < 64 && 2 * run <= a.tokens && (int64_t)a.c.num_seqs * ((a.tokens + 2 * run - 1) / (2 * run)) >= 148 * 8 && (int64_t)2 * run * all <= 65536) run *= 2;
    const int runs = (int)(((int64_t)a.tokens + run - 1) / run);
    const int64_t blocks = (int64_t)a.c.num_seqs * runs;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    const unsigned unit_mul = (unsigned)((((uint64_t)1 << 32) + units - 1) / units);
    k_packed_read<T, Code><<<(unsigned)blocks, kReadThreads, 0, s>>>(a, runs, run, unit_mul); count_launch();
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_packed_read(const ReadArgs &a, int dtype, int code, cudaStream_t s)
{
    if (code == G10_INT8) return dtype == G10_BF16 ? launch<__nv_bfloat16, Int8>(a, s) : launch<__half, Int8>(a, s);
    return dtype == G10_BF16 ? launch<__nv_bfloat16, E4m3>(a, s) : launch<__half, E4m3>(a, s);
}

}  // namespace g10
