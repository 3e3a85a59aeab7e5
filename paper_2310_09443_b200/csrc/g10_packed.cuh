// Rows of 8-bit codes: what a code stands for, and back.
#pragma once
#include <cuda_fp8.h>

#include "g10_cache.cuh"

namespace g10 {

// The two kinds of codes.  Values are taken out as pairs of fp16, which holds both exactly: the matrix instructions take them from there, with the scales
// left to the logits and the weights.
struct Int8 {
    static constexpr float kLargest = 127.0f;
    // four codes to two pairs of fp16 (below 0x64 a byte, its top bit flipped, is 1024 + 128 + code)
    static __device__ __forceinline__ void halves(unsigned u, unsigned &a, unsigned &b)
    {
        const unsigned x = u ^ 0x80808080u, kMore = 0x64806480u, y = __byte_perm(x, kMore, 0x5150), z = __byte_perm(x, kMore, 0x5352);
        const __half2 p = __hsub2(*(const __half2 *)&y, *(const __half2 *)&kMore), q = __hsub2(*(const __half2 *)&z, *(const __half2 *)&kMore);
        a = *(const unsigned *)&p; b = *(const unsigned *)&q;
    }
    // four numbers up to kLargest to four codes
    static __device__ __forceinline__ unsigned pack(float a, float b, float c, float d, float by)
    {
        // (1.5 * 2^23 more: the sum's last bits are the rounded number)
        const float kShift = 12582912.0f;
        const unsigned x = __float_as_uint(fmaf(a, by, kShift)), y = __float_as_uint(fmaf(b, by, kShift));
        const unsigned z = __float_as_uint(fmaf(c, by, kShift)), w = __float_as_uint(fmaf(d, by, kShift));
        return __byte_perm(__byte_perm(x, y, 0x0040), __byte_perm(z, w, 0x0040), 0x5410);
    }
    // four codes to four numbers (2^23 and a byte beside each other: the byte's number, 128 more)
    static __device__ __forceinline__ float4 unpack(unsigned u)
    {
        const unsigned x = u ^ 0x80808080u, kOne = 0x4b000000u;
        const float kLess = 8388736.0f;
        return make_float4(__uint_as_float(__byte_perm(x, kOne, 0x7440)) - kLess, __uint_as_float(__byte_perm(x, kOne, 0x7441)) - kLess,
                           __uint_as_float(__byte_perm(x, kOne, 0x7442)) - kLess, __uint_as_float(__byte_perm(x, kOne, 0x7443)) - kLess);
    }
};
struct E4m3 {
    static constexpr float kLargest = 448.0f;
    // four codes to two pairs of fp16
    static __device__ __forceinline__ void halves(unsigned u, unsigned &a, unsigned &b)
    {
        const __half2 x = halves(u & 0xffffu), y = halves(u >> 16);
        a = *(const unsigned *)&x; b = *(const unsigned *)&y;
    }
    static __device__ __forceinline__ unsigned pack(float a, float b, float c, float d, float by)
    {
        const unsigned x = __nv_cvt_float2_to_fp8x2(make_float2(a * by, b * by), __NV_SATFINITE, __NV_E4M3);
        const unsigned y = __nv_cvt_float2_to_fp8x2(make_float2(c * by, d * by), __NV_SATFINITE, __NV_E4M3);
        return x | y << 16;
    }
    static __device__ __forceinline__ __half2 halves(unsigned two) { return __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3)); }
    static __device__ __forceinline__ float4 unpack(unsigned u)
    {
        const float2 x = __half22float2(halves(u & 0xffffu)), y = __half22float2(halves(u >> 16));
        return make_float4(x.x, x.y, y.x, y.y);
    }
};

__device__ __forceinline__ float log2_of(float x)
{
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Eight elements of a row whose largest magnitude is `top` (its bits), as codes, and the row's scale.
template <typename Code>
__device__ __forceinline__ uint2 packed_row(const float (&x)[8], unsigned top, float &scale)
{
    const float most = __uint_as_float(top);
    scale = most / Code::kLargest;
    if (top >= 0x7f800000u) { scale = __uint_as_float(0x7fc00000u); return make_uint2(0, 0); }   // not a number
    if (most < 7.8886090522101181e-31f) { scale = 0.0f; return make_uint2(0, 0); }               // 2^-100: Q / most has to be one
    const float by = Code::kLargest / most;
    return make_uint2(Code::pack(x[0], x[1], x[2], x[3], by), Code::pack(x[4], x[5], x[6], x[7], by));
}

}  // namespace g10
