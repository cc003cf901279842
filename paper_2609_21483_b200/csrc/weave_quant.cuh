// Rows to 8-bit integers with one scale per row: scale = max|x| / 127, q = the integer nearest to x / scale, ties to
// even, decided in exact arithmetic.  bf16 rows need that: with 8 bits of mantissa on both sides the quotient sits on a
// tie, or within a rounding of one, for about one value in a thousand, and a quotient rounded to fp32 would decide
// those by its own rounding.
//
// Bound: HBM (3 bytes per bf16 value).  One block per row, the row kept in registers between the two passes over it.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>
#include "weave_gemm.cuh"

namespace weave {

constexpr int kQuantThreads = 256;
constexpr int kQuantKeep = 8;          // 16-byte vectors of a row that a thread keeps

struct QuantRow {
    float k, s, inv, half;             // x and the scale are multiplied by k (a power of two, exact) so that 1 / s is finite
    bool zero;                         // nothing but zeros: an all-zero row, or one with inf or NaN in it
};

// t is within one of the quotient; the remainder d = x - t s is exact (a multiple of half an ulp of s below s), so
// comparing it with s / 2 decides the rounding
__device__ __forceinline__ int quant_one(float x, const QuantRow &r)
{
    const float y = x * r.k;
    float t = rintf(y * r.inv);
    const float d = fmaf(-t, r.s, y);
    if (fabsf(d) >= r.half) {
        if (fabsf(d) > r.half || ((int)t & 1)) t += d > 0.0f ? 1.0f : -1.0f;
        t = fminf(fmaxf(t, -127.0f), 127.0f);        // only rows whose scale is a denormal number reach beyond
    }
    return (int)t;
}
__device__ __forceinline__ uint32_t quant_four(float a, float b, float c, float d, const QuantRow &r)
{
    if (r.zero) return 0u;
    return (uint32_t)(quant_one(a, r) & 255) | (uint32_t)(quant_one(b, r) & 255) << 8 | (uint32_t)(quant_one(c, r) & 255) << 16 |
           (uint32_t)quant_one(d, r) << 24;
}

// the largest |x| as bits: NaN above inf above every number, so that either shows in the result
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t abs_bits_bf16x2(uint32_t u)
{
    return max((u << 16) & 0x7FFFFFFFu, u & 0x7FFF0000u);
}

__device__ __forceinline__ QuantRow quant_row(uint32_t amax_bits, float &scale)
{
    QuantRow r;
    scale = __fdiv_rn(__uint_as_float(amax_bits), 127.0f);
    r.zero = amax_bits >= 0x7F800000u || scale == 0.0f;
    r.k = scale < 1e-30f ? 18446744073709551616.0f : 1.0f;      // 2^64
    r.s = scale * r.k;
    r.inv = __fdiv_rn(1.0f, r.s);
    r.half = 0.5f * r.s;
    return r;
}

// kVec: rows start on 16-byte boundaries and are whole 16-byte vectors long
template <typename X, bool kVec>
__global__ void __launch_bounds__(kQuantThreads) weave_quant_kernel(const X *x, int8_t *q, float *scale, long long rows, long long cols)
{
    __shared__ uint32_t warp_max[2][kQuantThreads / 32];
    constexpr bool kBf16 = sizeof(X) == 2;
    constexpr int kPer = 16 / sizeof(X);
    int flip = 0;
    pdl_launch_dependents();
    pdl_wait();
    for (long long row = blockIdx.x; row < rows; row += gridDim.x, flip ^= 1) {
        const X *src = x + row * cols;
        int8_t *dst = q + row * cols;
        uint32_t m = 0;
        uint4 keep[kQuantKeep];
        const long long nv = cols / kPer;
        if constexpr (kVec) {
            auto max_of = [&](const uint4 &v) {
                if constexpr (kBf16)
                    m = max(m, max(max(abs_bits_bf16x2(v.x), abs_bits_bf16x2(v.y)), max(abs_bits_bf16x2(v.z), abs_bits_bf16x2(v.w))));
                else
                    m = max(m, max(max(v.x & 0x7FFFFFFFu, v.y & 0x7FFFFFFFu), max(v.z & 0x7FFFFFFFu, v.w & 0x7FFFFFFFu)));
            };
#pragma unroll
            for (int i = 0; i < kQuantKeep; ++i) {
                const long long at = threadIdx.x + (long long)i * kQuantThreads;
                keep[i] = at < nv ? reinterpret_cast<const uint4 *>(src)[at] : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < kQuantKeep; ++i) max_of(keep[i]);
            for (long long at = threadIdx.x + (long long)kQuantKeep * kQuantThreads; at < nv; at += kQuantThreads)
                max_of(reinterpret_cast<const uint4 *>(src)[at]);
        } else {
            for (long long at = threadIdx.x; at < cols; at += kQuantThreads) m = max(m, abs_bits((float)src[at]));
        }
        m = __reduce_max_sync(0xffffffffu, m);
        if ((threadIdx.x & 31) == 0) warp_max[flip][threadIdx.x >> 5] = m;
        __syncthreads();
        m = 0;
#pragma unroll
        for (int w = 0; w < kQuantThreads / 32; ++w) m = max(m, warp_max[flip][w]);
        float s;
        const QuantRow r = quant_row(m, s);
        if (threadIdx.x == 0) scale[row] = s;
        if constexpr (kVec) {
            auto put = [&](const uint4 &v, long long at) {
                if constexpr (kBf16) {
                    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
                    float f[8];
#pragma unroll
                    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
                    reinterpret_cast<uint2 *>(dst)[at] = make_uint2(quant_four(f[0], f[1], f[2], f[3], r), quant_four(f[4], f[5], f[6], f[7], r));
                } else {
                    reinterpret_cast<uint32_t *>(dst)[at] =
                        quant_four(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w), r);
                }
            };
#pragma unroll
            for (int i = 0; i < kQuantKeep; ++i) {
                const long long at = threadIdx.x + (long long)i * kQuantThreads;
                if (at < nv) put(keep[i], at);
            }
            for (long long at = threadIdx.x + (long long)kQuantKeep * kQuantThreads; at < nv; at += kQuantThreads)
                put(reinterpret_cast<const uint4 *>(src)[at], at);
        } else {
            for (long long at = threadIdx.x; at < cols; at += kQuantThreads) dst[at] = r.zero ? 0 : (int8_t)quant_one((float)src[at], r);
        }
    }
}

}  // namespace weave
