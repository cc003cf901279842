// Rows to 8-bit integers with one scale per row: scale = max|x| / 127, q = the integer nearest to x / scale, ties to
// even, decided in exact arithmetic.  bf16 rows need that: with 8 bits of mantissa on both sides the quotient sits on a
// tie, or within a rounding of one, for about one value in a thousand, and a quotient rounded to fp32 would decide
// those by its own rounding.
//
// Bound: HBM (3 bytes per bf16 value).  A row is read once: its threads keep it in registers (up to eight 16-byte
// vectors each) between the search for the largest magnitude and the rounding.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>
#include "weave_gemm.cuh"

namespace weave {

constexpr float kQuantMagic = 12582912.0f;      // 1.5 * 2^23: adding it rounds to an integer, in the low bits of the sum

struct QuantRow {
    float k, s, inv, half;             // x and the scale are multiplied by k (a power of two, exact) so that 1 / s is finite
    bool zero;                         // nothing but zeros: an all-zero row, or one with inf or NaN in it
};

// The sum's low bits are the integer; it may be one off next to a tie, and a tie may have gone the wrong way, which the
// remainder shows: d = x - t s is exact (a multiple of half an ulp of s, at most about s / 2).
__device__ __forceinline__ uint32_t quant_guess(float x, const QuantRow &r, float &d)
{
    const float y = x * r.k;
    const float m = fmaf(y, r.inv, kQuantMagic);
    d = fmaf(kQuantMagic - m, r.s, y);
    return __float_as_uint(m);
}
__device__ __forceinline__ uint32_t quant_mend(uint32_t v, float d, const QuantRow &r)
{
    const float ad = fabsf(d);
    int t = (int)(v - __float_as_uint(kQuantMagic));
    if (ad > r.half || (ad == r.half && (t & 1))) t += d > 0.0f ? 1 : -1;
    return (uint32_t)min(max(t, -127), 127);       // beyond only in a row whose scale is a denormal number
}
__device__ __forceinline__ uint32_t quant_four(float a, float b, float c, float e, const QuantRow &r)
{
    float d[4];
    uint32_t v[4] = {quant_guess(a, r, d[0]), quant_guess(b, r, d[1]), quant_guess(c, r, d[2]), quant_guess(e, r, d[3])};
    if (fmaxf(fmaxf(fabsf(d[0]), fabsf(d[1])), fmaxf(fabsf(d[2]), fabsf(d[3]))) >= r.half || r.k != 1.0f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = quant_mend(v[i], d[i], r);
    }
    return r.zero ? 0u : __byte_perm(__byte_perm(v[0], v[1], 0x0040), __byte_perm(v[2], v[3], 0x0040), 0x5410);
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

// the largest magnitudes as bits: NaN above inf above every number, so that either shows in the result
template <class X>
__device__ __forceinline__ uint32_t quant_max(uint32_t m, const uint4 &v)
{
    if constexpr (sizeof(X) == 2) {      // two maxima, one per half
        m = __vmaxu2(__vmaxu2(m, v.x & 0x7FFF7FFFu), v.y & 0x7FFF7FFFu);
        return __vmaxu2(__vmaxu2(m, v.z & 0x7FFF7FFFu), v.w & 0x7FFF7FFFu);
    } else {
        m = max(max(m, v.x & 0x7FFFFFFFu), v.y & 0x7FFFFFFFu);
        return max(max(m, v.z & 0x7FFFFFFFu), v.w & 0x7FFFFFFFu);
    }
}
template <class X>
__device__ __forceinline__ void quant_put(int8_t *dst, int at, const uint4 &v, const QuantRow &r)
{
    if constexpr (sizeof(X) == 2) {
        const uint32_t lo = quant_four(bf16lo_to_f32(v.x), bf16hi_to_f32(v.x), bf16lo_to_f32(v.y), bf16hi_to_f32(v.y), r);
        const uint32_t hi = quant_four(bf16lo_to_f32(v.z), bf16hi_to_f32(v.z), bf16lo_to_f32(v.w), bf16hi_to_f32(v.w), r);
        reinterpret_cast<uint2 *>(dst)[at] = make_uint2(lo, hi);
    } else {
        reinterpret_cast<uint32_t *>(dst)[at] =
            quant_four(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w), r);
    }
}

// One row by kThreads threads (tid from 0), which meet at __syncthreads() or, kNamed, at named barrier 1.  kVec: rows
// start on 16-byte boundaries and are whole 16-byte vectors long.  kKeep: vectors that a thread keeps.  `part`: one word of
// shared memory per warp.  The row is read past L1, as another SM may just have written it.
template <class X, int kThreads, int kKeep, bool kVec, bool kNamed>
__device__ __forceinline__ void quant_row_by(const X *x, int8_t *q, float *scale, long long row, int cols, int tid, uint32_t *part)
{
    const X *src = x + row * cols;
    int8_t *dst = q + row * cols;
    const uint4 *vec = reinterpret_cast<const uint4 *>(src);
    const int nv = cols / (int)(16 / sizeof(X));
    uint32_t m = 0;
    uint4 keep[kKeep];
    if constexpr (kVec) {
#pragma unroll
        for (int i = 0; i < kKeep; ++i) keep[i] = tid + i * kThreads < nv ? __ldcg(vec + tid + i * kThreads) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < kKeep; ++i) m = quant_max<X>(m, keep[i]);
#pragma unroll 1
        for (int at = tid + kKeep * kThreads; at < nv; at += kThreads) m = quant_max<X>(m, __ldcg(vec + at));
        if constexpr (sizeof(X) == 2) m = max(m << 16, m & 0xFFFF0000u);
    } else {
        for (int at = tid; at < cols; at += kThreads) m = max(m, __float_as_uint((float)src[at]) & 0x7FFFFFFFu);
    }
    m = __reduce_max_sync(0xffffffffu, m);
    if constexpr (kThreads > 32) {
        if ((tid & 31) == 0) part[tid >> 5] = m;
        if constexpr (kNamed) named_barrier_sync<1, kThreads>();
        else __syncthreads();
        m = part[0];
#pragma unroll
        for (int w = 1; w < kThreads / 32; ++w) m = max(m, part[w]);
        // (a second row needs another barrier before it writes `part`: callers have one)
    }
    float s;
    const QuantRow r = quant_row(m, s);
    if (tid == 0) scale[row] = s;
    if constexpr (kVec) {
        // kNamed: a rolled loop that turns the vectors through keep[0].  In a kernel that runs this once, beside a saturated
        // HBM, it is the fetch of unrolled instructions that takes the time (13 us for a row of 14336 instead of 2)
        if constexpr (kNamed) {
#pragma unroll 1
            for (int at = tid; at < nv && at < kKeep * kThreads; at += kThreads) {
                quant_put<X>(dst, at, keep[0], r);
#pragma unroll
                for (int i = 1; i < kKeep; ++i) keep[i - 1] = keep[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < kKeep; ++i)
                if (tid + i * kThreads < nv) quant_put<X>(dst, tid + i * kThreads, keep[i], r);
        }
#pragma unroll 1
        for (int at = tid + kKeep * kThreads; at < nv; at += kThreads) quant_put<X>(dst, at, __ldcg(vec + at), r);
    } else {
        for (int at = tid; at < cols; at += kThreads) {
            float d;
            const uint32_t v = quant_guess((float)src[at], r, d);
            dst[at] = r.zero ? 0 : (int8_t)quant_mend(v, d, r);
        }
    }
}

// one row per block
template <class X, int kThreads, bool kVec>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) weave_quant_kernel(const X *x, int8_t *q, float *scale, int cols)
{
    __shared__ uint32_t part[kThreads / 32];
    pdl_launch_dependents();
    pdl_wait();
    quant_row_by<X, kThreads, 8, kVec, false>(x, q, scale, blockIdx.x, cols, threadIdx.x, part);
}

// one row per warp, for many short rows: what they cost in blocks of their own is the start of a block
template <class X, bool kVec>
__global__ void __launch_bounds__(128, 8) weave_quant_short_kernel(const X *x, int8_t *q, float *scale, int rows, int cols)
{
    pdl_launch_dependents();
    pdl_wait();
    const int row = blockIdx.x * 4 + (threadIdx.x >> 5);
    if (row < rows) quant_row_by<X, 32, 8, kVec, false>(x, q, scale, row, cols, threadIdx.x & 31, nullptr);
}

}  // namespace weave
