// The products of the feed-forward block for small batches (up to 128 tokens), where they are a stream of weights:
// weights on the MMA's M axis (two accumulators of 128 rows: gate and up rows, or 256 rows of one matrix), tokens on
// its N axis.  The work - (tile of 256 weight rows) x (128 bytes of K) units, 32 KB of weights each - is cut into
// ranges of equal length, one per CTA, that pass over tile borders.  A tile that several CTAs share is added up from
// their partial sums in the workspace by the one that arrives last, in the order of K: nobody waits, and the result
// does not depend on who it is.
//
// Bound: HBM (the weights).  Up to 190 KB per SM are in flight.
#pragma once
#include "weave_gemm.cuh"

namespace weave {

// ------------------------------------------------------------------------------------ PTX forms, one CTA

__device__ __forceinline__ void tmem_alloc_one(uint32_t *smem_slot, uint32_t ncols)
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(smem_slot)), "r"(ncols) : "memory");
}
__device__ __forceinline__ void tmem_relinquish_one()
{
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc_one(uint32_t taddr, uint32_t ncols)
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
__device__ __forceinline__ void tc_commit_one(uint64_t *bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// four products over 128 bytes of K, K-major operands; called by one thread
template <bool kI8>
__device__ __forceinline__ void ffn_mma_kstep_one(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate_first)
{
#define WEAVE_KSTEP_ONE(KIND)                                                                   \
    asm volatile(                                                                               \
        "{\n\t.reg .pred pa, pt;\n\t"                                                           \
        ".reg .b64 a1, a2, a3, b1, b2, b3;\n\t"                                                 \
        "setp.ne.b32 pa, %4, 0;\n\t"                                                            \
        "setp.eq.u32 pt, %0, %0;\n\t"                                                           \
        "add.u64 a1, %1, 2;\n\tadd.u64 a2, %1, 4;\n\tadd.u64 a3, %1, 6;\n\t"                    \
        "add.u64 b1, %2, 2;\n\tadd.u64 b2, %2, 4;\n\tadd.u64 b3, %2, 6;\n\t"                    \
        "tcgen05.mma.cta_group::1.kind::" KIND " [%0], %1, %2, %3, pa;\n\t"                     \
        "tcgen05.mma.cta_group::1.kind::" KIND " [%0], a1, b1, %3, pt;\n\t"                     \
        "tcgen05.mma.cta_group::1.kind::" KIND " [%0], a2, b2, %3, pt;\n\t"                     \
        "tcgen05.mma.cta_group::1.kind::" KIND " [%0], a3, b3, %3, pt;\n\t}"                    \
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate_first) : "memory")
    if (kI8) WEAVE_KSTEP_ONE("i8");
    else WEAVE_KSTEP_ONE("f16");
#undef WEAVE_KSTEP_ONE
}
__device__ __forceinline__ void tma_load_2d_one(uint32_t dst, const void *map, int x, int y, uint64_t *bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(smem_u32(bar))
                 : "memory");
}
__device__ __forceinline__ void tma_load_3d_one(uint32_t dst, const void *map, int x, int y, int z, uint64_t *bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
                 : "memory");
}
// 32 lanes x 8 consecutive columns
__device__ __forceinline__ void tmem_ld_32x8(uint32_t taddr, uint32_t (&r)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void tmem_ld_wait8x2(uint32_t (&r)[8], uint32_t (&s)[8])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(s[0]),
                   "+r"(s[1]), "+r"(s[2]), "+r"(s[3]), "+r"(s[4]), "+r"(s[5]), "+r"(s[6]), "+r"(s[7])
                 :: "memory");
}

// a barrier of some of the CTA's warps that also says whether all of their threads brought `true`
template <int ID, int THREADS>
__device__ __forceinline__ bool named_barrier_and(bool mine)
{
    uint32_t all;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "bar.red.and.pred q, %2, %3, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(all)
        : "r"((uint32_t)mine), "n"(ID), "n"(THREADS)
        : "memory");
    return all != 0;
}

// ------------------------------------------------------------------------------------ the kernel

struct alignas(64) FfnStreamArgs {
    CUtensorMap w;           // 256 rows x 128 bytes of K; gated: 128 rows x 128 bytes of each half
    CUtensorMap x;           // box_t rows x 128 bytes of K
    FfnCtl *ctl;
    unsigned long long timeout_ns;
    unsigned *arrived;       // [tiles], zero between launches
    uint32_t *partials;      // [CTA][first, last segment][accumulator][T][128]
    const float *row_scale;  // 8-bit forms: [T] and [N] (gated: [2N], gate then up)
    const float *col_scale;
    void *out;
    long long ld_out;
    int T, N;                // N: columns of the result
    int ksteps, tiles;
    int units;               // ksteps * tiles
    int units_per_cta;
    int box_t, stages;
    int out_f32;
};

constexpr int kFfnStreamThreads = 320;           // producer, issuer, eight epilogue warps
constexpr int kFfnStreamMaxT = 128;
constexpr int kFfnStreamWeights = 32768;         // weight bytes of a unit
constexpr int kFfnStreamSmem = 232448 - 1024;
constexpr int kFfnStreamMaxStages = 6;

struct FfnStreamBars {
    uint64_t full[kFfnStreamMaxStages], empty[kFfnStreamMaxStages];
    uint64_t acc_full[2], acc_empty[2];
    uint32_t tmem_base;
    uint32_t last;
};

// stages that fit beside the barriers
__host__ __device__ inline int ffn_stream_stages(int box_t)
{
    const int n = (kFfnStreamSmem - 1024 - 512) / (kFfnStreamWeights + box_t * 128);
    return n < kFfnStreamMaxStages ? n : kFfnStreamMaxStages;
}

struct FfnSegment { int tile, k0, k1; };
__host__ __device__ inline FfnSegment ffn_segment_at(int at, int end, int ksteps)
{
    FfnSegment s;
    s.tile = at / ksteps;
    s.k0 = at - s.tile * ksteps;
    s.k1 = s.k0 + (end - at);
    if (s.k1 > ksteps) s.k1 = ksteps;
    return s;
}
// the partial sums of CTA c for this tile lie in its first or in its second place
__host__ __device__ inline int ffn_partial_slot(int c, int tile, int units_per_cta, int ksteps)
{
    return 2 * c + (c * units_per_cta / ksteps == tile ? 0 : 1);
}

template <bool kI8, bool kGated>
__device__ __forceinline__ void ffn_stream_store(const FfnStreamArgs &p, int t, int row, uint32_t a, uint32_t b, float sw0, float sw1)
{
    // row: this thread's row of the tile's first accumulator in the result
    const long long at = (long long)t * p.ld_out + row;
    float fa, fb;
    if constexpr (kI8) {
        const float sx = p.row_scale[t];
        fa = __int2float_rn((int)a) * (sx * sw0);
        fb = __int2float_rn((int)b) * (sx * sw1);
    } else {
        fa = __uint_as_float(a);
        fb = __uint_as_float(b);
    }
    if constexpr (kGated) {
        if (row < p.N) static_cast<__nv_bfloat16 *>(p.out)[at] = __float2bfloat16_rn(gated(fa, fb));
    } else if (p.out_f32) {
        if (row < p.N) static_cast<float *>(p.out)[at] = fa;
        if (row + 128 < p.N) static_cast<float *>(p.out)[at + 128] = fb;
    } else {
        if (row < p.N) static_cast<__nv_bfloat16 *>(p.out)[at] = __float2bfloat16_rn(fa);
        if (row + 128 < p.N) static_cast<__nv_bfloat16 *>(p.out)[at + 128] = __float2bfloat16_rn(fb);
    }
}

template <bool kI8>
__device__ __forceinline__ uint32_t add_partial(uint32_t a, uint32_t b)
{
    return kI8 ? a + b : __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
}

// kTok tokens of a shared tile: the partial sums of its segments c0 .. c1, in this order, kSegs of them on their way at once
template <bool kI8, bool kGated, int kTok, int kSegs>
__device__ __forceinline__ void ffn_stream_join(const FfnStreamArgs &p, int tile, int c0, int c1, int t0, int lane_row, int row, float sw0, float sw1)
{
    uint32_t sum[2][kTok];
#pragma unroll
    for (int i = 0; i < kTok; ++i) sum[0][i] = sum[1][i] = 0u;
    for (int c = c0; c <= c1; c += kSegs) {
        uint32_t v[kSegs][2][kTok];
#pragma unroll
        for (int s = 0; s < kSegs; ++s) {
            const uint32_t *src = p.partials + (size_t)ffn_partial_slot(min(c + s, c1), tile, p.units_per_cta, p.ksteps) * 256 * p.T + lane_row;
#pragma unroll
            for (int i = 0; i < kTok; ++i) {
                const bool there = c + s <= c1 && t0 + i < p.T;
                v[s][0][i] = there ? __ldcg(src + (size_t)(t0 + i) * 128) : 0u;
                v[s][1][i] = there ? __ldcg(src + (size_t)(p.T + t0 + i) * 128) : 0u;
            }
        }
#pragma unroll
        for (int s = 0; s < kSegs; ++s)
#pragma unroll
            for (int i = 0; i < kTok; ++i) {
                sum[0][i] = add_partial<kI8>(sum[0][i], v[s][0][i]);
                sum[1][i] = add_partial<kI8>(sum[1][i], v[s][1][i]);
            }
    }
#pragma unroll
    for (int i = 0; i < kTok; ++i)
        if (t0 + i < p.T) ffn_stream_store<kI8, kGated>(p, t0 + i, row, sum[0][i], sum[1][i], sw0, sw1);
}

template <bool kI8, bool kGated>
__global__ void __launch_bounds__(kFfnStreamThreads, 1) weave_ffn_stream_kernel(const __grid_constant__ FfnStreamArgs p)
{
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int stage_bytes = kFfnStreamWeights + p.box_t * 128;
    FfnStreamBars &bars = *reinterpret_cast<FfnStreamBars *>(smem_raw + (smem - smem_u32(smem_raw)) + p.stages * stage_bytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const WaitCtx wc = {p.ctl, p.timeout_ns};
    const int begin = blockIdx.x * p.units_per_cta, end = min(begin + p.units_per_cta, p.units);
    constexpr int kStepK = kI8 ? 128 : 64;
    constexpr int kTileRows = kGated ? 128 : 256;
    const uint32_t tmem_cols = 4u * p.box_t;           // two tiles of two accumulators

    pdl_launch_dependents();
    if (threadIdx.x == 0) {
        for (int i = 0; i < p.stages; ++i) { mbar_init(&bars.full[i], 1); mbar_init(&bars.empty[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&bars.acc_full[i], 1); mbar_init(&bars.acc_empty[i], 8); }
        fence_mbar_init();
        tma_prefetch_desc(&p.w);
        tma_prefetch_desc(&p.x);
    }
    if (warp == 1) { tmem_alloc_one(&bars.tmem_base, tmem_cols); tmem_relinquish_one(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars.tmem_base;

    bool ok = true;
    if (warp == 0) {
        if (lane == 0) {
            const auto load_w = [&](int unit, int s) {
                const int tile = unit / p.ksteps, k = (unit - tile * p.ksteps) * kStepK;
                mbar_arrive_expect_tx(&bars.full[s], (uint32_t)stage_bytes);
                if (kGated) tma_load_3d_one(smem + s * stage_bytes, &p.w, k, tile * kTileRows, 0, &bars.full[s]);
                else tma_load_2d_one(smem + s * stage_bytes, &p.w, k, tile * kTileRows, &bars.full[s]);
            };
            const auto load_x = [&](int unit, int s) {
                tma_load_2d_one(smem + s * stage_bytes + kFfnStreamWeights, &p.x, unit % p.ksteps * kStepK, 0, &bars.full[s]);
            };
            // the weights do not depend on the launch before this one: the ring is filled with them while it ends
            const int ahead = min(p.stages, end - begin);
            for (int i = 0; i < ahead; ++i) load_w(begin + i, i);
            pdl_wait();
            for (int i = 0; i < ahead; ++i) load_x(begin + i, i);
            int s = ahead == p.stages ? 0 : ahead;
            uint32_t ph = 1u;              // the second round of the ring waits for its first release
            for (int unit = begin + ahead; unit < end; ++unit) {
                ok = ffn_wait(&bars.empty[s], ph ^ 1u, wc, 11);
                if (!ok) break;
                load_w(unit, s);
                load_x(unit, s);
                if (++s == p.stages) { s = 0; ph ^= 1u; }
            }
            if (!ok) ffn_linger();
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            const uint32_t idesc = kI8 ? umma_idesc_i8(128, p.box_t) : umma_idesc_bf16(128, p.box_t);
            int s = 0, n = 0;
            uint32_t ph = 0;
            for (int at = begin; at < end && ok; ++n) {
                const FfnSegment g = ffn_segment_at(at, end, p.ksteps);
                at += g.k1 - g.k0;
                const int buf = n & 1;
                ok = ffn_wait(&bars.acc_empty[buf], ((n >> 1) & 1) ^ 1, wc, 12);
                tc_fence_after();
                const uint32_t d = tmem + (uint32_t)(buf * 2 * p.box_t);
                for (int k = g.k0; k < g.k1 && ok; ++k) {
                    ok = ffn_wait(&bars.full[s], ph, wc, 13);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t w = smem + s * stage_bytes;
                    const uint64_t b = umma_desc_sw128(w + kFfnStreamWeights);
                    ffn_mma_kstep_one<kI8>(d, umma_desc_sw128(w), b, idesc, (uint32_t)(k != g.k0));
                    ffn_mma_kstep_one<kI8>(d + p.box_t, umma_desc_sw128(w + 16384), b, idesc, (uint32_t)(k != g.k0));
                    tc_commit_one(&bars.empty[s]);
                    if (++s == p.stages) { s = 0; ph ^= 1u; }
                }
                if (ok) tc_commit_one(&bars.acc_full[buf]);
            }
            if (!ok) ffn_linger();
        }
        __syncwarp();
    } else {
        // ---- epilogue: warps 2-9; the 32 accumulator lanes that a warp can read are those of its number mod 4
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        const int lane_row = quarter * 32 + lane;
        const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
        pdl_wait();                      // the scales of the rows and the workspace come from the launch before
        int n = 0;
        for (int at = begin; at < end; ++n) {
            const FfnSegment g = ffn_segment_at(at, end, p.ksteps);
            const bool whole = g.k1 - g.k0 == p.ksteps;
            const int buf = n & 1;
            const int row = g.tile * kTileRows + lane_row;
            float sw0 = 0.0f, sw1 = 0.0f;
            if constexpr (kI8) {
                if (row < p.N) sw0 = p.col_scale[row];
                const int second = kGated ? p.N + row : row + 128;
                if (kGated ? row < p.N : second < p.N) sw1 = p.col_scale[second];
            }
            ok = __all_sync(0xffffffffu, ffn_wait(&bars.acc_full[buf], (n >> 1) & 1, wc, 14));
            // the epilogue warps meet at barriers below: they leave together
            ok = named_barrier_and<2, 256>(ok);
            if (!ok) break;
            tc_fence_after();
            uint32_t *mine = p.partials + (size_t)(2 * blockIdx.x + (at == begin ? 0 : 1)) * 256 * p.T + lane_row;
            for (int t0 = half * 8; t0 < p.T; t0 += 16) {
                uint32_t a[8], b[8];
                const uint32_t src = lane_base + (uint32_t)(buf * 2 * p.box_t + t0);
                tmem_ld_32x8(src, a);
                tmem_ld_32x8(src + p.box_t, b);
                tmem_ld_wait8x2(a, b);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (t0 + i >= p.T) break;
                    if (whole) {
                        ffn_stream_store<kI8, kGated>(p, t0 + i, row, a[i], b[i], sw0, sw1);
                    } else {
                        __stcg(mine + (size_t)(t0 + i) * 128, a[i]);
                        __stcg(mine + (size_t)(p.T + t0 + i) * 128, b[i]);
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.acc_empty[buf]);
            at += g.k1 - g.k0;
            if (whole) continue;
            // CTAs whose ranges touch this tile
            const int first = g.tile * p.ksteps, c0 = first / p.units_per_cta, c1 = (first + p.ksteps - 1) / p.units_per_cta;
            __threadfence();
            named_barrier_sync<1, 256>();
            if (threadIdx.x == 64) {
                const unsigned before = atom_acqrel_add_u32(p.arrived + g.tile, 1u);
                const bool last = before == (unsigned)(c1 - c0);
                if (last) p.arrived[g.tile] = 0u;
                bars.last = last;
            }
            named_barrier_sync<1, 256>();
            if (bars.last) {
                __threadfence();
                if (p.T <= 2) {
                    if (half < p.T) ffn_stream_join<kI8, kGated, 1, 16>(p, g.tile, c0, c1, half, lane_row, row, sw0, sw1);
                } else {
                    for (int t0 = half * 8; t0 < p.T; t0 += 16)
                        ffn_stream_join<kI8, kGated, 8, 2>(p, g.tile, c0, c1, t0, lane_row, row, sw0, sw1);
                }
            }
            // nobody overwrites bars.last before all have read it: the next arrival is behind the next barrier
        }
        if (!ok) ffn_linger();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc_one(tmem, tmem_cols);
}

}  // namespace weave
