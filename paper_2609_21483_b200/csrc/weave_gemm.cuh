// Dense matrix products for the feed-forward block: one persistent kernel on pairs of neighbouring SMs
// (tcgen05.mma.cta_group::2, operands by TMA, accumulators in tensor memory), in the forms that the block and its
// gradient need:
//
//   epilogue        D (columns of one tile)                                              operands
//   kEpiStore       D = A B, rounded to bf16 (256)                                       either may be MN-major
//   kEpiGated       h = silu(g) u, g = A Bg, u = A Bu, rounded to bf16 (128)             K-major
//   kEpiGrad        dh = A0 B0 and g, u as above -> h, dg, du, rounded to bf16 (128)     B0 MN-major
//   kEpiScaled      D = (A B) * (row scale * column scale) in bf16 or fp32 (256)         8-bit integers, K-major
//   kEpiScaledGated h as above from scaled g and u (128)                                 8-bit integers, K-major
//
// A tile is 256 rows of A (128 per CTA) by up to 256 accumulator columns (fewer where that fills the last wave).  A k-step
// is 128 bytes of K (64 bf16 or 128 8-bit integers): 16 KB of A and up to 16 KB of B per CTA, 192 KB of them in flight.  Rows, columns and K that stick out over
// the matrices are zero-filled by the tensor maps on the way in and clipped by them on the way out.
//
// Bound: the tensor pipe (256 x 256 x 16 takes 128 cycles) and, over more than some milliseconds, the power limit.
#pragma once
#include <cuda.h>
#include "weave_ptx.cuh"

namespace weave {

enum { kEpiStore = 0, kEpiGated = 1, kEpiGrad = 2, kEpiScaled = 3, kEpiScaledGated = 4 };

// first words of a handle's workspace
struct FfnCtl {
    int status;          // 0 or the error that the first failed wait recorded
    int where;           // which wait that was
    unsigned pad[30];
    unsigned long long barrier[16];      // grid barriers of the small batches' kernel: arrivals since creation
};
static_assert(sizeof(FfnCtl) == 256, "the workspace layout counts on it");

constexpr int kFfnErrTimeout = -6;      // WEAVE_ERR_TIMEOUT

// ------------------------------------------------------------------------------------ waits
// As in the MoE kernels every wait is bounded: it polls the status word (another wait may have given up) and a
// wall-clock limit, and returns false instead of spinning forever.

struct WaitCtx {
    FfnCtl *ctl;
    unsigned long long timeout_ns;
};

__device__ __noinline__ bool mbar_wait_slow(uint64_t *bar, uint32_t parity, FfnCtl *ctl, unsigned long long timeout_ns, int where)
{
    unsigned long long t0 = 0;
    unsigned it = 0;
    while (!mbar_try_wait_cluster(bar, parity)) {
        if ((++it & 31u) == 0u) {
            if (*reinterpret_cast<volatile int *>(&ctl->status) != 0) return false;
            const unsigned long long now = globaltimer_ns();
            if (t0 == 0) t0 = now;
            else if ((long long)(now - t0) > (long long)timeout_ns) {
                if (atomicCAS(&ctl->status, 0, kFfnErrTimeout) == 0) ctl->where = where;
                return false;
            }
        }
    }
    return true;
}
__device__ __forceinline__ bool ffn_wait(uint64_t *bar, uint32_t parity, const WaitCtx &w, int where)
{
    if (mbar_try_wait(bar, parity)) return true;
    return mbar_wait_slow(bar, parity, w.ctl, w.timeout_ns, where);
}
// lets copies and products that are in flight land before this CTA can leave
__device__ __forceinline__ void ffn_linger()
{
    const unsigned long long t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 50000ull) __nanosleep(1000);
}

// ------------------------------------------------------------------------------------ PTX forms the MoE kernels lack

// Launches behind one another: a kernel that was launched as the programmatic dependent of the one before it in the
// stream starts when all CTAs of that one have called the first function, and sees what it wrote behind the second.
// Every kernel of a chain calls the second one, so that its end means the end of all before it.
__device__ __forceinline__ void pdl_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// MN-major operand, 128-byte swizzle: boxes of 64 elements along MN by 64 of K.  Eight K rows (1024 bytes) are one
// swizzle atom: stride byte offset = the next eight of K; leading byte offset = the next 64 along MN (the next box).
__device__ __forceinline__ uint64_t umma_desc_mn_sw128(uint32_t smem_addr)
{
    return (uint64_t)((smem_addr >> 4) & 0x3FFFu) | (512ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// kind::i8: D int32 (2 at bit 4), A and B signed (1 at bits 7 and 10)
__device__ __forceinline__ uint32_t umma_idesc_i8(uint32_t M, uint32_t N)
{
    return (2u << 4) | (1u << 7) | (1u << 10) | ((N >> 3) << 17) | ((M >> 4) << 24);
}
constexpr uint32_t kIdescAMn = 1u << 15, kIdescBMn = 1u << 16;

// One k-step of a pair tile: four products over 128 bytes of K each operand's descriptor of which moves on by its own
// increment (16-byte units), then the commit that frees the stage in both CTAs.  Called by the whole converged warp.
template <bool kI8>
__device__ __forceinline__ void ffn_mma_kstep_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint64_t a_inc, uint64_t b_inc,
                                                   uint32_t idesc, uint32_t accumulate_first, uint64_t *empty_bar)
{
#define WEAVE_KSTEP_PAIR(KIND)                                                                                        \
    asm volatile(                                                                                                     \
        "{\n\t.reg .pred pe, pa, pt;\n\t"                                                                             \
        ".reg .b64 a1, a2, a3, b1, b2, b3;\n\t"                                                                       \
        "elect.sync _|pe, 0xffffffff;\n\t"                                                                            \
        "setp.ne.b32 pa, %6, 0;\n\t"                                                                                  \
        "setp.eq.u32 pt, %0, %0;\n\t"                                                                                 \
        "add.u64 a1, %1, %3;\n\tadd.u64 a2, a1, %3;\n\tadd.u64 a3, a2, %3;\n\t"                                       \
        "add.u64 b1, %2, %4;\n\tadd.u64 b2, b1, %4;\n\tadd.u64 b3, b2, %4;\n\t"                                       \
        "@pe tcgen05.mma.cta_group::2.kind::" KIND " [%0], %1, %2, %5, pa;\n\t"                                       \
        "@pe tcgen05.mma.cta_group::2.kind::" KIND " [%0], a1, b1, %5, pt;\n\t"                                       \
        "@pe tcgen05.mma.cta_group::2.kind::" KIND " [%0], a2, b2, %5, pt;\n\t"                                       \
        "@pe tcgen05.mma.cta_group::2.kind::" KIND " [%0], a3, b3, %5, pt;\n\t"                                       \
        "@pe tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%7], %8;\n\t}" \
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "l"(a_inc), "l"(b_inc), "r"(idesc), "r"(accumulate_first),           \
          "r"(smem_u32(empty_bar)), "h"((uint16_t)3)                                                                  \
        : "memory")
    if (kI8) WEAVE_KSTEP_PAIR("i8");
    else WEAVE_KSTEP_PAIR("f16");
#undef WEAVE_KSTEP_PAIR
}

// shared -> global through a tensor map (clips what sticks out), tracked by the thread's bulk async-groups
__device__ __forceinline__ void tma_store_2d(const void *map, uint32_t smem_src, int x, int row)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(smem_src), "r"(x),
                 "r"(row)
                 : "memory");
}

// ------------------------------------------------------------------------------------ the activation

// s = sigmoid(g).  exp overflows to inf for g below -88, where s is 0 either way; NaN and +inf come through.
// __expf and the approximate division are off by 2^-21 and 2^-22 relative near 0 and by 2^-17 where |g| nears 88:
// nothing next to the rounding to bf16 behind them.
__device__ __forceinline__ float fast_sigmoid(float g) { return __fdividef(1.0f, 1.0f + __expf(-g)); }
__device__ __forceinline__ float gated(float g, float u) { return g * fast_sigmoid(g) * u; }

// ------------------------------------------------------------------------------------ the kernel

// One product.  kEpiGrad has two over the same tiles, job 0 for dh and job 1 for g and u; kEpiStore up to three
// independent ones in one launch; the other forms have one.
struct alignas(64) GemmJob {
    CUtensorMap a;
    CUtensorMap b[2];        // [rank of the CTA in its pair]: the gated forms give gate rows to one, up rows to the other
    CUtensorMap d;           // results; kEpiGrad: h, dg, du in jobs 0, 1, 2
    CUtensorMap d8;          // results in bf16, eight columns at a time: what a width leaves over 64
    int M, N;                // rows and columns of the result
    int ksteps;
    int a_mn, b_mn;          // kEpiStore: operand is MN-major
    int width;               // columns of the result in a tile: a multiple of 16 up to 256, gated of 8 up to 128; of 32 where
                             // the result is in fp32, of 64 where B is MN-major (kEpiGrad, too): with 16 of them in a CTA
                             // the products came out wrong, with 32 right
    int tiles_m, tiles_n, group_m;
};

struct alignas(64) GemmArgs {
    GemmJob job[3];
    FfnCtl *ctl;
    unsigned long long timeout_ns;
    const float *row_scale;  // scaled forms: [M] and [N] (gated: [2N], gate then up)
    const float *col_scale;
    void *out;               // kEpiScaled, for rows that no tensor map can describe
    long long ld_out;
    int out_f32, direct;     // kEpiScaled: type of the result; 1 = ordinary stores (row length not a multiple of 16 bytes)
    int extra;               // kEpiStore: see gemm_tile()
    int stages, stage_bytes;
};

constexpr int kGemmThreads = 256;
constexpr int kGemmMaxStages = 9;
constexpr int kGemmHalf = 16384;                    // A's bytes of one k-step in one CTA, B's at most
constexpr int kGemmRing = 6 * 2 * kGemmHalf;
constexpr int kGemmStaging = 8192;                  // per epilogue warp
constexpr int kGemmSmemStaging = kGemmRing;
constexpr int kGemmSmemScales = kGemmSmemStaging + 4 * kGemmStaging;
constexpr int kGemmSmemBars = kGemmSmemScales + 4 * 256;
constexpr int kGemmSmemBytes = kGemmSmemBars + 256 + 1024;      // 1024: the stages start on a swizzle atom's boundary
static_assert(kGemmSmemBytes <= 232448, "227 KB per CTA");

struct GemmBars {
    uint64_t full[kGemmMaxStages], empty[kGemmMaxStages];
    uint64_t acc_full[2], acc_empty[2];
    uint32_t tmem_base;
};
static_assert(sizeof(GemmBars) <= 256, "the barriers' place in shared memory");

struct GemmTile { int job, m0, n0; };

// Tiles of a job in groups of group_m row tiles, all columns of a group before the next group, row tiles fastest: the
// pairs at work at one time share a few panels of B and the group's rows of A in L2.
__device__ __forceinline__ void gemm_tile_at(const GemmJob &p, int t, GemmTile &at)
{
    const int per = p.group_m * p.tiles_n;
    const int g = t / per, r = t - g * per;
    const int gm = min(p.group_m, p.tiles_m - g * p.group_m);
    const int n = r / gm;
    at.m0 = (g * p.group_m + r - n * gm) * 256;
    at.n0 = n * p.width;
}

// The i-th tile of a CTA pair; false behind its last.  Job 0's tiles go round the pairs; the pairs that get one less of
// them take `extra` tiles of jobs 1 and 2 for it (as many as cost the same), whose remaining ones go round all pairs.
template <bool kJobs>
__device__ __forceinline__ bool gemm_tile(const GemmArgs &p, int i, int pair, int pairs, GemmTile &at)
{
    const int n0 = p.job[0].tiles_m * p.job[0].tiles_n;
    int t = pair + i * pairs;
    at.job = 0;
    if constexpr (kJobs) {
        if (t >= n0) {
            const int n1 = p.job[1].tiles_m * p.job[1].tiles_n, n2 = p.job[2].tiles_m * p.job[2].tiles_n;
            const int rest = n0 % pairs, few = rest ? pairs - rest : 0;
            const int j = i - (n0 > pair ? (n0 - pair + pairs - 1) / pairs : 0);
            if (few == 0 || pair < rest) t = few * p.extra + j * pairs + pair;
            else if (j < p.extra) t = j * few + pair - rest;
            else t = few * p.extra + (j - p.extra) * pairs + pair;
            if (t >= n1 + n2) return false;
            at.job = t < n1 ? 1 : 2;
            if (t >= n1) t -= n1;
            gemm_tile_at(p.job[at.job], t, at);
            return true;
        }
    }
    if (t >= n0) return false;
    gemm_tile_at(p.job[0], t, at);
    return true;
}

// A warp's 32 rows x 64 columns in bf16 on their way out: 128-byte rows, swizzled, for one tensor copy; of a narrower rest
// of a tile eight columns lie together, for copies of their own.
__device__ __forceinline__ uint32_t gemm_staged(uint32_t dst, int lane, int j, int there)
{
    return there == 64 ? dst + lane * 128 + ((j ^ (lane & 7)) << 4) : dst + j * 512 + lane * 16;
}
__device__ __forceinline__ void gemm_store_bf16(const GemmJob &job, uint32_t src, int lane, int col, int row0, int there, bool any_row)
{
    fence_proxy_async_shared();
    __syncwarp();
    if (lane == 0) {
        if (any_row) {
            if (there == 64) {
                if (col < job.N) tma_store_2d(&job.d, src, col, row0);
            } else {
                for (int j = 0; j * 8 < there && col + j * 8 < job.N; ++j) tma_store_2d(&job.d8, src + j * 512, col + j * 8, row0);
            }
        }
        bulk_commit();
    }
}

template <int kEpi, bool kI8>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kGemmThreads, 1) weave_gemm_kernel(const __grid_constant__ GemmArgs p)
{
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *const smem_g = smem_raw + (smem - smem_u32(smem_raw));
    GemmBars &bars = *reinterpret_cast<GemmBars *>(smem_g + kGemmSmemBars);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const WaitCtx wc = {p.ctl, p.timeout_ns};
    constexpr bool kGatedTile = kEpi == kEpiGated || kEpi == kEpiGrad || kEpi == kEpiScaledGated;
    constexpr bool kJobs = kEpi == kEpiStore;
    constexpr int kPhases = kEpi == kEpiGrad ? 2 : 1;
    constexpr int kStepK = kI8 ? 128 : 64;          // elements of K in a k-step
    GemmTile at;

    pdl_launch_dependents();
    if (threadIdx.x == 0) {
        for (int i = 0; i < kGemmMaxStages; ++i) { mbar_init(&bars.full[i], 1); mbar_init(&bars.empty[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&bars.acc_full[i], 1); mbar_init(&bars.acc_empty[i], 8); }
        fence_mbar_init();
    }
    if (warp == 3) { tmem_alloc_pair(&bars.tmem_base, 512); tmem_relinquish_pair(); }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = bars.tmem_base;

    bool ok = true;
    if (warp < 2) {
        // ---- producers: warp 0 brings this CTA's rows of A, warp 1 its part of B; all bytes of a stage are credited
        // to the full barrier in the pair's leader
        const bool load_a = warp == 0;
        pdl_wait();
        int s = 0;
        uint32_t ph = 0;
        for (int i = 0; ok && gemm_tile<kJobs>(p, i, pair, pairs, at); ++i) {
            for (int phase = 0; phase < kPhases && ok; ++phase) {
                const GemmJob &job = p.job[kPhases == 2 ? phase : at.job];
                const bool dh = kPhases == 2 && phase == 0;
                const bool a_mn = kJobs && job.a_mn, b_mn = kJobs ? job.b_mn != 0 : dh;
                const int half = kGatedTile && !dh ? job.width : job.width / 2;          // this CTA's rows of B
                const int b_boxes = b_mn ? (half + 63) / 64 : 1;
                const uint32_t tx = 2u * (kGemmHalf + (b_mn ? (uint32_t)b_boxes * 8192u : (uint32_t)half * 128u));
                const void *map = load_a ? &job.a : &job.b[rank];
                const int mn = load_a ? at.m0 + (int)rank * 128 : at.n0 + (kGatedTile && !dh ? 0 : (int)rank * half);
                const bool mn_major = load_a ? a_mn : b_mn;
                const bool second = load_a ? a_mn : b_boxes == 2;
                const int ks = job.ksteps;
                for (int k = 0; k < ks; ++k) {
                    ok = __all_sync(0xffffffffu, ffn_wait(&bars.empty[s], ph ^ 1u, wc, 1 + warp));
                    if (!ok) break;
                    const uint32_t dst = smem + s * p.stage_bytes + (load_a ? 0 : kGemmHalf);
                    const uint32_t full = mapa_u32(smem_u32(&bars.full[s]), 0);
                    if (elect_one()) {
                        if (load_a && rank == 0) mbar_arrive_expect_tx(&bars.full[s], tx);
                        tma_load_2d_pair(dst, map, mn_major ? mn : k * kStepK, mn_major ? k * kStepK : mn, full);
                        if (second) tma_load_2d_pair(dst + 8192, map, mn + 64, k * kStepK, full);
                    }
                    __syncwarp();
                    if (++s == p.stages) { s = 0; ph ^= 1u; }
                }
            }
        }
        if (!ok) ffn_linger();
    } else if (warp == 2) {
        if (rank == 0) {
            // ---- the pair's issuer
            int s = 0;
            uint32_t ph = 0;
            for (int n = 0; ok && gemm_tile<kJobs>(p, n, pair, pairs, at); ++n) {
                // kEpiGrad: g and u in columns 0-255, dh in 256-383 or 384-511: the next tile's dh is summed up
                // while the epilogue still reads this one's
                const int buf = n & 1;
                if (kEpi != kEpiGrad) ok = __all_sync(0xffffffffu, ffn_wait(&bars.acc_empty[buf], ((n >> 1) & 1) ^ 1, wc, 3));
                for (int phase = 0; phase < kPhases && ok; ++phase) {
                    const GemmJob &job = p.job[kPhases == 2 ? phase : at.job];
                    const bool dh = kPhases == 2 && phase == 0;
                    if (kPhases == 2 && phase == 1) {
                        ok = __all_sync(0xffffffffu, ffn_wait(&bars.acc_empty[0], (n & 1) ^ 1, wc, 3));
                        if (!ok) break;
                    }
                    tc_fence_after();
                    const bool a_mn = kJobs && job.a_mn, b_mn = kJobs ? job.b_mn != 0 : dh;
                    const uint32_t d = tmem + (kEpi != kEpiGrad ? buf * 256 : dh ? 256 + buf * 128 : 0);
                    const uint32_t n_mma = (uint32_t)(kGatedTile && !dh ? 2 * job.width : job.width);
                    const uint32_t idesc = (kI8 ? umma_idesc_i8(256, n_mma) : umma_idesc_bf16(256, n_mma)) | (a_mn ? kIdescAMn : 0u) |
                                           (b_mn ? kIdescBMn : 0u);
                    const uint64_t a_inc = a_mn ? 128 : 2, b_inc = b_mn ? 128 : 2;
                    const int ks = job.ksteps;
                    for (int k = 0; k < ks; ++k) {
                        ok = __all_sync(0xffffffffu, ffn_wait(&bars.full[s], ph, wc, 4));
                        if (!ok) break;
                        tc_fence_after();
                        const uint32_t a = smem + s * p.stage_bytes, b = a + kGemmHalf;
                        ffn_mma_kstep_pair<kI8>(d, a_mn ? umma_desc_mn_sw128(a) : umma_desc_sw128(a),
                                                b_mn ? umma_desc_mn_sw128(b) : umma_desc_sw128(b), a_inc, b_inc, idesc, (uint32_t)(k != 0),
                                                &bars.empty[s]);
                        if (++s == p.stages) { s = 0; ph ^= 1u; }
                    }
                }
                if (ok && elect_one()) tc_commit_pair(&bars.acc_full[buf], 3);
                __syncwarp();
            }
            if (!ok) ffn_linger();
        }
    } else if (warp >= 4) {
        // ---- epilogue: each warp the 32 accumulator lanes of its quarter; rows m0 + 128 rank + 32 quarter + lane
        const int quarter = warp - 4;
        const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
        const uint32_t stage = smem + kGemmSmemStaging + quarter * kGemmStaging;
        float *const scales = reinterpret_cast<float *>(smem_g + kGemmSmemScales + quarter * 256);
        const uint32_t empty0 = mapa_u32(smem_u32(&bars.acc_empty[0]), 0);
        pdl_wait();
        uint32_t slot = 0;          // half of the staging buffer that is written next (not kEpiGrad)
        for (int n = 0; gemm_tile<kJobs>(p, n, pair, pairs, at); ++n) {
            const GemmJob &job = p.job[at.job];
            const int M = job.M, N = job.N, width = job.width, n0 = at.n0;
            const int row0 = at.m0 + (int)rank * 128 + quarter * 32;
            const int buf = n & 1;
            ok = __all_sync(0xffffffffu, ffn_wait(&bars.acc_full[buf], (n >> 1) & 1, wc, 5));
            if (!ok) break;
            tc_fence_after();
            const bool any_row = row0 < M;       // whole warp
            float sx = 0.0f;
            if constexpr (kI8) sx = row0 + lane < M ? p.row_scale[row0 + lane] : 0.0f;

            if constexpr (kEpi == kEpiStore || kEpi == kEpiScaled) {
#pragma unroll 1
                for (int c = 0; c * 64 < width; ++c) {
                    const int col = n0 + c * 64, there = min(64, width - c * 64);
                    uint32_t v[64];
                    tmem_ld_32x64(lane_base + buf * 256 + c * 64, v);
                    tmem_ld_wait64(v);
                    if (!any_row || col >= N) continue;
                    if constexpr (kEpi == kEpiScaled) {
                        __syncwarp();
                        scales[lane] = col + lane < N ? p.col_scale[col + lane] : 0.0f;
                        scales[lane + 32] = col + 32 + lane < N ? p.col_scale[col + 32 + lane] : 0.0f;
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 64; i += 4) {
                            const float4 w = *reinterpret_cast<const float4 *>(scales + i);
                            v[i] = __float_as_uint(__int2float_rn((int)v[i]) * (sx * w.x));
                            v[i + 1] = __float_as_uint(__int2float_rn((int)v[i + 1]) * (sx * w.y));
                            v[i + 2] = __float_as_uint(__int2float_rn((int)v[i + 2]) * (sx * w.z));
                            v[i + 3] = __float_as_uint(__int2float_rn((int)v[i + 3]) * (sx * w.w));
                        }
                    }
                    const bool f32 = kEpi == kEpiScaled && p.out_f32;
                    if (kEpi == kEpiScaled && p.direct) {
                        // row by row through shared memory, so that a warp's stores lie side by side
                        float *const out_f = static_cast<float *>(p.out);
                        __nv_bfloat16 *const out_b = static_cast<__nv_bfloat16 *>(p.out);
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            __syncwarp();
#pragma unroll
                            for (int i = 0; i < 32; ++i) st_shared_u32(stage + lane * 132 + i * 4, v[half * 32 + i]);
                            __syncwarp();
                            const int cc = half * 32 + lane < there ? col + half * 32 + lane : N;
                            const int rows = min(32, M - row0);
                            if (cc < N)
#pragma unroll 8
                                for (int r = 0; r < rows; ++r) {
                                    const float y = ld_shared_f32(stage + r * 132 + lane * 4);
                                    const long long at = (long long)(row0 + r) * p.ld_out + cc;
                                    if (f32) out_f[at] = y;
                                    else out_b[at] = __float2bfloat16_rn(y);
                                }
                        }
                        continue;
                    }
                    if (f32) {
                        // two tiles of 32 rows x 32 columns, one in each half of the staging buffer
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            if (lane == 0) bulk_wait_read<1>();
                            __syncwarp();
                            const uint32_t dst = stage + half * 4096;
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                st_shared_v4(dst + lane * 128 + ((j ^ (lane & 7)) << 4),
                                             make_uint4(v[half * 32 + j * 4], v[half * 32 + j * 4 + 1], v[half * 32 + j * 4 + 2],
                                                        v[half * 32 + j * 4 + 3]));
                            fence_proxy_async_shared();
                            __syncwarp();
                            if (lane == 0 && half * 32 < there && col + half * 32 < N) tma_store_2d(&job.d, dst, col + half * 32, row0);
                            if (lane == 0) bulk_commit();
                        }
                    } else {
                        if (lane == 0) bulk_wait_read<1>();
                        __syncwarp();
                        const uint32_t dst = stage + slot * 4096;
                        slot ^= 1u;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            uint32_t w[4];
#pragma unroll
                            for (int q = 0; q < 4; ++q)
                                w[q] = pack_bf16x2(__uint_as_float(v[j * 8 + q * 2]), __uint_as_float(v[j * 8 + q * 2 + 1]));
                            st_shared_v4(gemm_staged(dst, lane, j, there), make_uint4(w[0], w[1], w[2], w[3]));
                        }
                        gemm_store_bf16(job, dst, lane, col, row0, there, true);
                    }
                }
            } else if constexpr (kEpi == kEpiGated || kEpi == kEpiScaledGated) {
#pragma unroll 1
                for (int c = 0; c * 64 < width; ++c) {
                    const int there = min(64, width - c * 64);
                    const uint32_t dst = stage + slot * 4096;
                    slot ^= 1u;
                    if (lane == 0) bulk_wait_read<1>();
                    __syncwarp();
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int cc = c * 64 + half * 32;
                        uint32_t g[32], u[32];
                        tmem_ld_32x32(lane_base + buf * 256 + cc, g);
                        tmem_ld_32x32(lane_base + buf * 256 + width + cc, u);
                        tmem_ld_wait32(g);
                        reg_fence32(u);
                        if constexpr (kEpi == kEpiScaledGated) {
                            const int col = n0 + cc + lane;
                            __syncwarp();
                            scales[lane] = col < N ? p.col_scale[col] : 0.0f;
                            scales[lane + 32] = col < N ? p.col_scale[N + col] : 0.0f;
                            __syncwarp();
#pragma unroll
                            for (int i = 0; i < 32; i += 4) {
                                const float4 wg = *reinterpret_cast<const float4 *>(scales + i);
                                const float4 wu = *reinterpret_cast<const float4 *>(scales + 32 + i);
                                const float fg[4] = {wg.x, wg.y, wg.z, wg.w}, fu[4] = {wu.x, wu.y, wu.z, wu.w};
#pragma unroll
                                for (int q = 0; q < 4; ++q) {
                                    g[i + q] = __float_as_uint(__int2float_rn((int)g[i + q]) * (sx * fg[q]));
                                    u[i + q] = __float_as_uint(__int2float_rn((int)u[i + q]) * (sx * fu[q]));
                                }
                            }
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            uint32_t w[4];
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                const int i = j * 8 + q * 2;
                                w[q] = pack_bf16x2(gated(__uint_as_float(g[i]), __uint_as_float(u[i])),
                                                   gated(__uint_as_float(g[i + 1]), __uint_as_float(u[i + 1])));
                            }
                            st_shared_v4(gemm_staged(dst, lane, half * 4 + j, there), make_uint4(w[0], w[1], w[2], w[3]));
                        }
                    }
                    gemm_store_bf16(job, dst, lane, n0 + c * 64, row0, there, any_row);
                }
            } else {
                // kEpiGrad: 32 columns at a time, three results of 32 x 32 bf16 (64-byte swizzle) in rotating quarters
                // of the staging buffer
                int quad = 0;
#pragma unroll 1
                for (int c = 0; c < width / 32; ++c) {
                    uint32_t g[32], u[32], d[32];
                    tmem_ld_32x32(lane_base + c * 32, g);
                    tmem_ld_32x32(lane_base + width + c * 32, u);
                    tmem_ld_32x32(lane_base + 256 + buf * 128 + c * 32, d);
                    tmem_ld_wait32(g);
                    reg_fence32(u);
                    reg_fence32(d);
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const float fg = __uint_as_float(g[i]), fu = __uint_as_float(u[i]), fd = __uint_as_float(d[i]);
                        const float sg = fast_sigmoid(fg);
                        const float si = fg * sg;
                        g[i] = __float_as_uint(si * fu);                                    // h
                        u[i] = __float_as_uint(fd * fu * sg * (1.0f + fg * (1.0f - sg)));   // dg
                        d[i] = __float_as_uint(fd * si);                                    // du
                    }
#pragma unroll
                    for (int which = 0; which < 3; ++which) {
                        const uint32_t *v = which == 0 ? g : which == 1 ? u : d;
                        const uint32_t dst = stage + quad * 2048;
                        quad = (quad + 1) & 3;
                        if (lane == 0) bulk_wait_read<3>();
                        __syncwarp();
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            uint32_t w[4];
#pragma unroll
                            for (int q = 0; q < 4; ++q)
                                w[q] = pack_bf16x2(__uint_as_float(v[j * 8 + q * 2]), __uint_as_float(v[j * 8 + q * 2 + 1]));
                            st_shared_v4(dst + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4), make_uint4(w[0], w[1], w[2], w[3]));
                        }
                        fence_proxy_async_shared();
                        __syncwarp();
                        if (lane == 0) {
                            if (any_row && n0 + c * 32 < N) tma_store_2d(&p.job[which].d, dst, n0 + c * 32, row0);
                            bulk_commit();
                        }
                    }
                }
            }
            // accumulator read: hand it back to the pair's issuer
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_remote(kEpi == kEpiGrad ? empty0 : empty0 + buf * 8);
        }
        if (lane == 0) bulk_wait<0>();
        if (!ok) ffn_linger();
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    if (warp == 3) tmem_dealloc_pair(tmem, 512);
}

}  // namespace weave
