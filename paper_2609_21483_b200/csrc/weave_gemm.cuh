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
// is 128 bytes of K (64 bf16 or 128 8-bit integers): up to 16 KB of A and of B per CTA, 192 KB of them in flight.  Rows,
// columns and K that stick out over the matrices are zero-filled by the tensor maps on the way in and clipped on the way out.
//
// Where tiles are few and K is long, K is cut into parts for different pairs (kSplit): each part's sums go to the workspace,
// and the last to arrive at a tile, which waits for nobody, adds them up in the order of K: the same bits every time.
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
    unsigned arrived[192];               // products whose K is split: arrivals per tile and CTA of a pair, zero between launches
};
static_assert(sizeof(FfnCtl) == 1024, "the workspace layout counts on it");
constexpr int kGemmSplitUnits = 74;      // tiles times parts of K, at most, and
constexpr int kGemmSplitWidth = 128;     // columns of such a tile
constexpr size_t kGemmSplitBytes = (size_t)kGemmSplitUnits * 2 * kGemmSplitWidth * 128 * 4;

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
// The same for boxes of 32 elements along MN, 64-byte swizzle: eight K rows are an atom of 512 bytes.  For operands of which a CTA has
// only 32 along MN: half an atom of 64 is no layout that the instruction is defined for.
__device__ __forceinline__ uint64_t umma_desc_mn_sw64(uint32_t smem_addr)
{
    return (uint64_t)((smem_addr >> 4) & 0x3FFFu) | (256ull << 16) | (32ull << 32) | (1ull << 46) | (4ull << 61);
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

// a barrier of some of the CTA's warps that also says whether all of their threads brought `true`
__device__ __forceinline__ bool barrier_and_64(int id, bool mine)
{
    uint32_t all;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "bar.red.and.pred q, %2, 64, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(all)
        : "r"((uint32_t)mine), "r"(id)
        : "memory");
    return all != 0;
}
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

// ------------------------------------------------------------------------------------ the activation

// s = sigmoid(g) = (g < 0 ? e : 1) / (1 + e) with e = exp(-|g|): the divisor lies between 1 and 2, whatever g is, and s is a number
// as small as fp32 has them (in 1 / (1 + exp(-g)) exp overflows from -88.7 on, and __fdividef() gives 0 for divisors above 2^126,
// from -87.3 on: a large u makes these count).  NaN comes through.  __expf is off by 2^-21 relative near 0 and by 2^-17 where |g|
// nears 88, the reciprocal by 2^-23: nothing next to the rounding to bf16 behind them.
__device__ __forceinline__ float fast_sigmoid(float g)
{
    const float e = __expf(-fabsf(g));
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
    return (g < 0.0f ? e : 1.0f) * r;
}
// Where h, dg or du are an operand of the next product they are rounded to bf16, the type of the other operand: 0.0024 of a result's
// size in the root of the mean square instead of the 0.0017 that its own rounding makes.
__device__ __forceinline__ float gated(float g, float u) { return g * fast_sigmoid(g) * u; }

// ------------------------------------------------------------------------------------ the kernel

// One product.  kEpiGrad has two over the same tiles, job 0 for dh and job 1 for g and u; kEpiStore up to three
// independent ones in one launch; the other forms have one.
struct alignas(64) GemmJob {
    CUtensorMap a;
    CUtensorMap b[2];        // [rank of the CTA in its pair]: the gated forms give gate rows to one, up rows to the other
    void *out;               // result, rows `ld` elements apart; kEpiGrad: h, dg, du in jobs 0, 1, 2
    long long ld;
    int M, N;                // rows and columns of the result
    int ksteps;
    int a_mn, b_mn;          // kEpiStore: operand is MN-major
    int rows;                // rows of A that a CTA takes of a tile, a multiple of 8 up to 128: a tile is 2 x rows high
    int width;               // columns of the result in a tile, up to 256 (gated 128): a product's N, twice that in the gated
                             // forms, is a multiple of 16 in bf16 and of 32 in 8-bit integers.  Where B is MN-major a CTA's half
                             // of them is whole swizzle atoms: 64 or 128 in 128-byte swizzle, 32 (kEpiGrad) in 64-byte swizzle
    int tiles_m, tiles_n, group_m;
    int splits;              // parts of K that are worked on by different pairs (kEpiStore's job 0, not in kEpiGrad): fp32 or
                             // int32 sums in `partials`, added up in the order of K by whoever arrives last
};

struct alignas(64) GemmArgs {
    GemmJob job[3];
    FfnCtl *ctl;
    uint32_t *partials;      // [tile][part][CTA of the pair][column][128]
    unsigned long long timeout_ns;
    const float *row_scale;  // scaled forms: [M] and [N] (gated: [2N], gate then up)
    const float *col_scale;
    int out_f32, direct;     // kEpiScaled: type of the result; 1 = row length not a multiple of 16 bytes
    int extra;               // kEpiStore: see gemm_tile()
    int stages, a_bytes, stage_bytes;
    unsigned withhold;       // test hook: the first CTA of a pair whose stages wait for bytes that nobody sends (none: all ones)
};

constexpr int kGemmThreads = 384;                   // two producers, the issuer, one idle warp, eight epilogue warps
constexpr int kGemmMaxStages = 12;
constexpr int kGemmHalf = 16384;                    // A's or B's bytes of one k-step in one CTA, at most
constexpr int kGemmRing = 6 * 2 * kGemmHalf;
constexpr int kGemmStaging = 4096;                  // per epilogue warp
constexpr int kGemmSmemStaging = kGemmRing;
constexpr int kGemmSmemBars = kGemmSmemStaging + 8 * kGemmStaging;
constexpr int kGemmSmemBytes = kGemmSmemBars + 256 + 1024;      // 1024: the stages start on a swizzle atom's boundary
static_assert(kGemmSmemBytes <= 232448, "227 KB per CTA");

struct GemmBars {
    uint64_t full[kGemmMaxStages], empty[kGemmMaxStages];
    uint64_t acc_full[2], acc_empty[2];
    uint32_t tmem_base, last;
};
static_assert(sizeof(GemmBars) <= 256, "the barriers' place in shared memory");

struct GemmTile { int job, m0, n0, index, part; };

// Tiles of a job in groups of group_m row tiles, all columns of a group before the next group, row tiles fastest: the
// pairs at work at one time share a few panels of B and the group's rows of A in L2.
template <bool kSplit>
__device__ __forceinline__ void gemm_tile_at(const GemmJob &p, int t, GemmTile &at)
{
    if constexpr (kSplit) {
        at.part = t % p.splits;
        t /= p.splits;
        at.index = t;
    }
    const int per = p.group_m * p.tiles_n;
    const int g = t / per, r = t - g * per;
    const int gm = min(p.group_m, p.tiles_m - g * p.group_m);
    const int n = r / gm;
    at.m0 = (g * p.group_m + r - n * gm) * 2 * p.rows;
    at.n0 = n * p.width;
}

// first k-step of a tile's part of K, and the one behind its last
template <bool kSplit>
__device__ __forceinline__ int gemm_first(const GemmJob &p, const GemmTile &at) { return kSplit ? at.part * p.ksteps / p.splits : 0; }
template <bool kSplit>
__device__ __forceinline__ int gemm_end(const GemmJob &p, const GemmTile &at) { return kSplit ? (at.part + 1) * p.ksteps / p.splits : p.ksteps; }

// The i-th tile of a CTA pair; false behind its last.  Job 0's tiles go round the pairs; the pairs that get one less of
// them take `extra` tiles of jobs 1 and 2 for it (as many as cost the same), whose remaining ones go round all pairs.
template <bool kJobs, bool kSplit>
__device__ __forceinline__ bool gemm_tile(const GemmArgs &p, int i, int pair, int pairs, GemmTile &at)
{
    const int n0 = p.job[0].tiles_m * p.job[0].tiles_n * (kSplit ? p.job[0].splits : 1);
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
            gemm_tile_at<kSplit>(p.job[at.job], t, at);
            return true;
        }
    }
    if (t >= n0) return false;
    gemm_tile_at<kSplit>(p.job[0], t, at);
    return true;
}

// 32 rows of 128 bytes on their way out: staged by lane = row with 16-byte chunks swizzled (no bank conflicts
// either way), stored with the lanes of a row side by side, whole 128-byte lines at a time.  (Tensor-map stores from the
// same place took 2.4 us per tile of 256 x 256 instead of 1.2: a copy costs its thread 130 ns, and the next one waits.)
// rows, bytes: how much of it is there, bytes a multiple of 16.
__device__ __forceinline__ uint32_t gemm_staged(uint32_t stage, int row, int chunk)
{
    return stage + row * 128 + ((chunk ^ (row & 7)) << 4);
}
// kTimes x 4 rows from row `first` on
template <int kTimes>
__device__ __forceinline__ void gemm_store_rows(void *to, long long pitch_bytes, int rows, int bytes, uint32_t stage, int lane, int first)
{
    const int chunk = lane & 7, mine = first + (lane >> 3);
    if (chunk * 16 < bytes) {
        uint8_t *at = static_cast<uint8_t *>(to) + mine * pitch_bytes + chunk * 16;
#pragma unroll
        for (int i = 0; i < kTimes; ++i) {
            const int row = mine + i * 4;
            if (row < rows) *reinterpret_cast<uint4 *>(at) = ld_shared_v4(gemm_staged(stage, row, chunk));
            at += 4 * pitch_bytes;
        }
    }
}
// 64 threads in two whole warps
__device__ __forceinline__ void barrier_sync_64(int id) { asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory"); }

// Rows of up to kCols accumulator columns, scaled where there are scales, as the result's type to where they belong.
// Lane = row; `stage` is the warp's, `scales` the same place before results lie there.
template <int kEpi, int kCols>
__device__ __forceinline__ void gemm_finish(const GemmArgs &p, const GemmJob &job, uint32_t (&v)[kCols], int row0, int rows, int col, int cols, float sx,
                                            uint32_t stage, float *scales, int lane)
{
    if constexpr (kEpi == kEpiScaled) {
        __syncwarp();
        scales[lane] = lane < cols ? p.col_scale[col + lane] : 0.0f;
        if (kCols == 64) scales[lane + 32] = lane + 32 < cols ? p.col_scale[col + 32 + lane] : 0.0f;
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kCols; i += 4) {
            const float4 w = *reinterpret_cast<const float4 *>(scales + i);
            v[i] = __float_as_uint(__int2float_rn((int)v[i]) * (sx * w.x));
            v[i + 1] = __float_as_uint(__int2float_rn((int)v[i + 1]) * (sx * w.y));
            v[i + 2] = __float_as_uint(__int2float_rn((int)v[i + 2]) * (sx * w.z));
            v[i + 3] = __float_as_uint(__int2float_rn((int)v[i + 3]) * (sx * w.w));
        }
    }
    const bool f32 = kEpi == kEpiScaled && p.out_f32;
    if (kEpi == kEpiScaled && p.direct) {
        // rows that start anywhere: a warp's stores of one row lie side by side
        float *const out_f = static_cast<float *>(job.out);
        __nv_bfloat16 *const out_b = static_cast<__nv_bfloat16 *>(job.out);
#pragma unroll
        for (int half = 0; half < kCols / 32; ++half) {
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 32; ++i) st_shared_u32(stage + lane * 128 + ((i ^ lane) << 2), v[half * 32 + i]);
            __syncwarp();
            const int cc = half * 32 + lane;
            if (cc < cols)
#pragma unroll 8
                for (int r = 0; r < rows; ++r) {
                    const float y = ld_shared_f32(stage + r * 128 + ((lane ^ r) << 2));
                    const long long to = (long long)(row0 + r) * job.ld + col + cc;
                    if (f32) out_f[to] = y;
                    else out_b[to] = __float2bfloat16_rn(y);
                }
        }
    } else if (f32) {
#pragma unroll
        for (int half = 0; half < kCols / 32; ++half) {
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 8; ++j)
                st_shared_v4(gemm_staged(stage, lane, j), make_uint4(v[half * 32 + j * 4], v[half * 32 + j * 4 + 1],
                                                                       v[half * 32 + j * 4 + 2], v[half * 32 + j * 4 + 3]));
            __syncwarp();
            gemm_store_rows<8>(static_cast<float *>(job.out) + row0 * job.ld + col + half * 32, job.ld * 4, rows,
                               (cols - half * 32) * 4, stage, lane, 0);
        }
    } else {
        __syncwarp();
#pragma unroll
        for (int j = 0; j < kCols / 8; ++j) {
            uint32_t w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                w[q] = pack_bf16x2(__uint_as_float(v[j * 8 + q * 2]), __uint_as_float(v[j * 8 + q * 2 + 1]));
            st_shared_v4(gemm_staged(stage, lane, j), make_uint4(w[0], w[1], w[2], w[3]));
        }
        __syncwarp();
        gemm_store_rows<8>(static_cast<__nv_bfloat16 *>(job.out) + row0 * job.ld + col, job.ld * 2, rows, cols * 2, stage, lane, 0);
    }
}

// The parts' sums of 32 columns, added up in the order of K.
template <bool kI8>
__device__ __forceinline__ void gemm_join(uint32_t (&v)[32], const uint32_t *sums, size_t part_words, int splits)
{
    uint32_t w[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __ldcg(sums + i * 128);
#pragma unroll 1
    for (int part = 1; part < splits; ++part) {
#pragma unroll
        for (int i = 0; i < 32; ++i) w[i] = __ldcg(sums + part * part_words + i * 128);
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = kI8 ? v[i] + w[i] : __float_as_uint(__uint_as_float(v[i]) + __uint_as_float(w[i]));
    }
}

// h of 32 columns from col on (N: columns of g), packed to bf16.
template <bool kI8>
__device__ __forceinline__ void gemm_gate(const GemmArgs &p, uint32_t (&g)[32], uint32_t (&u)[32], uint32_t *packed, int col, int cols, int N, float sx,
                                          float *scales, int lane)
{
    if constexpr (kI8) {
        const bool there = lane < cols;
        __syncwarp();
        scales[lane] = there ? p.col_scale[col + lane] : 0.0f;
        scales[lane + 32] = there ? p.col_scale[N + col + lane] : 0.0f;
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
    for (int i = 0; i < 16; ++i)
        packed[i] = pack_bf16x2(gated(__uint_as_float(g[2 * i]), __uint_as_float(u[2 * i])),
                                gated(__uint_as_float(g[2 * i + 1]), __uint_as_float(u[2 * i + 1])));
}

// kSplit: job 0's K cut into parts.  (A form of its own: the same code under a branch took 0.4 to 0.9 us from every other call.)
template <int kEpi, bool kI8, bool kSplit>
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
        for (int i = 0; i < 2; ++i) { mbar_init(&bars.acc_full[i], 1); mbar_init(&bars.acc_empty[i], 16); }
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
        fence_proxy_async_global();      // what the launch before wrote with ordinary stores is read by tensor copies
        int s = 0;
        uint32_t ph = 0;
        for (int i = 0; ok && gemm_tile<kJobs, kSplit>(p, i, pair, pairs, at); ++i) {
            for (int phase = 0; phase < kPhases && ok; ++phase) {
                const GemmJob &job = p.job[kPhases == 2 ? phase : at.job];
                const bool dh = kPhases == 2 && phase == 0;
                const bool a_mn = kJobs && job.a_mn, b_mn = kJobs ? job.b_mn != 0 : dh;
                const int half = kGatedTile && !dh ? job.width : job.width / 2;          // this CTA's rows of B
                const uint32_t tx = 2u * (uint32_t)(job.rows + half) * 128u + ((blockIdx.x & ~1u) == p.withhold ? 16u : 0u);
                const void *map = load_a ? &job.a : &job.b[rank];
                const int mn = load_a ? at.m0 + (int)rank * job.rows : at.n0 + (kGatedTile && !dh ? 0 : (int)rank * half);
                const bool mn_major = load_a ? a_mn : b_mn;
                const bool second = load_a ? a_mn : b_mn && half == 128;
                const int from = gemm_first<kSplit>(job, at), to = gemm_end<kSplit>(job, at);
                for (int k = from; k < to; ++k) {
                    ok = __all_sync(0xffffffffu, ffn_wait(&bars.empty[s], ph ^ 1u, wc, 1 + warp));
                    if (!ok) break;
                    const uint32_t dst = smem + s * p.stage_bytes + (load_a ? 0 : p.a_bytes);
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
            for (int n = 0; ok && gemm_tile<kJobs, kSplit>(p, n, pair, pairs, at); ++n) {
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
                    const bool b_32 = dh && job.width == 64;
                    const uint64_t a_inc = a_mn ? 128 : 2, b_inc = b_32 ? 64 : b_mn ? 128 : 2;
                    const int from = gemm_first<kSplit>(job, at), to = gemm_end<kSplit>(job, at);
                    for (int k = from; k < to; ++k) {
                        ok = __all_sync(0xffffffffu, ffn_wait(&bars.full[s], ph, wc, 4));
                        if (!ok) break;
                        tc_fence_after();
                        const uint32_t a = smem + s * p.stage_bytes, b = a + p.a_bytes;      // (128 rows are read from a on, whatever lies there)
                        ffn_mma_kstep_pair<kI8>(d, a_mn ? umma_desc_mn_sw128(a) : umma_desc_sw128(a),
                                                b_32 ? umma_desc_mn_sw64(b) : b_mn ? umma_desc_mn_sw128(b) : umma_desc_sw128(b), a_inc, b_inc, idesc, (uint32_t)(k != from),
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
        // ---- epilogue: each warp the 32 accumulator lanes of its quarter, this CTA's rows from 32 quarter on; two warps
        // share a quarter, 64 columns in turn
        const int quarter = warp & 3, group = (warp - 4) >> 2;
        const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
        const uint32_t stage = smem + kGemmSmemStaging + (warp - 4) * kGemmStaging;
        float *const scales = reinterpret_cast<float *>(smem_g + kGemmSmemStaging + (warp - 4) * kGemmStaging);      // before results lie there
        const uint32_t empty0 = mapa_u32(smem_u32(&bars.acc_empty[0]), 0);
        pdl_wait();
        for (int n = 0; gemm_tile<kJobs, kSplit>(p, n, pair, pairs, at); ++n) {
            const GemmJob &job = p.job[at.job];
            const int N = job.N, width = job.width, n0 = at.n0, buf = n & 1;
            const int row0 = at.m0 + (int)rank * job.rows + quarter * 32;
            const int rows = min(min(32, job.rows - quarter * 32), job.M - row0);       // the warp's; may be none
            ok = __all_sync(0xffffffffu, ffn_wait(&bars.acc_full[buf], (n >> 1) & 1, wc, 5));
            const bool split = kSplit && (!kJobs || job.splits > 1);
            // where barriers follow, all of those who meet there go on or none
            if (split) ok = named_barrier_and<6, 256>(ok);
            if (kEpi == kEpiGrad) ok = barrier_and_64(1 + quarter, ok);
            if (!ok) break;
            tc_fence_after();
            // accumulator read: hand it back to the pair's issuer
            const auto release = [&]() {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_remote(kEpi == kEpiGrad ? empty0 : empty0 + buf * 8);
            };
            if (rows <= 0 && !split) {
                release();
                continue;
            }
            float sx = 0.0f;
            if constexpr (kI8) sx = lane < rows ? p.row_scale[row0 + lane] : 0.0f;

            // A part's sums, of `columns` of the accumulator; whoever is last adds them all up.  32 columns by each group in turn, so
            // that both have some in narrow tiles.  (64 at a time: 25.3 instead of 22.1 us for T = 128, 264 x 8120, 17.5 instead of
            // 15.7 for 100 x 14336 -> 520 in 8 bits, the same in wide ones; loads of two parts at a time: within 3 % either way.)
            const size_t part_words = (size_t)(((kGatedTile ? 2 : 1) * width + 63) / 64) * 64 * 128 * 2;        // of a pair
            uint32_t *const sums = p.partials + (size_t)at.index * job.splits * part_words + rank * (part_words / 2) + quarter * 32 + lane;
            const int there = min(width, N - n0);
            const auto arrive = [&](int columns) -> bool {
                for (int c = group * 32; c < columns; c += 64) {
                    uint32_t v[32];
                    tmem_ld_32x32(lane_base + buf * 256 + c, v);
                    tmem_ld_wait32(v);
                    if (rows > 0)
#pragma unroll
                        for (int i = 0; i < 32; ++i) __stcg(sums + at.part * part_words + (size_t)(c + i) * 128, v[i]);
                }
                release();
                __threadfence();
                named_barrier_sync<6, 256>();
                if (threadIdx.x == 128) {
                    unsigned *const arrived = &p.ctl->arrived[at.index * 2 + rank];
                    bars.last = atom_acqrel_add_u32(arrived, 1u) == (unsigned)job.splits - 1u;
                    if (bars.last) *arrived = 0u;
                }
                named_barrier_sync<6, 256>();
                __threadfence();
                return bars.last && rows > 0;
            };

            if constexpr (kEpi == kEpiStore || kEpi == kEpiScaled) {
                if (split) {
                    if (!arrive(there)) continue;
#pragma unroll 1
                    for (int c = group * 32; c < there; c += 64) {
                        uint32_t v[32];
                        gemm_join<kI8>(v, sums + (size_t)c * 128, part_words, job.splits);
                        gemm_finish<kEpi, 32>(p, job, v, row0, rows, n0 + c, min(32, there - c), sx, stage, scales, lane);
                    }
                    continue;
                }
                const int last = min((width - 1) / 64, (N - 1 - n0) / 64);
                if (group > last) release();
#pragma unroll 1
                for (int c = group; c <= last; c += 2) {
                    const int col = n0 + c * 64, cols = min(min(64, width - c * 64), N - col);
                    uint32_t v[64];
                    tmem_ld_32x64(lane_base + buf * 256 + c * 64, v);
                    tmem_ld_wait64(v);
                    if (c + 2 > last) release();
                    gemm_finish<kEpi, 64>(p, job, v, row0, rows, col, cols, sx, stage, scales, lane);
                }
            } else if constexpr (kEpi == kEpiGated || kEpi == kEpiScaledGated) {
                __nv_bfloat16 *const out = static_cast<__nv_bfloat16 *>(job.out) + row0 * job.ld + n0;
                if (split) {
                    if (!arrive(2 * width)) continue;
#pragma unroll 1
                    for (int c = group * 32; c < there; c += 64) {
                        const int cols = min(32, there - c);
                        uint32_t g[32], u[32], packed[16];
                        gemm_join<kI8>(g, sums + (size_t)c * 128, part_words, job.splits);
                        gemm_join<kI8>(u, sums + (size_t)(width + c) * 128, part_words, job.splits);
                        gemm_gate<kI8>(p, g, u, packed, n0 + c, cols, N, sx, scales, lane);
                        __syncwarp();
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            st_shared_v4(gemm_staged(stage, lane, j), make_uint4(packed[j * 4], packed[j * 4 + 1], packed[j * 4 + 2], packed[j * 4 + 3]));
                        __syncwarp();
                        gemm_store_rows<8>(out + c, job.ld * 2, rows, cols * 2, stage, lane, 0);
                    }
                    continue;
                }
                const int last = (there - 1) / 64;
                if (group > last) release();
#pragma unroll 1
                for (int c = group; c <= last; c += 2) {
                    const int cols = min(64, there - c * 64);
                    uint32_t packed[32];
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int cc = c * 64 + half * 32;
                        uint32_t g[32], u[32];
                        tmem_ld_32x32(lane_base + buf * 256 + cc, g);
                        tmem_ld_32x32(lane_base + buf * 256 + width + cc, u);
                        tmem_ld_wait32(g);
                        reg_fence32(u);
                        if (c + 2 > last && half == 1) release();
                        gemm_gate<kI8>(p, g, u, packed + half * 16, n0 + cc, cols - half * 32, N, sx, scales, lane);
                    }
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        st_shared_v4(gemm_staged(stage, lane, j), make_uint4(packed[j * 4], packed[j * 4 + 1], packed[j * 4 + 2], packed[j * 4 + 3]));
                    __syncwarp();
                    gemm_store_rows<8>(out + c * 64, job.ld * 2, rows, cols * 2, stage, lane, 0);
                }
            } else {
                // 64 columns at a time, 32 of them by each of a quarter's two warps, which stage a result's rows side by side
                // and store half of them each: whole lines.  Two places in turn; a place's readers have met at the barrier
                // of the other one
                const int last = (min(width, N - n0) - 1) / 64;
                const uint32_t place = smem + kGemmSmemStaging + quarter * kGemmStaging;
                uint32_t turn = 0;
#pragma unroll 1
                for (int c = 0; c <= last; ++c) {
                    const int from = c * 64 + group * 32, col = n0 + c * 64, cols = min(64, N - col);
                    uint32_t g[32], u[32], d[32];
                    tmem_ld_32x32(lane_base + from, g);
                    tmem_ld_32x32(lane_base + width + from, u);
                    tmem_ld_32x32(lane_base + 256 + buf * 128 + from, d);
                    tmem_ld_wait32(g);
                    reg_fence32(u);
                    reg_fence32(d);
                    if (c == last) release();
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        float r[3][2];
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const float fg = __uint_as_float(g[i + q]), fu = __uint_as_float(u[i + q]), fd = __uint_as_float(d[i + q]);
                            const float sg = fast_sigmoid(fg), si = fg * sg;
                            r[0][q] = si * fu;                                         // h
                            r[1][q] = fd * fu * sg * (1.0f + fg * (1.0f - sg));        // dg
                            r[2][q] = fd * si;                                         // du
                        }
                        g[i / 2] = pack_bf16x2(r[0][0], r[0][1]);
                        u[i / 2] = pack_bf16x2(r[1][0], r[1][1]);
                        d[i / 2] = pack_bf16x2(r[2][0], r[2][1]);
                    }
#pragma unroll
                    for (int w = 0; w < 3; ++w) {
                        const uint32_t *v = w == 0 ? g : w == 1 ? u : d;
                        const GemmJob &to = p.job[w];
                        const uint32_t at_place = place + turn * (4 * kGemmStaging);
                        turn ^= 1u;
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            st_shared_v4(gemm_staged(at_place, lane, group * 4 + j), make_uint4(v[j * 4], v[j * 4 + 1], v[j * 4 + 2], v[j * 4 + 3]));
                        barrier_sync_64(1 + quarter);
                        gemm_store_rows<4>(static_cast<__nv_bfloat16 *>(to.out) + row0 * to.ld + col, to.ld * 2, rows, cols * 2, at_place, lane, group * 16);
                    }
                }
            }
        }
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
