// The feed-forward block, or one 8-bit product, for up to 128 tokens in ONE cooperative launch: a stream of weights
// that never stops between the two products.
//
// Split.  Each CTA gets an equal range of the result's columns (rows of the weight matrix; a TMA box may have any
// number of rows) and the whole of K, so no sum is shared between CTAs.  (A first version cut K as well and joined
// partial sums through L2: with HBM saturated every dependent access takes 3-4 us, and 64 tokens through 4096 -> 28672
// took 45 us instead of 28.)
//
// Products.  Weights on the MMA's M axis (128), tokens on its N axis.  A tcgen05.mma takes 48 cycles however few of its
// rows and columns are used, so where a CTA has few rows, `kbs` blocks of K lie side by side: A = (block, row) on M,
// B = (block, token) on N, of D only the blocks on the diagonal are used, and the epilogue adds them up.  With 28 rows
// and 16 tokens that is 4 blocks per product, 5.6 us of tensor pipe for K = 14336 instead of 23.6.  One tensor copy
// brings all blocks of a step: they are a dimension of the tensor map (where K is whole blocks; else kbs = 1).
//
// Order.  Weights are fetched as fast as slots of the ring become free, straight from the first product into the
// second; tokens follow when they are there.  The result h of the first product crosses between SMs through L2 behind a
// grid barrier, which the up to 190 KB of weights in flight per SM cover.  The 8-bit forms round the tokens to integers
// in the kernel, one row per CTA, behind barriers of the same kind.
//
// Bound: HBM (the weights).
#pragma once
#include "weave_gemm.cuh"
#include "weave_quant.cuh"

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
__device__ __forceinline__ void tma_load_3d_one(uint32_t dst, const void *map, int x, int y, int z, uint64_t *bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
                 : "memory");
}
__device__ __forceinline__ void tma_load_4d_one(uint32_t dst, const void *map, int x, int y, int z, int w, uint64_t *bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
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
__device__ __forceinline__ void tmem_ld_wait8(uint32_t (&r)[8])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7])
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
__device__ __forceinline__ void red_release_add_u64(unsigned long long *p, unsigned long long v)
{
    asm volatile("red.release.gpu.global.add.u64 [%0], %1;" ::"l"(p), "l"(v) : "memory");
}
__device__ __forceinline__ unsigned long long ld_acquire_u64(const unsigned long long *p)
{
    unsigned long long v;
    asm volatile("ld.acquire.gpu.global.u64 %0, [%1];" : "=l"(v) : "l"(p) : "memory");
    return v;
}

// ------------------------------------------------------------------------------------ the plan

constexpr int kSmallThreads = 384;               // weights, tokens, issuer, (idle), eight epilogue warps
constexpr int kSmallMaxT = 128;
constexpr int kSmallMaxSlots = 16;
constexpr int kSmallRed = 128 * 9 * 4;           // an epilogue group's exchange buffer: 128 rows x 8 tokens, padded
constexpr int kSmallSmemMax = 232448;
constexpr int kSmallTail = 16384;                // behind the ring: exchange buffers and barriers
constexpr int kSmallRing = kSmallSmemMax - 1024 - kSmallTail;

// one product: how its columns are cut into tiles and its K into steps
struct SmallShape {
    int n;               // columns of the result (gated: of h)
    int ct;              // columns of a tile
    int rounds;          // tiles of a CTA, at most: CTA c has tiles c * rounds ...
    int rows;            // weight rows per block of K: ct, gated 2 ct
    int kbs;             // blocks of K per step
    int steps;           // steps of a tile
    int box_t;           // tokens of a block, padded
    int w_bytes, x_bytes;
    int slots, slot_bytes, x_offset;     // of the ring while this product runs
};

__host__ __device__ inline int small_box(int T, int kbs)
{
    const int b = T <= 8 ? 8 : T <= 16 ? 16 : T <= 32 ? 32 : T <= 64 ? 64 : 128;
    return b == 8 && kbs == 1 ? 16 : b;          // N is a multiple of 16
}

// The ring's slots have another size in the second product.  Its first one is the first that starts behind the slot the
// first product wrote last, so that slots are taken over in the order in which they become free.
__device__ __forceinline__ int small_first_slot(const SmallShape &before, const SmallShape &s, int steps_before)
{
    const int at = (steps_before % before.slots * before.slot_bytes + s.slot_bytes - 1) / s.slot_bytes;
    return at < s.slots ? at : 0;
}
// steps of a CTA's tiles
__device__ __forceinline__ int small_steps(const SmallShape &s)
{
    const int tiles = (s.n + s.ct - 1) / s.ct, first = blockIdx.x * s.rounds;
    return max(0, min(s.rounds, tiles - first)) * s.steps;
}

// block: elements of K in 128 bytes
inline SmallShape small_shape(int n, bool gated, long long K, int block, int T, int ctas)
{
    SmallShape s;
    s.n = n;
    const int most = gated ? 64 : 128;
    s.rounds = (int)((n + (long long)ctas * most - 1) / ((long long)ctas * most));
    s.ct = (int)((n + (long long)ctas * s.rounds - 1) / ((long long)ctas * s.rounds));
    s.rows = gated ? 2 * s.ct : s.ct;
    const long long blocks = (K + block - 1) / block;
    s.kbs = 1;
    if (K % block == 0)
        // cycles per block of a product over kbs of them, half of N but at least 48; fewer only if that is worth it
        for (int k = 2; k <= 8 && k * s.rows <= 128 && k * small_box(T, k) <= 256 && k <= blocks; k *= 2) {
            const int now = small_box(T, s.kbs) * s.kbs / 2, then = small_box(T, k) * k / 2;
            if ((then < 48 ? 48 : then) * s.kbs < (now < 48 ? 48 : now) * k) s.kbs = k;
        }
    s.box_t = small_box(T, s.kbs);
    s.steps = (int)((blocks + s.kbs - 1) / s.kbs);
    s.w_bytes = s.kbs * s.rows * 128;
    s.x_bytes = s.kbs * s.box_t * 128;
    s.x_offset = (s.w_bytes + 1023) & ~1023;
    s.slot_bytes = s.x_offset + ((s.x_bytes + 1023) & ~1023);
    s.slots = kSmallRing / s.slot_bytes;
    if (s.slots > kSmallMaxSlots) s.slots = kSmallMaxSlots;
    return s;
}

// ------------------------------------------------------------------------------------ the kernel

struct alignas(64) SmallProduct {
    CUtensorMap w;           // {K, rows, halves, 1} or {block, rows, halves, blocks}
    CUtensorMap x;           // {K, T, 1} or {block, T, blocks}
    SmallShape s;
    int gated, out_f32;
    const float *row_scale;  // 8-bit forms: [T], and [n] (gated: [2n], gate then up)
    const float *col_scale;
    void *out;
    // 8-bit forms: the tokens in bf16 or fp32 that are rounded before this product (NULL: they are integers already)
    const void *round_src;
    int8_t *round_dst;
    float *round_scale;
    int round_f32, K;
};

struct alignas(64) SmallArgs {
    SmallProduct p[2];
    FfnCtl *ctl;
    unsigned long long timeout_ns;
    int products, T;
    int acc_cols, tmem_cols;
};

struct SmallBars {
    uint64_t full[2][kSmallMaxSlots], empty[2][kSmallMaxSlots];      // [product]
    uint64_t acc_full[2], acc_empty[2];
    uint64_t tokens[2];          // the tokens of product i are in memory
    uint32_t tmem_base;
    uint32_t row_max[8];
    float row_scale[kSmallMaxT];
};
// a product reads 128 rows from the start of a slot, whatever it holds: the 16 KB behind the ring are ours, too
static_assert(2 * kSmallRed + sizeof(SmallBars) <= kSmallTail, "the tail of shared memory");

// All CTAs' epilogue warps arrive here with what they wrote; true when everybody has.  The counter only grows, by the
// grid size per barrier and launch, so nothing has to be reset; what it will reach is known to whoever reads it before
// his own arrival (small_barrier_target).
__device__ __forceinline__ unsigned long long small_barrier_target(const unsigned long long *counter)
{
    const unsigned long long g = gridDim.x;
    return (ld_acquire_u64(counter) / g + 1) * g;
}
__device__ __forceinline__ bool small_grid_barrier(unsigned long long *counter, unsigned long long target, bool ok, const WaitCtx &wc, int where)
{
    __threadfence();
    fence_proxy_async_global();          // ordinary stores here, tensor-map loads there
    ok = named_barrier_and<1, 256>(ok);
    if (ok && threadIdx.x == 128) {
        red_release_add_u64(counter, 1ull);
        unsigned long long t0 = 0;
        unsigned it = 0;
        while (ld_acquire_u64(counter) < target) {
            __nanosleep(64);             // 148 of these loads at once would keep the last arrivals from the counter
            if ((++it & 31u) == 0u) {
                if (*reinterpret_cast<volatile int *>(&wc.ctl->status) != 0) { ok = false; break; }
                const unsigned long long now = globaltimer_ns();
                if (t0 == 0) t0 = now;
                else if ((long long)(now - t0) > (long long)wc.timeout_ns) {
                    if (atomicCAS(&wc.ctl->status, 0, kFfnErrTimeout) == 0) wc.ctl->where = where;
                    ok = false;
                    break;
                }
            }
        }
        fence_proxy_async_global();
    }
    ok = named_barrier_and<1, 256>(ok);
    __threadfence();
    return ok;
}

template <bool kI8>
__device__ __forceinline__ float small_value(uint32_t acc, float sx, float sw)
{
    return kI8 ? __int2float_rn((int)acc) * (sx * sw) : __uint_as_float(acc);
}

template <bool kI8>
__global__ void __launch_bounds__(kSmallThreads, 1) weave_ffn_small_kernel(const __grid_constant__ SmallArgs a)
{
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *const behind = smem_raw + (smem - smem_u32(smem_raw)) + kSmallRing;
    SmallBars &bars = *reinterpret_cast<SmallBars *>(behind + 2 * kSmallRed);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const WaitCtx wc = {a.ctl, a.timeout_ns};
    constexpr int kBlock = kI8 ? 128 : 64;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kSmallMaxSlots; ++i)
            for (int j = 0; j < 2; ++j) { mbar_init(&bars.full[j][i], 2); mbar_init(&bars.empty[j][i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&bars.acc_full[i], 1); mbar_init(&bars.acc_empty[i], 8); mbar_init(&bars.tokens[i], 1); }
        fence_mbar_init();
    }
    if (warp == 2) { tmem_alloc_one(&bars.tmem_base, (uint32_t)a.tmem_cols); tmem_relinquish_one(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars.tmem_base;

    bool ok = true;
    if (warp < 2) {
        // ---- producers: warp 0 the weights, warp 1 the tokens
        if (lane == 0) {
            const bool weights = warp == 0;
#pragma unroll          // both products' parameters at fixed places of the constant bank
            for (int i = 0; i < 2; ++i) {
                if (i >= a.products || !ok) break;
                const SmallProduct &p = a.p[i];
                const int before = i > 0 ? small_steps(a.p[0].s) : 0, start = i > 0 ? small_first_slot(a.p[0].s, p.s, before) : 0;
                const int turns = i > 0 ? before / a.p[0].s.slots : 0, rest = i > 0 ? before % a.p[0].s.slots : 0;
                int slot = start, n = 0;
                uint32_t ph = 0;
                tma_prefetch_desc(weights ? &p.w : &p.x);
                if (!weights && (i > 0 || (kI8 && p.round_src))) {
                    ok = ffn_wait(&bars.tokens[i], 0, wc, 20 + i);
                    fence_proxy_async_global();
                }
                const bool one = p.s.kbs == 1;
                for (int r = 0; r < p.s.rounds && ok; ++r) {
                    const int col0 = (blockIdx.x * p.s.rounds + r) * p.s.ct;
                    if (col0 >= p.s.n) break;
                    for (int k = 0; k < p.s.steps; ++k) {
                        if (i == 0 || n >= p.s.slots) {
                            ok = ffn_wait(&bars.empty[i][slot], ph ^ 1u, wc, 22 + (int)weights);
                        } else if (weights) {
                            // first use of a slot: the newest step of the product before that lies in it.  (Tokens come
                            // behind the grid barrier, when all of those are done with.)
                            const SmallShape &o = a.p[0].s;
                            int j = min(o.slots - 1, ((slot + 1) * p.s.slot_bytes - 1) / o.slot_bytes);
                            if (j >= rest && slot * p.s.slot_bytes < rest * o.slot_bytes) j = rest - 1;
                            const int uses = turns + (j < rest ? 1 : 0);
                            if (uses > 0) ok = ffn_wait(&bars.empty[0][j], (uint32_t)(uses - 1) & 1u, wc, 23);
                        }
                        if (!ok) break;
                        uint64_t *full = &bars.full[i][slot];
                        const uint32_t dst = smem + slot * p.s.slot_bytes;
                        mbar_arrive_expect_tx(full, (uint32_t)(weights ? p.s.w_bytes : p.s.x_bytes));
                        if (weights) tma_load_4d_one(dst, &p.w, one ? k * kBlock : 0, col0, 0, one ? 0 : k * p.s.kbs, full);
                        else tma_load_3d_one(dst + p.s.x_offset, &p.x, one ? k * kBlock : 0, 0, one ? 0 : k * p.s.kbs, full);
                        ++n;
                        if (++slot == p.s.slots) slot = 0;
                        if (slot == start) ph ^= 1u;
                    }
                }
            }
            if (!ok) ffn_linger();
        }
        __syncwarp();
    } else if (warp == 2) {
        if (lane == 0) {
            int n = 0;
#pragma unroll          // both products' parameters at fixed places of the constant bank
            for (int i = 0; i < 2; ++i) {
                if (i >= a.products || !ok) break;
                const SmallShape &s = a.p[i].s;
                const int start = i > 0 ? small_first_slot(a.p[0].s, s, small_steps(a.p[0].s)) : 0;
                int slot = start;
                uint32_t ph = 0;
                const uint32_t idesc = kI8 ? umma_idesc_i8(128, s.kbs * s.box_t) : umma_idesc_bf16(128, s.kbs * s.box_t);
                for (int r = 0; r < s.rounds && ok; ++r, ++n) {
                    if ((blockIdx.x * s.rounds + r) * s.ct >= s.n) break;
                    const int buf = n & 1;
                    ok = ffn_wait(&bars.acc_empty[buf], ((n >> 1) & 1) ^ 1, wc, 24);
                    tc_fence_after();
                    for (int k = 0; k < s.steps && ok; ++k) {
                        ok = ffn_wait(&bars.full[i][slot], ph, wc, 25);
                        if (!ok) break;
                        tc_fence_after();
                        const uint32_t w = smem + slot * s.slot_bytes;
                        ffn_mma_kstep_one<kI8>(tmem + (uint32_t)(buf * a.acc_cols), umma_desc_sw128(w), umma_desc_sw128(w + s.x_offset), idesc,
                                               (uint32_t)(k != 0));
                        tc_commit_one(&bars.empty[i][slot]);
                        if (++slot == s.slots) slot = 0;
                        if (slot == start) ph ^= 1u;
                    }
                    if (ok) tc_commit_one(&bars.acc_full[buf]);
                }
            }
            if (!ok) ffn_linger();
        }
        __syncwarp();
    } else if (warp >= 4) {
        // ---- epilogue: two groups of four warps take turns in blocks of eight tokens; a warp reads the accumulator
        // lanes of its number mod 4
        const int quarter = warp & 3, group = (warp - 4) >> 2, tid = threadIdx.x - 128 - group * 128;
        const int acc_row = quarter * 32 + lane;
        uint32_t *const red = reinterpret_cast<uint32_t *>(behind + group * kSmallRed);
        unsigned long long target[3] = {0, 0, 0};
        if (threadIdx.x == 128)
#pragma unroll
            for (int j = 0; j < 3; ++j) target[j] = small_barrier_target(&a.ctl->barrier[j]);
        int n = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (i >= a.products || !ok) break;
            const SmallProduct &p = a.p[i];
            const SmallShape &s = p.s;
            if (i > 0) ok = small_grid_barrier(&a.ctl->barrier[0], target[0], ok, wc, 26);
            if constexpr (kI8) {
                if (ok && p.round_src) {
                    for (int row = blockIdx.x; row < a.T; row += gridDim.x) {
                        const int tid256 = threadIdx.x - 128;
                        if (p.round_f32)
                            quant_row_by<float, 256, true, true>(static_cast<const float *>(p.round_src), p.round_dst, p.round_scale, row, p.K, tid256,
                                                                 bars.row_max);
                        else
                            quant_row_by<__nv_bfloat16, 256, true, true>(static_cast<const __nv_bfloat16 *>(p.round_src), p.round_dst, p.round_scale,
                                                                         row, p.K, tid256, bars.row_max);
                        named_barrier_sync<1, 256>();
                    }
                    ok = small_grid_barrier(&a.ctl->barrier[1 + i], i == 0 ? target[1] : target[2], ok, wc, 27);
                }
            }
            if (!ok) break;
            if (threadIdx.x == 128) mbar_arrive(&bars.tokens[i]);
            if constexpr (kI8) {
                // (read behind the barriers in the tile's loop)
                for (int t = threadIdx.x - 128; t < a.T; t += 256) bars.row_scale[t] = __ldcg(p.row_scale + t);
            }
            const int blocks_from = quarter * 32 / s.rows, blocks_to = min(s.kbs - 1, (quarter * 32 + 31) / s.rows), mine = acc_row / s.rows;
            int pow2 = 1;
            while (pow2 < s.ct) pow2 *= 2;
            for (int r = 0; r < s.rounds; ++r, ++n) {
                const int col0 = (blockIdx.x * s.rounds + r) * s.ct;
                if (col0 >= s.n) break;
                const int cols = min(s.ct, s.n - col0), buf = n & 1;
                // a thread's column of the tile, and which of the eight tokens it starts with
                const int c = tid & (pow2 - 1), t_first = tid / pow2, t_step = 128 / pow2;
                float sw0 = 0.0f, sw1 = 0.0f;
                if constexpr (kI8) {
                    if (c < cols) {
                        sw0 = p.col_scale[col0 + c];
                        if (p.gated) sw1 = p.col_scale[s.n + col0 + c];
                    }
                }
                ok = ffn_wait(&bars.acc_full[buf], (n >> 1) & 1, wc, 28);
                ok = named_barrier_and<1, 256>(ok);       // barriers follow: all warps leave together
                if (!ok) break;
                tc_fence_after();
                const uint32_t acc = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * a.acc_cols);
                for (int t0 = group * 8; t0 < a.T; t0 += 16) {
                    uint32_t v[8];
                    for (int b = blocks_from; b <= blocks_to; ++b) {
                        uint32_t w[8];
                        tmem_ld_32x8(acc + (uint32_t)(b * s.box_t + t0), w);
                        tmem_ld_wait8(w);
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] = b == mine || b == blocks_from ? w[j] : v[j];
                    }
                    if (blocks_from <= blocks_to) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) red[acc_row * 9 + j] = v[j];
                    }
                    if (group == 0) named_barrier_sync<2, 128>();
                    else named_barrier_sync<3, 128>();
                    const int left = min(8, a.T - t0);
                    if (c < cols) {
                        uint8_t *const to = static_cast<uint8_t *>(p.out) + ((long long)(t0 + t_first) * s.n + col0 + c) * (p.out_f32 ? 4 : 2);
                        const int step_bytes = s.n * t_step * (p.out_f32 ? 4 : 2);
                        const uint32_t *const from = red + c * 9 + t_first;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int t = t_first + j * t_step;
                            if (t >= left) break;
                            const uint32_t *const v = from + j * t_step;
                            uint32_t sum0 = v[0], sum1 = p.gated ? v[s.ct * 9] : 0u;
                            for (int b = 1; b < s.kbs; ++b) {
                                const uint32_t *const w = v + b * s.rows * 9;
                                if constexpr (kI8) {
                                    sum0 += w[0];
                                    if (p.gated) sum1 += w[s.ct * 9];
                                } else {
                                    sum0 = __float_as_uint(__uint_as_float(sum0) + __uint_as_float(w[0]));
                                    if (p.gated) sum1 = __float_as_uint(__uint_as_float(sum1) + __uint_as_float(w[s.ct * 9]));
                                }
                            }
                            const float sx = kI8 ? bars.row_scale[t0 + t] : 0.0f;
                            float y = small_value<kI8>(sum0, sx, sw0);
                            if (p.gated) y = gated(y, small_value<kI8>(sum1, sx, sw1));
                            uint8_t *const at = to + (long long)j * step_bytes;
                            if (p.out_f32) *reinterpret_cast<float *>(at) = y;
                            else *reinterpret_cast<__nv_bfloat16 *>(at) = __float2bfloat16_rn(y);
                        }
                    }
                    if (group == 0) named_barrier_sync<2, 128>();
                    else named_barrier_sync<3, 128>();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.acc_empty[buf]);
            }
        }
        if (!ok) ffn_linger();
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 2) tmem_dealloc_one(tmem, (uint32_t)a.tmem_cols);
}

}  // namespace weave
