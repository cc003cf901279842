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
// brings all blocks of a step: they are a dimension of the tensor map.  What K has behind its last whole block is a step
// of its own, clipped by another map, whose product is the block's own N wide.
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
// The forms below are called by a whole converged warp; the elected thread issues, everything else stays
// warp-uniform, so that operands live in uniform registers (from one lane of a divergent branch a step of the ring took
// 330 ns however little it moved).

// four products over 128 bytes of K, K-major operands, and the commit that frees their slot
template <bool kI8>
__device__ __forceinline__ void ffn_mma_kstep_one(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate_first,
                                                  uint64_t *empty_bar)
{
#define WEAVE_KSTEP_ONE(KIND)                                                                   \
    asm volatile(                                                                               \
        "{\n\t.reg .pred pe, pa, pt;\n\t"                                                       \
        ".reg .b64 a1, a2, a3, b1, b2, b3;\n\t"                                                 \
        "elect.sync _|pe, 0xffffffff;\n\t"                                                      \
        "setp.ne.b32 pa, %4, 0;\n\t"                                                            \
        "setp.eq.u32 pt, %0, %0;\n\t"                                                           \
        "add.u64 a1, %1, 2;\n\tadd.u64 a2, %1, 4;\n\tadd.u64 a3, %1, 6;\n\t"                    \
        "add.u64 b1, %2, 2;\n\tadd.u64 b2, %2, 4;\n\tadd.u64 b3, %2, 6;\n\t"                    \
        "@pe tcgen05.mma.cta_group::1.kind::" KIND " [%0], %1, %2, %3, pa;\n\t"                 \
        "@pe tcgen05.mma.cta_group::1.kind::" KIND " [%0], a1, b1, %3, pt;\n\t"                 \
        "@pe tcgen05.mma.cta_group::1.kind::" KIND " [%0], a2, b2, %3, pt;\n\t"                 \
        "@pe tcgen05.mma.cta_group::1.kind::" KIND " [%0], a3, b3, %3, pt;\n\t"                 \
        "@pe tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%5];\n\t}"  \
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate_first), "r"(smem_u32(empty_bar)) : "memory")
    if (kI8) WEAVE_KSTEP_ONE("i8");
    else WEAVE_KSTEP_ONE("f16");
#undef WEAVE_KSTEP_ONE
}
__device__ __forceinline__ void tc_commit_one(uint64_t *bar)
{
    asm volatile(
        "{\n\t.reg .pred pe;\n\t"
        "elect.sync _|pe, 0xffffffff;\n\t"
        "@pe tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar)) : "memory");
}
// arrival with the byte count, and the copy
__device__ __forceinline__ void tma_fill(uint32_t dst, const void *map, int x, int y, int z, int w, uint64_t *bar, uint32_t bytes)
{
    asm volatile(
        "{\n\t.reg .pred pe;\n\t"
        "elect.sync _|pe, 0xffffffff;\n\t"
        "@pe mbarrier.arrive.expect_tx.shared::cta.b64 _, [%6], %7;\n\t"
        "@pe cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];\n\t}"
        ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar)), "r"(bytes)
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
__device__ __forceinline__ void red_release_add_u64(unsigned long long *p, unsigned long long v)
{
    asm volatile("red.release.gpu.global.add.u64 [%0], %1;" ::"l"(p), "l"(v) : "memory");
}
__device__ __forceinline__ unsigned long long ld_relaxed_u64(const unsigned long long *p)
{
    unsigned long long v;
    asm volatile("ld.relaxed.gpu.global.u64 %0, [%1];" : "=l"(v) : "l"(p) : "memory");
    return v;
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
constexpr int kSmallRedRow = 12;                 // words of a row of an epilogue group's exchange buffer: 8 tokens, padded
constexpr int kSmallRed = 128 * kSmallRedRow * 4;
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
    int full;            // whole blocks of K
    int tail_at;         // kbs > 1: the step of what is left behind them, or -1
    int box_t;           // tokens of a block, padded
    int w_bytes, x_bytes;
    int slots, slot_bytes, x_offset;     // of the ring while this product runs
};

// N = kbs * box is a multiple of 16, and so is the box where a tail's product is one box wide
__host__ __device__ inline int small_box(int T, int kbs, bool tail)
{
    return kbs == 1 || tail ? (T + 15) & ~15 : (T + 7) & ~7;
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

// The plan with kbs blocks of K per step; block: elements of K in 128 bytes.
inline SmallShape small_shape(int n, bool gated, long long K, int block, int T, int ctas, int kbs)
{
    SmallShape s;
    s.n = n;
    const int most = 128 / (gated ? 2 * kbs : kbs);
    s.rounds = (int)((n + (long long)ctas * most - 1) / ((long long)ctas * most));
    s.ct = (int)((n + (long long)ctas * s.rounds - 1) / ((long long)ctas * s.rounds));
    s.rows = gated ? 2 * s.ct : s.ct;
    s.kbs = kbs;
    s.full = (int)(K / block);
    const bool tail = kbs > 1 && K % block != 0;
    s.box_t = small_box(T, kbs, tail);
    s.steps = kbs > 1 ? (s.full + kbs - 1) / kbs + tail : (int)((K + block - 1) / block);
    s.tail_at = tail ? s.steps - 1 : -1;
    s.w_bytes = kbs * s.rows * 128;
    s.x_bytes = kbs * s.box_t * 128;
    s.x_offset = (s.w_bytes + 1023) & ~1023;
    s.slot_bytes = s.x_offset + ((s.x_bytes + 1023) & ~1023);
    s.slots = kSmallRing / s.slot_bytes;
    if (s.slots > kSmallMaxSlots) s.slots = kSmallMaxSlots;
    return s;
}
// Microseconds that a product takes with this plan, from measurements: the chip reads weights at 6.4 TB/s (a little less
// where a step takes only 128 or 256 bytes of each row), an SM takes in 90 bytes per ns, weights and tokens, a step of the
// ring is 250 ns at least, a tile's epilogue holds up the next one by some 0.15 us, a tail's own maps cost 1 us.  (16
// tokens, 4096 -> 2 x 14336 -> 4096, us for 1, 2, 4, 8 blocks per step in both products: 99, 72, 59.5, 63; 64 tokens with
// 1, 2, 4 in the first and 4 in the second: 74, 78, 90; one token through 2048 x 768: 17.2, 12.6, 9.8, 9.6; 1672 x 12720
// with one block per step and with more and a tail: 58, 31.)
inline double small_cost(const SmallShape &s, long long K, int block, int T)
{
    const double weights = (double)s.n * (s.rows / s.ct) * ((double)K / block * 128.0);
    const double chip = weights / (s.kbs == 1 ? 5900.0 : s.kbs == 2 ? 6100.0 : 6400.0);
    const double steps = (double)s.rounds * s.steps;
    const double sm = steps * (s.w_bytes + s.kbs * T * 128.0) / 90.0, issue = steps * 250.0;
    return ((chip > sm ? chip : sm) > issue ? (chip > sm ? chip : sm) : issue) / 1000.0 + 0.15 * s.rounds + (s.tail_at >= 0 ? 1.0 : 0.0);
}
inline SmallShape small_plan(int n, bool gated, long long K, int block, int T, int ctas)
{
    SmallShape best = small_shape(n, gated, K, block, T, ctas, 1);
    for (int kbs = 2; kbs <= 8 && kbs <= K / block && kbs * small_box(T, kbs, K % block != 0) <= 256; kbs *= 2) {
        const SmallShape s = small_shape(n, gated, K, block, T, ctas, kbs);
        if (small_cost(s, K, block, T) < small_cost(best, K, block, T)) best = s;
    }
    return best;
}

// ------------------------------------------------------------------------------------ the kernel

struct alignas(64) SmallProduct {
    CUtensorMap w;           // {K, rows, halves, 1} or {block, rows, halves, blocks}
    CUtensorMap x;           // {K, T, 1, copies} or {block, T, blocks, copies}
    CUtensorMap w_tail, x_tail;      // with a tail: the first forms
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
    int round_local;         // every CTA rounds all rows for itself, into a copy of its own
};

struct alignas(64) SmallArgs {
    SmallProduct p[2];
    FfnCtl *ctl;
    unsigned long long timeout_ns;
    int products, T;
    int withhold;            // test hook: this CTA never arrives at a grid barrier (-1: none)
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
// grid size per barrier and launch, so nothing has to be reset; what it will reach follows from any value of it that was
// read before the own arrival (`seen`).
__device__ __forceinline__ bool small_grid_barrier(unsigned long long *counter, unsigned long long seen, bool ok, bool withheld, const WaitCtx &wc,
                                                   int where)
{
    __threadfence();
    fence_proxy_async_global();          // ordinary stores here, tensor-map loads there
    ok = named_barrier_and<1, 256>(ok);
    if (ok && threadIdx.x == 128) {
        const unsigned long long g = gridDim.x, target = (seen / g + 1) * g;
        if (!withheld) red_release_add_u64(counter, 1ull);
        unsigned long long t0 = 0;
        unsigned it = 0;
        while (ld_acquire_u64(counter) < target) {
            __nanosleep(32);             // 148 of these loads at once would keep the last arrivals from the counter
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
    return named_barrier_and<1, 256>(ok);
}

// The epilogue warps round the tokens of a product: one row per CTA, or all rows into this CTA's own copy.
template <class X>
__device__ __noinline__ void small_round_rows(const X *src, const SmallProduct &p, int T, uint32_t *part)
{
    const int tid = threadIdx.x - 128;
    const size_t copy = p.round_local ? (size_t)blockIdx.x * T : 0;
    for (int row = p.round_local ? 0 : blockIdx.x; row < T; row += p.round_local ? 1 : gridDim.x) {
        quant_row_by<X, 256, 8, true, true>(src, p.round_dst + copy * p.K, p.round_scale + copy, row, p.K, tid, part);
        named_barrier_sync<1, 256>();
    }
}

// a step's copies
template <bool kTail>
__device__ __forceinline__ void small_fill_weights(const SmallProduct &p, int k, int tail_at, int block, int col0, uint32_t dst, uint64_t *full)
{
    const SmallShape &s = p.s;
    if (kTail && k == tail_at) tma_fill(dst, &p.w_tail, s.full * block, col0, 0, 0, full, (uint32_t)(s.rows * 128));
    else tma_fill(dst, &p.w, s.kbs == 1 ? k * block : 0, col0, 0, s.kbs == 1 ? 0 : k * s.kbs, full, (uint32_t)s.w_bytes);
}
template <bool kTail>
__device__ __forceinline__ void small_fill_tokens(const SmallProduct &p, int k, int tail_at, int block, int copy, uint32_t dst, uint64_t *full)
{
    const SmallShape &s = p.s;
    if (kTail && k == tail_at) tma_fill(dst, &p.x_tail, s.full * block, 0, 0, copy, full, (uint32_t)(s.box_t * 128));
    else tma_fill(dst, &p.x, s.kbs == 1 ? k * block : 0, 0, s.kbs == 1 ? 0 : k * s.kbs, copy, full, (uint32_t)s.x_bytes);
}

template <bool kI8>
__device__ __forceinline__ float small_value(uint32_t acc, float sx, float sw)
{
    return kI8 ? __int2float_rn((int)acc) * (sx * sw) : __uint_as_float(acc);
}

template <bool kI8>
__device__ __forceinline__ uint4 small_add(uint4 a, uint4 b)
{
    if constexpr (kI8) return make_uint4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w);
    else
        return make_uint4(__float_as_uint(__uint_as_float(a.x) + __uint_as_float(b.x)), __float_as_uint(__uint_as_float(a.y) + __uint_as_float(b.y)),
                          __float_as_uint(__uint_as_float(a.z) + __uint_as_float(b.z)), __float_as_uint(__uint_as_float(a.w) + __uint_as_float(b.w)));
}

// kTail: one of the products has a tail
template <bool kI8, bool kTail>
__global__ void __launch_bounds__(kSmallThreads, 1) weave_ffn_small_kernel(const __grid_constant__ SmallArgs a)
{
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *const behind = smem_raw + (smem - smem_u32(smem_raw)) + kSmallRing;
    SmallBars &bars = *reinterpret_cast<SmallBars *>(behind + 2 * kSmallRed);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const WaitCtx wc = {a.ctl, a.timeout_ns};
    constexpr int kBlock = kI8 ? 128 : 64;

    int ahead = 0;           // steps of the first product whose weights are on their way before anything else is set up
    if (warp == 0) {
        if (lane < kSmallMaxSlots) {
#pragma unroll
            for (int j = 0; j < 2; ++j) { mbar_init(&bars.full[j][lane], 2); mbar_init(&bars.empty[j][lane], 1); }
        } else if (lane < kSmallMaxSlots + 2) {
            const int i = lane - kSmallMaxSlots;
            mbar_init(&bars.acc_full[i], 1);
            mbar_init(&bars.acc_empty[i], 8);
            mbar_init(&bars.tokens[i], 1);
        }
        fence_mbar_init();
        fence_proxy_async_shared();
        __syncwarp();
        const SmallShape &s = a.p[0].s;
        const int col0 = blockIdx.x * s.rounds * s.ct;
        // (not in front of tokens that every CTA rounds itself: their loads would come behind the weights)
        if (col0 < s.n && !(kI8 && a.p[0].round_local)) ahead = min(s.slots, s.steps);
        for (int k = 0; k < ahead; ++k) small_fill_weights<kTail>(a.p[0], k, s.tail_at, kBlock, col0, smem + k * s.slot_bytes, &bars.full[0][k]);
    }
    if (warp == 2) { tmem_alloc_one(&bars.tmem_base, (uint32_t)a.tmem_cols); tmem_relinquish_one(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars.tmem_base;

    bool ok = true;
    if (warp < 2) {
        // ---- producers: warp 0 the weights, warp 1 the tokens
        const bool weights = warp == 0;
#pragma unroll          // both products' parameters at fixed places of the constant bank
        for (int i = 0; i < 2; ++i) {
            if (i >= a.products || !ok) break;
            const SmallProduct &p = a.p[i];
            const int before = i > 0 ? small_steps(a.p[0].s) : 0, start = i > 0 ? small_first_slot(a.p[0].s, p.s, before) : 0;
            const int turns = i > 0 ? before / a.p[0].s.slots : 0, rest = i > 0 ? before % a.p[0].s.slots : 0;
            int n = i == 0 ? ahead : 0, slot = start + n;
            uint32_t ph = 0;
            if (i == 0 && slot == p.s.slots) { slot = 0; ph = 1u; }
            if (lane == 0) tma_prefetch_desc(weights ? &p.w : &p.x);
            if (!weights && (i > 0 || (kI8 && p.round_src))) {
                ok = __all_sync(0xffffffffu, ffn_wait(&bars.tokens[i], 0, wc, 20 + i));
                fence_proxy_async_global();
            }
            const int copy = p.round_local ? (int)blockIdx.x : 0, tail_at = p.s.tail_at;
            for (int r = 0; r < p.s.rounds && ok; ++r) {
                const int col0 = (blockIdx.x * p.s.rounds + r) * p.s.ct;
                if (col0 >= p.s.n) break;
                for (int k = i == 0 && r == 0 ? ahead : 0; k < p.s.steps; ++k) {
                    bool there = true;
                    if (i == 0 || n >= p.s.slots) {
                        there = ffn_wait(&bars.empty[i][slot], ph ^ 1u, wc, 22 + (int)weights);
                    } else if (weights) {
                        // first use of a slot: the newest step of the product before that lies in it.  (Tokens come
                        // behind the grid barrier, when all of those are done with.)
                        const SmallShape &o = a.p[0].s;
                        int j = min(o.slots - 1, ((slot + 1) * p.s.slot_bytes - 1) / o.slot_bytes);
                        if (j >= rest && slot * p.s.slot_bytes < rest * o.slot_bytes) j = rest - 1;
                        const int uses = turns + (j < rest ? 1 : 0);
                        if (uses > 0) there = ffn_wait(&bars.empty[0][j], (uint32_t)(uses - 1) & 1u, wc, 23);
                    }
                    ok = __all_sync(0xffffffffu, there);
                    if (!ok) break;
                    uint64_t *full = &bars.full[i][slot];
                    const uint32_t dst = smem + slot * p.s.slot_bytes;
                    if (weights) small_fill_weights<kTail>(p, k, tail_at, kBlock, col0, dst, full);
                    else small_fill_tokens<kTail>(p, k, tail_at, kBlock, copy, dst + p.s.x_offset, full);
                    ++n;
                    if (++slot == p.s.slots) slot = 0;
                    if (slot == start) ph ^= 1u;
                }
            }
        }
        if (!ok) ffn_linger();
    } else if (warp == 2) {
        int n = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (i >= a.products || !ok) break;
            const SmallShape &s = a.p[i].s;
            const int start = i > 0 ? small_first_slot(a.p[0].s, s, small_steps(a.p[0].s)) : 0;
            int slot = start;
            uint32_t ph = 0;
            const uint32_t idesc = kI8 ? umma_idesc_i8(128, s.kbs * s.box_t) : umma_idesc_bf16(128, s.kbs * s.box_t);
            const int tail_at = s.tail_at;
            // the first block's columns alone: what lies in the other blocks' places is not this step's
            const uint32_t idesc_tail = kI8 ? umma_idesc_i8(128, s.box_t) : umma_idesc_bf16(128, s.box_t);
            for (int r = 0; r < s.rounds && ok; ++r, ++n) {
                if ((blockIdx.x * s.rounds + r) * s.ct >= s.n) break;
                const int buf = n & 1;
                ok = __all_sync(0xffffffffu, ffn_wait(&bars.acc_empty[buf], ((n >> 1) & 1) ^ 1, wc, 24));
                tc_fence_after();
                for (int k = 0; k < s.steps && ok; ++k) {
                    ok = __all_sync(0xffffffffu, ffn_wait(&bars.full[i][slot], ph, wc, 25));
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t w = smem + slot * s.slot_bytes;
                    ffn_mma_kstep_one<kI8>(tmem + (uint32_t)(buf * a.acc_cols), umma_desc_sw128(w), umma_desc_sw128(w + s.x_offset),
                                           kTail && k == tail_at ? idesc_tail : idesc,
                                           (uint32_t)(k != 0), &bars.empty[i][slot]);
                    if (++slot == s.slots) slot = 0;
                    if (slot == start) ph ^= 1u;
                }
                if (ok) tc_commit_one(&bars.acc_full[buf]);
            }
        }
        if (!ok) ffn_linger();
    } else if (warp >= 4) {
        // ---- epilogue: two groups of four warps take turns in blocks of eight tokens; a warp reads the accumulator
        // lanes of its number mod 4
        const int quarter = warp & 3, group = (warp - 4) >> 2, tid = threadIdx.x - 128 - group * 128;
        const int acc_row = quarter * 32 + lane;
        uint32_t *const red = reinterpret_cast<uint32_t *>(behind + group * kSmallRed);
        const bool withheld = (int)blockIdx.x == a.withhold;
        unsigned long long seen[3] = {0, 0, 0};
        if (threadIdx.x == 128)
#pragma unroll
            for (int j = 0; j < 3; ++j) seen[j] = ld_relaxed_u64(&a.ctl->barrier[j]);
        int n = 0;
#pragma unroll 1        // the second product finds these instructions in the cache
        for (int i = 0; i < a.products && ok; ++i) {
            const SmallProduct &p = a.p[i];
            const SmallShape s = p.s;
            const bool gate = p.gated, out_f32 = p.out_f32;
            if (i > 0) ok = small_grid_barrier(&a.ctl->barrier[0], seen[0], ok, withheld, wc, 26);
            if constexpr (kI8) {
                if (ok && p.round_src) {
                    if (p.round_f32) small_round_rows(static_cast<const float *>(p.round_src), p, a.T, bars.row_max);
                    else small_round_rows(static_cast<const __nv_bfloat16 *>(p.round_src), p, a.T, bars.row_max);
                    if (p.round_local) {
                        fence_proxy_async_global();
                        named_barrier_sync<1, 256>();
                    } else {
                        ok = small_grid_barrier(&a.ctl->barrier[1 + i], i == 0 ? seen[1] : seen[2], ok, withheld, wc, 27);
                    }
                }
            }
            if (!ok) break;
            if (threadIdx.x == 128) mbar_arrive(&bars.tokens[i]);
            if constexpr (kI8) {
                // (read behind the barriers in the tile's loop)
                const float *scales = p.row_scale + (p.round_local ? (size_t)blockIdx.x * a.T : 0);
                for (int t = threadIdx.x - 128; t < a.T; t += 256) bars.row_scale[t] = __ldcg(scales + t);
            }
            const int blocks_from = quarter * 32 / s.rows, blocks_to = min(s.kbs - 1, (quarter * 32 + 31) / s.rows), mine = acc_row / s.rows;
            for (int r = 0; r < s.rounds; ++r, ++n) {
                const int col0 = (blockIdx.x * s.rounds + r) * s.ct;
                if (col0 >= s.n) break;
                const int cols = min(s.ct, s.n - col0), buf = n & 1;
                // a thread has one or two items: a column of the tile and the first or second four of eight tokens
                float sw[2][2] = {{0.0f, 0.0f}, {0.0f, 0.0f}};
                if constexpr (kI8) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int item = tid + j * 128, c = item < s.ct ? item : item - s.ct;
                        if (c < cols) {
                            sw[j][0] = p.col_scale[col0 + c];
                            if (gate) sw[j][1] = p.col_scale[s.n + col0 + c];
                        }
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
                        uint4 *const to = reinterpret_cast<uint4 *>(red + acc_row * kSmallRedRow);
                        to[0] = make_uint4(v[0], v[1], v[2], v[3]);
                        to[1] = make_uint4(v[4], v[5], v[6], v[7]);
                    }
                    if (group == 0) named_barrier_sync<2, 128>();
                    else named_barrier_sync<3, 128>();
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int item = tid + j * 128, second = item >= s.ct, c = second ? item - s.ct : item, t = t0 + 4 * second;
                        if (c >= cols || t >= a.T) continue;
                        const uint4 *from = reinterpret_cast<const uint4 *>(red + c * kSmallRedRow) + second;
                        uint4 x = from[0], y = make_uint4(0, 0, 0, 0);
                        if (gate) y = from[s.ct * (kSmallRedRow / 4)];
#pragma unroll 1
                        for (int b = 1; b < s.kbs; ++b) {
                            from += s.rows * (kSmallRedRow / 4);
                            x = small_add<kI8>(x, from[0]);
                            if (gate) y = small_add<kI8>(y, from[s.ct * (kSmallRedRow / 4)]);
                        }
                        const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
                        const long long at = (long long)t * s.n + col0 + c;
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            if (t + q >= a.T) break;
                            const float sx = kI8 ? bars.row_scale[t + q] : 0.0f;
                            float f = small_value<kI8>(xs[q], sx, sw[j][0]);
                            if (gate) f = gated(f, small_value<kI8>(ys[q], sx, sw[j][1]));
                            if (out_f32) static_cast<float *>(p.out)[at + (long long)q * s.n] = f;
                            else static_cast<__nv_bfloat16 *>(p.out)[at + (long long)q * s.n] = __float2bfloat16_rn(f);
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
