// Host side of the dense feed-forward block and of the 8-bit product (include/weave_ffn.h): argument checks, tensor
// maps, the order of the launches.
#include "../../include/weave_ffn.h"

#include <cuda.h>
#include <cuda_runtime.h>
#include <string.h>
#include <new>

#include "weave_ffn_small.cuh"
#include "weave_gemm.cuh"
#include "weave_quant.cuh"

using namespace weave;

namespace {

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

constexpr int kMaxWidth = 65536;
constexpr int kMaxRows = 1 << 22;
constexpr int kMaxSms = 160;
constexpr int kMaxCols = 1 << 24;

size_t up1024(size_t n) { return (n + 1023) & ~(size_t)1023; }

// what both kinds of handle share
struct Engine {
    int device, n_sm;
    FfnCtl *ctl;
    uint32_t *partials;        // kGemmSplitBytes; null where no call splits K
    unsigned long long timeout_ns;
    int last_cuda_error;
    int withhold;              // weave_ffn_debug_withhold_arrival()
    EncodeTiledFn encode;
};

int cuda_fail(Engine &e, cudaError_t err)
{
    e.last_cuda_error = (int)err;
    (void)cudaGetLastError();       // reported here: not once more to whoever asks the runtime next
    return WEAVE_ERR_CUDA;
}

bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

struct Range { const void *p; size_t n; };
bool overlap(const Range &a, const Range &b)
{
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return a.n && b.n && x < y + b.n && y < x + a.n;
}
// none of the outputs may touch an input or another output
bool outputs_clear(const Range *out, int n_out, const Range *in, int n_in)
{
    for (int i = 0; i < n_out; ++i) {
        for (int j = 0; j < n_in; ++j)
            if (overlap(out[i], in[j])) return false;
        for (int j = i + 1; j < n_out; ++j)
            if (overlap(out[i], out[j])) return false;
    }
    return true;
}

template <int kEpi, bool kI8>
cudaError_t size_gemm()
{
    if constexpr (kEpi != kEpiGrad) {
        const cudaError_t err = cudaFuncSetAttribute(weave_gemm_kernel<kEpi, kI8, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kGemmSmemBytes);
        if (err != cudaSuccess) return err;
    }
    return cudaFuncSetAttribute(weave_gemm_kernel<kEpi, kI8, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kGemmSmemBytes);
}

template <bool kI8>
cudaError_t size_small()
{
    const cudaError_t err = cudaFuncSetAttribute(weave_ffn_small_kernel<kI8, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallSmemMax);
    return err != cudaSuccess ? err
                              : cudaFuncSetAttribute(weave_ffn_small_kernel<kI8, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallSmemMax);
}

int engine_create(Engine &e, void *workspace)
{
    cudaError_t err = cudaGetDevice(&e.device);
    if (err != cudaSuccess) return WEAVE_ERR_CUDA;
    int major = 0, smem = 0, sms = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, e.device) != cudaSuccess ||
        cudaDeviceGetAttribute(&smem, cudaDevAttrMaxSharedMemoryPerBlockOptin, e.device) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, e.device) != cudaSuccess)
        return WEAVE_ERR_CUDA;
    if (major != 10 || smem < kSmallSmemMax || sms < 2) return WEAVE_ERR_UNSUPPORTED_DEVICE;
    e.n_sm = (sms < kMaxSms ? sms : kMaxSms) & ~1;
    e.ctl = static_cast<FfnCtl *>(workspace);
    e.timeout_ns = 4000ull * 1000000ull;
    e.last_cuda_error = 0;
    e.withhold = -1;
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult res;
    err = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &res);
    if (err != cudaSuccess || !fn || res != cudaDriverEntryPointSuccess) return WEAVE_ERR_UNSUPPORTED_DEVICE;
    e.encode = reinterpret_cast<EncodeTiledFn>(fn);
    if ((err = size_gemm<kEpiStore, false>()) != cudaSuccess || (err = size_gemm<kEpiGated, false>()) != cudaSuccess ||
        (err = size_gemm<kEpiGrad, false>()) != cudaSuccess || (err = size_gemm<kEpiScaled, true>()) != cudaSuccess ||
        (err = size_gemm<kEpiScaledGated, true>()) != cudaSuccess || (err = size_small<false>()) != cudaSuccess ||
        (err = size_small<true>()) != cudaSuccess)
        return cuda_fail(e, err);
    return WEAVE_OK;
}

// Zeroes the control words, behind all work on the device that was given out before: an allocator may have made the workspace of
// memory that kernels in flight on some stream still write to.
int engine_clear(Engine &e, size_t bytes)
{
    cudaError_t err = cudaDeviceSynchronize();
    if (err == cudaSuccess) err = cudaMemset(e.ctl, 0, bytes);
    if (err == cudaSuccess) err = cudaDeviceSynchronize();
    return err == cudaSuccess ? WEAVE_OK : cuda_fail(e, err);
}

bool on_its_device(const Engine &e)
{
    int dev = -1;
    return cudaGetDevice(&dev) == cudaSuccess && dev == e.device;
}

// Behind all work on the device: a graph of the handle's calls may have been replayed on any stream.
int engine_status(Engine &e, size_t control_bytes)
{
    if (!on_its_device(e)) return WEAVE_ERR_INVALID_ARG;
    cudaError_t err = cudaDeviceSynchronize();
    if (err != cudaSuccess) return cuda_fail(e, err);
    int st = 0;
    err = cudaMemcpy(&st, &e.ctl->status, sizeof(st), cudaMemcpyDeviceToHost);
    if (err != cudaSuccess) return cuda_fail(e, err);
    if (st != 0) {
        const int rc = engine_clear(e, control_bytes);
        if (rc) return rc;
    }
    return st;
}

// [rows][cols] row-major, rows `pitch` elements apart (0: cols), box of box_cols x box_rows
bool map_2d(const Engine &e, CUtensorMap &m, int type, const void *p, long long rows, long long cols, int box_rows, int box_cols,
            long long pitch = 0, CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B)
{
    const int size = type == WEAVE_BF16 ? 2 : type == WEAVE_F32 ? 4 : 1;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)(pitch ? pitch : cols) * size};
    const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows};
    const cuuint32_t ones[2] = {1, 1};
    const CUtensorMapDataType dt = type == WEAVE_BF16  ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                   : type == WEAVE_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                                       : CU_TENSOR_MAP_DATA_TYPE_UINT8;
    return e.encode(&m, dt, 2, const_cast<void *>(p), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                    CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// operand whose K runs along the rows' elements: some rows x 128 bytes
bool map_k(const Engine &e, CUtensorMap &m, int type, const void *p, long long rows, long long cols, int box_rows = 128, long long pitch = 0)
{
    return map_2d(e, m, type, p, rows, cols, box_rows, type == WEAVE_INT8 ? 128 : 64, pitch);
}
// operand whose K runs across the rows (bf16), of which a CTA takes `run` elements along them: boxes of one swizzle atom x 64 rows
constexpr int mn_atom(int run) { return run % 64 == 0 ? 64 : 32; }
bool map_mn(const Engine &e, CUtensorMap &m, const void *p, long long rows, long long cols, int run, long long pitch = 0)
{
    return map_2d(e, m, WEAVE_BF16, p, rows, cols, 64, mn_atom(run), pitch,
                  mn_atom(run) == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
}

// kBehind: launched while the launch before it in the stream, one of the same call, still runs (see pdl_wait())
enum LaunchKind { kPlain, kBehind, kCooperative };
template <class... Params, class... Args>
cudaError_t launch(void (*kernel)(Params...), int grid, int block, size_t smem, LaunchKind kind, cudaStream_t stream, const Args &...args)
{
    cudaLaunchAttribute at;
    if (kind == kCooperative) {
        at.id = cudaLaunchAttributeCooperative;
        at.val.cooperative = 1;
    } else {
        at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at.val.programmaticStreamSerializationAllowed = 1;
    }
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(grid);
    lc.blockDim = dim3(block);
    lc.dynamicSmemBytes = smem;
    lc.stream = stream;
    lc.attrs = &at;
    lc.numAttrs = kind == kPlain ? 0 : 1;
    return cudaLaunchKernelEx(&lc, kernel, args...);
}

// Which kernel takes a call of up to kSmallMaxT tokens: the one whose modelled time is shorter, the products' cost and what
// else was measured of each.  (us, one launch against pairs of SMs: bf16 2048 x 768: 10.1 / 16.3 with 16 tokens, 16.4 / 16.8
// with 64, 18.6 / 16.2 with 96; 4096 x 14336: 76 / 92 with 64, 82 / 93 with 96; 8 bits 2048 x 1408: 16.6 / 18.3 with 16,
// 21.6 / 18.4 with 64; 4096 x 14336: 52 / 58 with 64, 61 / 59 with 128.  The pairs' launches take the host some 3 us each.)
bool small_wins(int T, int products, bool rounds, double small_us, double pairs_us)
{
    const double small_rest = 1.0 + products * (rounds ? 6.0 : 3.0) + products * 0.033 * T, pairs_rest = products * (rounds ? 7.0 : 4.0);
    return small_rest + small_us <= pairs_rest + pairs_us;
}
double small_us(const Engine &e, int n, bool gated, long long K, int block, int T)
{
    return small_cost(small_plan(n, gated, K, block, T, e.n_sm), K, block, T);
}

// The first product of a, or the next one: its plan and its tensor maps.  x: what the product reads, [copies][T][K].
bool small_product(const Engine &e, SmallArgs &a, int type, const void *w, const void *x, int n, bool gated, int K, int T, const float *row_scale,
                   const float *col_scale, void *out, bool out_f32, int copies)
{
    SmallProduct &p = a.p[a.products++];
    const int size = type == WEAVE_INT8 ? 1 : 2, block = 128 / size;
    p.s = small_plan(n, gated, K, block, T, e.n_sm);
    p.gated = gated;
    p.out_f32 = out_f32;
    p.row_scale = row_scale;
    p.col_scale = col_scale;
    p.out = out;
    p.round_src = nullptr;
    p.round_local = copies > 1;
    p.K = K;
    // with several blocks of K per step they are a dimension of the maps; with one, and behind the last whole block, K is the
    // first dimension, clipped at its end
    const CUtensorMapDataType dt = size == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    const cuuint64_t row = (cuuint64_t)K * size;
    const cuuint32_t ones[4] = {1, 1, 1, 1};
    const auto maps = [&](CUtensorMap &mw, CUtensorMap &mx, bool blocks) {
        const cuuint64_t inner = blocks ? (cuuint64_t)block : (cuuint64_t)K, count = blocks ? (cuuint64_t)p.s.full : 1;
        const cuuint32_t kbs = blocks ? (cuuint32_t)p.s.kbs : 1u;
        const cuuint64_t wd[4] = {inner, (cuuint64_t)n, gated ? 2u : 1u, count}, ws[3] = {row, row * (cuuint64_t)n, 128};
        const cuuint32_t wb[4] = {(cuuint32_t)block, (cuuint32_t)p.s.ct, gated ? 2u : 1u, kbs};
        const cuuint64_t xd[4] = {inner, (cuuint64_t)T, count, (cuuint64_t)copies}, xs[3] = {row, 128, row * (cuuint64_t)T};
        const cuuint32_t xb[4] = {(cuuint32_t)block, (cuuint32_t)p.s.box_t, kbs, 1};
        return e.encode(&mw, dt, 4, const_cast<void *>(w), wd, ws, wb, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS &&
               e.encode(&mx, dt, 4, const_cast<void *>(x), xd, xs, xb, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    };
    return maps(p.w, p.x, p.s.kbs > 1) && (p.s.tail_at < 0 || maps(p.w_tail, p.x_tail, false));
}
// Up to two tokens every CTA rounds for itself, 1.4 us each; from three on one row per CTA and a grid barrier behind them
// (3 to 4 us while the ring fills) take less.
constexpr int kSmallLocalT = 2, kSmallLocalK = 16384;
int small_copies(const Engine &e, int T, int K) { return T <= kSmallLocalT && K <= kSmallLocalK ? e.n_sm : 1; }
// scratch for the integers of a first product's tokens, and for their scales
size_t small_round_bytes(int max_tokens, int K)
{
    const size_t all = (size_t)max_tokens * K;
    const size_t copies = K <= kSmallLocalK ? (size_t)kMaxSms * (max_tokens < kSmallLocalT ? max_tokens : kSmallLocalT) * K : 0;
    return all > copies ? all : copies;
}
size_t small_round_scales(int max_tokens)
{
    const size_t copies = (size_t)kMaxSms * kSmallLocalT;
    return ((size_t)max_tokens > copies ? (size_t)max_tokens : copies) * 4;
}

// tokens that the kernel rounds to integers before the product made last
void small_round(SmallArgs &a, const void *src, int src_type, int8_t *dst, float *scale)
{
    SmallProduct &p = a.p[a.products - 1];
    p.round_src = src;
    p.round_dst = dst;
    p.round_scale = scale;
    p.round_f32 = src_type == WEAVE_F32;
}

template <bool kI8>
cudaError_t launch_small(const Engine &e, SmallArgs &a, int T, cudaStream_t stream)
{
    a.ctl = e.ctl;
    a.timeout_ns = e.timeout_ns;
    a.withhold = e.withhold;
    a.T = T;
    a.acc_cols = 0;
    bool tail = false;
    for (int i = 0; i < a.products; ++i) {
        tail = tail || a.p[i].s.tail_at >= 0;
        const int cols = a.p[i].s.kbs * a.p[i].s.box_t;
        a.acc_cols = cols > a.acc_cols ? cols : a.acc_cols;
    }
    for (a.tmem_cols = 32; a.tmem_cols < 2 * a.acc_cols;) a.tmem_cols *= 2;
    return launch(tail ? weave_ffn_small_kernel<kI8, true> : weave_ffn_small_kernel<kI8, false>, e.n_sm, kSmallThreads, kSmallSmemMax, kCooperative,
                  stream, a);
}

// Columns of a tile (a multiple of `unit`; each takes `columns` of the accumulator's): as narrow as the number of waves
// over the pairs of SMs allows, and rather more waves of narrower tiles than idle pairs.  A k-step takes the time of its
// bytes into an SM (94 per ns: 0.35 us for 32 KB), 0.2 us at least; a tile's epilogue is hidden but for the last one's.
constexpr int kSplitMinT = 32;
double gemm_tile_us(int ksteps, int accumulator_columns)
{
    const double bytes = kGemmHalf + accumulator_columns * 64.0, step = bytes / 94000.0 > 0.2 ? bytes / 94000.0 : 0.2;
    const double epilogue = 0.3 + 0.0055 * accumulator_columns;
    return ksteps * step > epilogue ? ksteps * step : epilogue;
}
long long gemm_tiles(int M, int N, int width) { return (long long)((M + 255) / 256) * ((N + width - 1) / width); }
// K is split over pairs where tiles are few and K is long: parts of at least eight steps, all of them in one wave.  (us
// whole / split: T = 128, 1016 x 14840: 62.5 / 36.9; T = 270: 72.1 / 50.5; 4096 x 14336: T = 128 92.7 / 82.1, T = 200 96.6 /
// 86.3; gradient T = 596, 264 x 8120: 71.9 / 47.1; 8 bits T = 257, 14336 -> 520: 28.4 / 17.7.  In the
// product with the activation: T = 128, 7168 x 2048: 36.3 / 31.2; T = 100, 8192 x 256: 29.3 / 20.9.)  Whoever adds the parts up
// needs a few round trips and reads them all.
double gemm_join_us(int splits, int width) { return 3.0 + splits * width * 512 / 36000.0; }
int gemm_splits(const Engine &e, long long tiles, int ksteps, int width)        // at most
{
    if (width > kGemmSplitWidth || !e.partials) return 1;
    const long long units = e.n_sm / 2 < kGemmSplitUnits ? e.n_sm / 2 : kGemmSplitUnits, s = units / tiles < ksteps / 8 ? units / tiles : ksteps / 8;
    return s < 1 ? 1 : (int)s;
}
// Workspace for it.  Up to 32 tokens the small batches' kernel leaves nothing to gain (within 1 % there), so that a handle for
// them, of which a model may have hundreds, stays small.
size_t gemm_split_room(long long columns, int ksteps, int max_tokens, bool backward)        // columns of accumulators
{
    const bool some = (max_tokens > kSplitMinT || backward) && ksteps >= 16 && 2 * ((columns + kGemmSplitWidth - 1) / kGemmSplitWidth) <= kGemmSplitUnits;
    return some ? kGemmSplitBytes : 0;
}
struct GemmWidth { int width, splits; double us; };
// N of a product on a pair of CTAs (M = 256) is a multiple of 16 in bf16 and of 32 in 8-bit integers, 256 at most.
constexpr int gemm_n_unit(bool i8) { return i8 ? 32 : 16; }
bool gemm_n_legal(bool i8, int n) { return n >= 32 && n <= 256 && n % gemm_n_unit(i8) == 0; }
// columns: of the accumulator, that a column of the result takes
GemmWidth gemm_width(const Engine &e, int M, int N, int ksteps, int widest, int unit, int columns, bool may_split)
{
    GemmWidth best = {widest, 1, 1e30};
    for (int w = widest; w * columns >= 64 && w > 0; w -= unit) {
        const long long tiles = gemm_tiles(M, N, w), pairs = e.n_sm / 2, waves = (tiles + pairs - 1) / pairs;
        const double end = 0.0055 * w * columns, us = waves * gemm_tile_us(ksteps, w * columns) + end;
        if (us < best.us) best = {w, 1, us};
        for (int s = may_split ? gemm_splits(e, tiles, ksteps, w * columns) : 1; s > 1; --s) {
            const double split_us = gemm_tile_us((ksteps + s - 1) / s, w * columns) + end + gemm_join_us(s, w * columns);
            if (split_us < best.us) best = {w, s, split_us};
        }
    }
    return best;
}
// ... of the long product in a launch with others, which fill the pairs that it leaves: the longer of its own waves and
// of all work spread evenly.  (Whole gradient, us with 256, 192, 128, 64 columns of dx in a tile: T = 257, 2048 x 1408: 35.5,
// 32.1, 30.7, 34.6; T = 777, 1096 x 2744: 66.5, 66.1, 67.0, 74.4.)  A join holds up the tiles behind it, too.
GemmWidth gemm_width_among(const Engine &e, int M, int N, int ksteps, double others_us)
{
    GemmWidth best = {256, 1, 1e30};
    const long long pairs = e.n_sm / 2;
    for (int w = 256; w >= 128; w /= 2) {        // (copies of an MN-major operand are 64 columns wide in each CTA)
        const long long tiles = gemm_tiles(M, N, w);
        for (int s = gemm_splits(e, tiles, ksteps, w); s > 0; --s) {
            const long long waves = (tiles * s + pairs - 1) / pairs;
            const double tile = gemm_tile_us((ksteps + s - 1) / s, w), even = (tiles * s * tile + others_us) / pairs;
            const double us = (waves * tile > even ? waves * tile : even) + (s > 1 ? 4.0 + gemm_join_us(s, w) : 0.0);
            if (us < best.us) best = {w, s, us};
        }
    }
    return best;
}

// How a forward call, and a gradient's two launches, are carried out.
struct ForwardPlan {
    bool small;
    GemmWidth up, down;
};
ForwardPlan plan_forward(const Engine &e, bool i8, int H, int I, int T)
{
    const int step = i8 ? 128 : 64, unit = gemm_n_unit(i8);
    ForwardPlan p;
    p.up = gemm_width(e, T, I, (H + step - 1) / step, 128, unit / 2, 2, T > kSplitMinT);
    p.down = gemm_width(e, T, H, (I + step - 1) / step, 256, unit, 1, T > kSplitMinT);
    p.small = T <= kSmallMaxT && small_wins(T, 2, i8, small_us(e, I, true, H, step, T) + small_us(e, H, false, I, step, T), p.up.us + p.down.us);
    return p;
}
struct LinearPlan {
    bool small;
    GemmWidth w;
};
LinearPlan plan_linear(const Engine &e, int K, int N, int T, bool rounds)
{
    LinearPlan p;
    p.w = gemm_width(e, T, N, (K + 127) / 128, 256, gemm_n_unit(true), 1, T > kSplitMinT);
    p.small = T <= kSmallMaxT && small_wins(T, 1, rounds, small_us(e, N, false, K, 128, T), p.w.us);
    return p;
}
struct BackwardPlan {
    int wide;            // of h, dg and du
    GemmWidth dx;
};
BackwardPlan plan_backward(const Engine &e, int H, int I, int T)
{
    BackwardPlan p;
    p.wide = gemm_width(e, T, I, (H + 63) / 64 * 3 / 2, 128, 64, 2, false).width;
    const double others = (gemm_tiles(2 * I, H, 256) + gemm_tiles(H, I, 256)) * gemm_tile_us((T + 63) / 64, 256);
    p.dx = gemm_width_among(e, T, H, (2 * I + 63) / 64, others);
    return p;
}

// Rows of A per CTA where A is K-major: those of the matrix spread evenly over its tiles.
int gemm_rows(int M)
{
    const int tiles = (M + 255) / 256;
    return (((M + 2 * tiles - 1) / (2 * tiles)) + 7) & ~7;
}

void gemm_job(GemmJob &j, int M, int N, long long K, int step, int width, bool a_mn, bool b_mn, void *out, long long ld, int splits = 1)
{
    j.M = M;
    j.splits = splits;
    j.N = N;
    j.ksteps = (int)((K + step - 1) / step);
    j.a_mn = a_mn;
    j.b_mn = b_mn;
    j.width = width;
    j.out = out;
    j.ld = ld;
    j.rows = a_mn ? 128 : gemm_rows(M);
    j.tiles_m = (M + 2 * j.rows - 1) / (2 * j.rows);
    j.tiles_n = (N + width - 1) / width;
    j.group_m = 8;
}

// jobs: of a.job; b_bytes: B's bytes of a k-step in one CTA, at most
template <int kEpi, bool kI8>
cudaError_t launch_gemm(const Engine &e, GemmArgs &a, int jobs, int b_bytes, LaunchKind kind, cudaStream_t stream)
{
    constexpr int columns = kEpi == kEpiGated || kEpi == kEpiGrad || kEpi == kEpiScaledGated ? 2 : 1;
    for (int i = 0; i < jobs; ++i)
        if (!gemm_n_legal(kI8, a.job[i].width * columns)) return cudaErrorInvalidValue;
    a.ctl = e.ctl;
    a.timeout_ns = e.timeout_ns;
    a.partials = e.partials;
    a.withhold = e.withhold < 0 ? ~0u : (unsigned)e.withhold & ~1u;
    a.a_bytes = 0;
    for (int i = 0; i < jobs; ++i) a.a_bytes = a.job[i].rows * 128 > a.a_bytes ? a.job[i].rows * 128 : a.a_bytes;
    a.stage_bytes = a.a_bytes + b_bytes;
    a.stages = kGemmRing / a.stage_bytes;
    if (a.stages > kGemmMaxStages) a.stages = kGemmMaxStages;
    const long long pairs = e.n_sm / 2;
    long long tiles = 0;
    for (int i = 0; i < jobs; ++i) tiles += (long long)a.job[i].tiles_m * a.job[i].tiles_n * a.job[i].splits;
    const int used = (int)(tiles < pairs ? tiles : pairs);
    a.extra = 0;
    if (kEpi == kEpiStore) {
        for (int i = jobs; i < 3; ++i) {
            a.job[i].tiles_m = a.job[i].tiles_n = 0;
            a.job[i].splits = 1;
        }
        if (jobs > 1) a.extra = (int)(gemm_tile_us(a.job[0].ksteps / a.job[0].splits, a.job[0].width) / gemm_tile_us(a.job[1].ksteps, a.job[1].width) + 0.5);
    }
    if constexpr (kEpi != kEpiGrad)
        if (a.job[0].splits > 1) return launch(weave_gemm_kernel<kEpi, kI8, true>, used * 2, kGemmThreads, kGemmSmemBytes, kind, stream, a);
    return launch(weave_gemm_kernel<kEpi, kI8, false>, used * 2, kGemmThreads, kGemmSmemBytes, kind, stream, a);
}

template <class X, int kThreads>
cudaError_t launch_quant_as(const void *x, int rows, int cols, int8_t *q, float *scale, LaunchKind kind, cudaStream_t stream)
{
    const bool vec = (long long)cols * (int)sizeof(X) % 16 == 0 && aligned(x, 16) && aligned(q, 16);
    return launch(vec ? weave_quant_kernel<X, kThreads, true> : weave_quant_kernel<X, kThreads, false>, rows, kThreads, 0, kind, stream,
                  static_cast<const X *>(x), q, scale, cols);
}
template <class X>
cudaError_t launch_quant_short(const void *x, int rows, int cols, int8_t *q, float *scale, LaunchKind kind, cudaStream_t stream)
{
    const bool vec = (long long)cols * (int)sizeof(X) % 16 == 0 && aligned(x, 16) && aligned(q, 16);
    return launch(vec ? weave_quant_short_kernel<X, true> : weave_quant_short_kernel<X, false>, (rows - 1) / 4 + 1, 128, 0, kind, stream,
                  static_cast<const X *>(x), q, scale, rows, cols);
}
template <class X>
cudaError_t launch_quant_rows(const void *x, int rows, int cols, int8_t *q, float *scale, LaunchKind kind, cudaStream_t stream)
{
    // threads with four to eight vectors each; few rows get many threads.  Many short rows: a warp each, four warps to a block.
    // (us, 64 threads in a block of their own / a warp: bf16 16384 x 512: 17.6 / 8.0; 9161 x 672: 10.2 / 6.1; 4096 x 2048: 6.3 /
    // 6.0; 2048 x 512: 2.9 / 2.5; but 2048 x 2048: 4.1 / 4.5, 1024 x 1024: 2.3 / 2.4.)
    const int vectors = cols / (int)(16 / sizeof(X));
    if ((vectors <= 128 && rows >= 2048) || (vectors <= 256 && rows >= 4096)) return launch_quant_short<X>(x, rows, cols, q, scale, kind, stream);
    if (vectors <= 512 && rows >= 1024) return launch_quant_as<X, 64>(x, rows, cols, q, scale, kind, stream);
    if (vectors <= 1024 && rows >= 512) return launch_quant_as<X, 128>(x, rows, cols, q, scale, kind, stream);
    return launch_quant_as<X, 256>(x, rows, cols, q, scale, kind, stream);
}
cudaError_t launch_quant(const void *x, int type, int rows, int cols, int8_t *q, float *scale, LaunchKind kind, cudaStream_t stream)
{
    return type == WEAVE_BF16 ? launch_quant_rows<__nv_bfloat16>(x, rows, cols, q, scale, kind, stream)
                              : launch_quant_rows<float>(x, rows, cols, q, scale, kind, stream);
}

// ---- the plans as weave_ffn_debug_plan() reports them

Engine engine_planned(int n_sm, size_t partial_bytes)
{
    Engine e = {};
    e.n_sm = (n_sm < kMaxSms ? n_sm : kMaxSms) & ~1;
    e.partials = partial_bytes ? reinterpret_cast<uint32_t *>(1024) : nullptr;      // only asked whether it is there
    return e;
}
struct Products {
    weave_ffn_product *out;
    int max, n;
    void put(const weave_ffn_product &p)
    {
        if (out && n < max) out[n] = p;
        ++n;
    }
    void small(const Engine &e, int columns, bool gated, long long K, int block, int T)
    {
        const SmallShape s = small_plan(columns, gated, K, block, T, e.n_sm);
        put({1, s.kbs * s.box_t, s.tail_at >= 0 ? s.box_t : 0, s.ct, 1, s.kbs, s.rounds, 0, 0});
    }
    void pairs(int M, int N, int width, int columns, int parts, bool b_mn)
    {
        put({0, width * columns, 0, width, parts, 1, (int)gemm_tiles(M, N, width), b_mn ? width * columns / 2 : 0, b_mn ? mn_atom(width * columns / 2) : 0});
    }
};

}  // namespace

// ------------------------------------------------------------------------------------ the block

namespace {
struct FfnLayout {
    size_t partials, partial_bytes, h, dgu, xq, x_scale, hq, h_scale, control, total;
};
bool ffn_shape_ok(const weave_ffn_config *c)
{
    if (!c || (c->weight_type != WEAVE_BF16 && c->weight_type != WEAVE_INT8)) return false;
    const int unit = c->weight_type == WEAVE_INT8 ? 16 : 8;
    return c->hidden > 0 && c->ffn > 0 && c->hidden % unit == 0 && c->ffn % unit == 0 && c->hidden <= kMaxWidth && c->ffn <= kMaxWidth &&
           c->max_tokens > 0 && c->max_tokens <= kMaxRows && (c->backward == 0 || (c->backward == 1 && c->weight_type == WEAVE_BF16));
}
// Rows of h and of [dg du] start on 128-byte lines: a copy's 128 bytes that straddle two take twice the requests (the
// gradient of T = 777, 1096 x 2744: 67 -> 64 us; were x and the weights aligned, too, 55).
long long line_pitch(long long cols) { return (cols + 63) / 64 * 64; }
FfnLayout ffn_layout(const weave_ffn_config *c)
{
    FfnLayout L;
    memset(&L, 0, sizeof(L));
    const size_t T = (size_t)c->max_tokens, I = (size_t)c->ffn;
    size_t at = up1024(sizeof(FfnCtl));
    L.control = at;
    L.partials = at;
    const int step = c->weight_type == WEAVE_INT8 ? 128 : 64;
    L.partial_bytes = gemm_split_room(c->hidden, (c->ffn * (c->backward ? 2 : 1) + step - 1) / step, c->max_tokens, c->backward);
    if (L.partial_bytes == 0) L.partial_bytes = gemm_split_room(2ll * c->ffn, (c->hidden + step - 1) / step, c->max_tokens, false);
    at += L.partial_bytes;
    L.h = at;
    at += up1024(T * (size_t)line_pitch(c->ffn) * 2);
    if (c->backward) {
        L.dgu = at;
        at += up1024(T * (size_t)line_pitch(2ll * c->ffn) * 2);
    }
    if (c->weight_type == WEAVE_INT8) {
        L.xq = at;
        at += up1024(small_round_bytes(c->max_tokens, c->hidden));
        L.x_scale = at;
        at += up1024(small_round_scales(c->max_tokens));
        L.hq = at;
        at += up1024(T * I);
        L.h_scale = at;
        at += up1024(T * 4);
    }
    L.total = at;
    return L;
}
}  // namespace

struct weave_ffn {
    Engine e;
    weave_ffn_config cfg;
    FfnLayout L;
    uint8_t *ws;
};

extern "C" {

size_t weave_ffn_workspace_bytes(const weave_ffn_config *cfg)
{
    return ffn_shape_ok(cfg) ? ffn_layout(cfg).total : 0;
}

int weave_ffn_create(const weave_ffn_config *cfg, weave_ffn_t *out)
{
    if (!out) return WEAVE_ERR_INVALID_ARG;
    *out = nullptr;
    if (!ffn_shape_ok(cfg) || !cfg->gate_up || !cfg->down || !cfg->workspace) return WEAVE_ERR_INVALID_ARG;
    if (!aligned(cfg->gate_up, 16) || !aligned(cfg->down, 16) || !aligned(cfg->workspace, 1024)) return WEAVE_ERR_INVALID_ARG;
    const bool i8 = cfg->weight_type == WEAVE_INT8;
    if (i8 != (cfg->gate_up_scale != nullptr) || i8 != (cfg->down_scale != nullptr)) return WEAVE_ERR_INVALID_ARG;
    if (!aligned(cfg->gate_up_scale, 4) || !aligned(cfg->down_scale, 4)) return WEAVE_ERR_INVALID_ARG;
    const FfnLayout L = ffn_layout(cfg);
    if (cfg->workspace_bytes < L.total) return WEAVE_ERR_WORKSPACE;
    weave_ffn *h = new (std::nothrow) weave_ffn();
    if (!h) return WEAVE_ERR_INVALID_ARG;
    h->cfg = *cfg;
    h->L = L;
    h->ws = static_cast<uint8_t *>(cfg->workspace);
    int rc = engine_create(h->e, cfg->workspace);
    h->e.partials = L.partial_bytes ? reinterpret_cast<uint32_t *>(h->ws + L.partials) : nullptr;
    if (rc == WEAVE_OK) rc = engine_clear(h->e, L.control);
    if (rc != WEAVE_OK) {
        delete h;
        return rc;
    }
    *out = h;
    return WEAVE_OK;
}

int weave_ffn_forward(weave_ffn_t h, const void *x, void *out, int T, void *cuda_stream)
{
    if (!h || T < 0 || T > h->cfg.max_tokens) return WEAVE_ERR_INVALID_ARG;
    if (T == 0) return WEAVE_OK;
    const int H = h->cfg.hidden, I = h->cfg.ffn;
    if (!x || !out || !aligned(x, 16) || !aligned(out, 16)) return WEAVE_ERR_INVALID_ARG;
    const size_t wsize = h->cfg.weight_type == WEAVE_INT8 ? 1 : 2, rows = (size_t)T * H * 2;
    const Range outs[1] = {{out, rows}};
    const bool i8 = h->cfg.weight_type == WEAVE_INT8;
    const Range ins[6] = {{x, rows}, {h->cfg.gate_up, (size_t)2 * I * H * wsize}, {h->cfg.down, (size_t)I * H * wsize}, {h->ws, h->L.total},
                          {h->cfg.gate_up_scale, i8 ? (size_t)2 * I * 4 : 0}, {h->cfg.down_scale, i8 ? (size_t)H * 4 : 0}};
    if (!outputs_clear(outs, 1, ins, 6) || !on_its_device(h->e)) return WEAVE_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    uint8_t *hbuf = h->ws + h->L.h;
    int8_t *xq = reinterpret_cast<int8_t *>(h->ws + h->L.xq), *hq = reinterpret_cast<int8_t *>(h->ws + h->L.hq);
    float *xs = reinterpret_cast<float *>(h->ws + h->L.x_scale), *hs = reinterpret_cast<float *>(h->ws + h->L.h_scale);
    const int type = i8 ? WEAVE_INT8 : WEAVE_BF16;
    const void *left = i8 ? static_cast<const void *>(xq) : x, *mid = i8 ? static_cast<const void *>(hq) : hbuf;
    cudaError_t err = cudaSuccess;
    const int step = i8 ? 128 : 64;
    const ForwardPlan plan = plan_forward(h->e, i8, H, I, T);
    if (plan.small) {
        SmallArgs a;
        a.products = 0;
        if (!small_product(h->e, a, type, h->cfg.gate_up, left, I, true, H, T, xs, h->cfg.gate_up_scale, hbuf, false,
                           i8 ? small_copies(h->e, T, H) : 1))
            return WEAVE_ERR_CUDA;
        if (i8) small_round(a, x, WEAVE_BF16, xq, xs);
        if (!small_product(h->e, a, type, h->cfg.down, mid, H, false, I, T, hs, h->cfg.down_scale, out, false, 1)) return WEAVE_ERR_CUDA;
        if (i8) small_round(a, hbuf, WEAVE_BF16, hq, hs);
        err = i8 ? launch_small<true>(h->e, a, T, stream) : launch_small<false>(h->e, a, T, stream);
        return err == cudaSuccess ? WEAVE_OK : cuda_fail(h->e, err);
    }
    // the wide products: gate and up with the activation, then down
    GemmArgs g, d;
    const int wide = plan.up.width, wide_d = plan.down.width;
    const uint8_t *up = static_cast<const uint8_t *>(h->cfg.gate_up) + (size_t)I * H * wsize;
    const long long pitch = i8 ? I : line_pitch(I);
    const int rows_a = gemm_rows(T);
    if (!map_k(h->e, g.job[0].a, type, left, T, H, rows_a) || !map_k(h->e, g.job[0].b[0], type, h->cfg.gate_up, I, H, wide) ||
        !map_k(h->e, g.job[0].b[1], type, up, I, H, wide) || !map_k(h->e, d.job[0].a, type, mid, T, I, rows_a, pitch) ||
        !map_k(h->e, d.job[0].b[0], type, h->cfg.down, H, I, wide_d / 2))
        return WEAVE_ERR_CUDA;
    gemm_job(g.job[0], T, I, H, step, wide, false, false, hbuf, pitch, plan.up.splits);
    gemm_job(d.job[0], T, H, I, step, wide_d, false, false, out, H, plan.down.splits);
    g.row_scale = xs;
    g.col_scale = h->cfg.gate_up_scale;
    d.job[0].b[1] = d.job[0].b[0];
    d.row_scale = hs;
    d.col_scale = h->cfg.down_scale;
    d.out_f32 = d.direct = 0;
    if (i8) {
        err = launch_quant(x, WEAVE_BF16, T, H, xq, xs, kPlain, stream);
        if (err == cudaSuccess) err = launch_gemm<kEpiScaledGated, true>(h->e, g, 1, wide * 128, kBehind, stream);
        if (err == cudaSuccess) err = launch_quant(hbuf, WEAVE_BF16, T, I, hq, hs, kBehind, stream);
        if (err == cudaSuccess) err = launch_gemm<kEpiScaled, true>(h->e, d, 1, wide_d * 64, kBehind, stream);
    } else {
        err = launch_gemm<kEpiGated, false>(h->e, g, 1, wide * 128, kPlain, stream);
        if (err == cudaSuccess) err = launch_gemm<kEpiStore, false>(h->e, d, 1, wide_d * 64, kBehind, stream);
    }
    return err == cudaSuccess ? WEAVE_OK : cuda_fail(h->e, err);
}

int weave_ffn_backward(weave_ffn_t h, const void *x, const void *dy, void *dx, void *dgate_up, void *ddown, int T, void *cuda_stream)
{
    if (!h || !h->cfg.backward || T < 0 || T > h->cfg.max_tokens) return WEAVE_ERR_INVALID_ARG;
    if (!dgate_up || !ddown || !aligned(dgate_up, 16) || !aligned(ddown, 16)) return WEAVE_ERR_INVALID_ARG;
    if (T > 0 && (!x || !dy || !dx || !aligned(x, 16) || !aligned(dy, 16) || !aligned(dx, 16))) return WEAVE_ERR_INVALID_ARG;
    const int H = h->cfg.hidden, I = h->cfg.ffn;
    const size_t rows = (size_t)T * H * 2, w_gu = (size_t)2 * I * H * 2, w_d = (size_t)I * H * 2;
    const Range outs[3] = {{dx, rows}, {dgate_up, w_gu}, {ddown, w_d}};
    const Range ins[5] = {{x, rows}, {dy, rows}, {h->cfg.gate_up, w_gu}, {h->cfg.down, w_d}, {h->ws, h->L.total}};
    if (!outputs_clear(outs, 3, ins, 5) || !on_its_device(h->e)) return WEAVE_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t err;
    if (T == 0) {
        err = cudaMemsetAsync(dgate_up, 0, w_gu, stream);
        if (err == cudaSuccess) err = cudaMemsetAsync(ddown, 0, w_d, stream);
        return err == cudaSuccess ? WEAVE_OK : cuda_fail(h->e, err);
    }
    uint8_t *hbuf = h->ws + h->L.h, *dgu = h->ws + h->L.dgu;
    // h and [dg du] from x and dy
    GemmArgs g;
    const BackwardPlan plan = plan_backward(h->e, H, I, T);
    const int wide = plan.wide;
    const uint8_t *up = static_cast<const uint8_t *>(h->cfg.gate_up) + (size_t)I * H * 2;
    const int rows_a = gemm_rows(T);
    const long long h_pitch = line_pitch(I), dgu_pitch = line_pitch(2ll * I);
    bool ok = map_k(h->e, g.job[0].a, WEAVE_BF16, dy, T, H, rows_a) && map_mn(h->e, g.job[0].b[0], h->cfg.down, H, I, wide / 2) &&
              map_k(h->e, g.job[1].a, WEAVE_BF16, x, T, H, rows_a) && map_k(h->e, g.job[1].b[0], WEAVE_BF16, h->cfg.gate_up, I, H, wide) &&
              map_k(h->e, g.job[1].b[1], WEAVE_BF16, up, I, H, wide);
    if (!ok) return WEAVE_ERR_CUDA;
    g.job[0].b[1] = g.job[0].b[0];
    // d(gate) and d(up) lie side by side in rows of 2I
    gemm_job(g.job[0], T, I, H, 64, wide, false, false, hbuf, h_pitch);
    gemm_job(g.job[1], T, I, H, 64, wide, false, false, dgu, dgu_pitch);
    gemm_job(g.job[2], T, I, H, 64, wide, false, false, dgu + (size_t)I * 2, dgu_pitch);
    err = launch_gemm<kEpiGrad, false>(h->e, g, 1, wide * 128, kPlain, stream);
    if (err != cudaSuccess) return cuda_fail(h->e, err);
    // dx = [dg du] W_gu, dW_gu = [dg du]^T x, dW_d = dy^T h: one launch, so that their last waves fill one another
    GemmArgs d;
    ok = map_k(h->e, d.job[0].a, WEAVE_BF16, dgu, T, 2ll * I, rows_a, dgu_pitch) && map_mn(h->e, d.job[0].b[0], h->cfg.gate_up, 2ll * I, H, plan.dx.width / 2) &&
         map_mn(h->e, d.job[1].a, dgu, T, 2ll * I, 128, dgu_pitch) && map_mn(h->e, d.job[1].b[0], x, T, H, 128) &&
         map_mn(h->e, d.job[2].a, dy, T, H, 128) && map_mn(h->e, d.job[2].b[0], hbuf, T, I, 128, h_pitch);
    if (!ok) return WEAVE_ERR_CUDA;
    for (int i = 0; i < 3; ++i) d.job[i].b[1] = d.job[i].b[0];
    gemm_job(d.job[0], T, H, 2ll * I, 64, plan.dx.width, false, true, dx, H, plan.dx.splits);
    gemm_job(d.job[1], 2 * I, H, T, 64, 256, true, true, dgate_up, H);
    gemm_job(d.job[2], H, I, T, 64, 256, true, true, ddown, I);
    err = launch_gemm<kEpiStore, false>(h->e, d, 3, kGemmHalf, kBehind, stream);
    return err == cudaSuccess ? WEAVE_OK : cuda_fail(h->e, err);
}

int weave_ffn_debug_plan(const weave_ffn_config *cfg, int backward, int T, int n_sm, weave_ffn_product *out, int max_products)
{
    if (!ffn_shape_ok(cfg) || T < 1 || T > cfg->max_tokens || n_sm < 2 || max_products < 0 || (backward && !cfg->backward)) return WEAVE_ERR_INVALID_ARG;
    const int H = cfg->hidden, I = cfg->ffn;
    const bool i8 = cfg->weight_type == WEAVE_INT8;
    const Engine e = engine_planned(n_sm, ffn_layout(cfg).partial_bytes);
    Products p = {out, max_products, 0};
    if (backward) {
        const BackwardPlan plan = plan_backward(e, H, I, T);
        p.pairs(T, I, plan.wide, 1, 1, true);        // dh
        p.pairs(T, I, plan.wide, 2, 1, false);       // g and u
        p.pairs(T, H, plan.dx.width, 1, plan.dx.splits, true);
        p.pairs(2 * I, H, 256, 1, 1, true);
        p.pairs(H, I, 256, 1, 1, true);
        return p.n;
    }
    const ForwardPlan plan = plan_forward(e, i8, H, I, T);
    if (plan.small) {
        p.small(e, I, true, H, i8 ? 128 : 64, T);
        p.small(e, H, false, I, i8 ? 128 : 64, T);
    } else {
        p.pairs(T, I, plan.up.width, 2, plan.up.splits, false);
        p.pairs(T, H, plan.down.width, 1, plan.down.splits, false);
    }
    return p.n;
}

int weave_ffn_status(weave_ffn_t h) { return h ? engine_status(h->e, h->L.control) : WEAVE_ERR_INVALID_ARG; }

int weave_ffn_set_timeout_ms(weave_ffn_t h, int ms)
{
    if (!h || ms <= 0) return WEAVE_ERR_INVALID_ARG;
    h->e.timeout_ns = (unsigned long long)ms * 1000000ull;
    return WEAVE_OK;
}

int weave_ffn_debug_withhold_arrival(weave_ffn_t h, int cta)
{
    if (!h || cta < -1) return WEAVE_ERR_INVALID_ARG;
    h->e.withhold = cta;
    return WEAVE_OK;
}

int weave_ffn_last_cuda_error(weave_ffn_t h) { return h ? h->e.last_cuda_error : 0; }

int weave_ffn_destroy(weave_ffn_t h)
{
    delete h;
    return WEAVE_OK;
}

}  // extern "C"

// ------------------------------------------------------------------------------------ 8-bit integers

namespace {
struct Int8Layout { size_t partials, partial_bytes, xq, x_scale, control, total; };
bool int8_shape_ok(const weave_int8_linear_config *c)
{
    return c && c->in_features > 0 && c->in_features % 16 == 0 && c->in_features <= kMaxWidth && c->out_features > 0 &&
           c->out_features <= kMaxRows && c->max_tokens > 0 && c->max_tokens <= kMaxRows;
}
Int8Layout int8_layout(const weave_int8_linear_config *c)
{
    Int8Layout L;
    size_t at = up1024(sizeof(FfnCtl));
    L.control = at;
    L.partials = at;
    L.partial_bytes = gemm_split_room(c->out_features, (c->in_features + 127) / 128, c->max_tokens, false);
    at += L.partial_bytes;
    L.xq = at;
    at += up1024(small_round_bytes(c->max_tokens, c->in_features));
    L.x_scale = at;
    at += up1024(small_round_scales(c->max_tokens));
    L.total = at;
    return L;
}
}  // namespace

struct weave_int8_linear {
    Engine e;
    weave_int8_linear_config cfg;
    Int8Layout L;
    uint8_t *ws;
};

extern "C" {

int weave_int8_quantize(const void *x, int x_type, int rows, int cols, void *q, float *scale, void *cuda_stream)
{
    if ((x_type != WEAVE_BF16 && x_type != WEAVE_F32) || rows < 0 || cols < 1 || cols > kMaxCols) return WEAVE_ERR_INVALID_ARG;
    if (rows == 0) return WEAVE_OK;
    const size_t size = x_type == WEAVE_BF16 ? 2 : 4, n = (size_t)rows * cols;
    if (!x || !q || !scale || !aligned(x, size) || !aligned(scale, 4)) return WEAVE_ERR_INVALID_ARG;
    const Range outs[2] = {{q, n}, {scale, (size_t)rows * 4}}, ins[1] = {{x, n * size}};
    if (!outputs_clear(outs, 2, ins, 1)) return WEAVE_ERR_INVALID_ARG;
    if (launch_quant(x, x_type, rows, cols, static_cast<int8_t *>(q), scale, kPlain, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess)
        return WEAVE_OK;
    (void)cudaGetLastError();
    return WEAVE_ERR_CUDA;
}

size_t weave_int8_linear_workspace_bytes(const weave_int8_linear_config *cfg)
{
    return int8_shape_ok(cfg) ? int8_layout(cfg).total : 0;
}

int weave_int8_linear_create(const weave_int8_linear_config *cfg, weave_int8_linear_t *out)
{
    if (!out) return WEAVE_ERR_INVALID_ARG;
    *out = nullptr;
    if (!int8_shape_ok(cfg) || !cfg->weight || !cfg->scale || !cfg->workspace) return WEAVE_ERR_INVALID_ARG;
    if (!aligned(cfg->weight, 16) || !aligned(cfg->scale, 4) || !aligned(cfg->workspace, 1024)) return WEAVE_ERR_INVALID_ARG;
    const Int8Layout L = int8_layout(cfg);
    if (cfg->workspace_bytes < L.total) return WEAVE_ERR_WORKSPACE;
    weave_int8_linear *h = new (std::nothrow) weave_int8_linear();
    if (!h) return WEAVE_ERR_INVALID_ARG;
    h->cfg = *cfg;
    h->L = L;
    h->ws = static_cast<uint8_t *>(cfg->workspace);
    int rc = engine_create(h->e, cfg->workspace);
    h->e.partials = L.partial_bytes ? reinterpret_cast<uint32_t *>(h->ws + L.partials) : nullptr;
    if (rc == WEAVE_OK) rc = engine_clear(h->e, L.control);
    if (rc != WEAVE_OK) {
        delete h;
        return rc;
    }
    *out = h;
    return WEAVE_OK;
}

int weave_int8_linear_forward(weave_int8_linear_t h, const void *x, int x_type, const float *x_scale, void *out, int out_type, int T,
                              void *cuda_stream)
{
    if (!h || T < 0 || T > h->cfg.max_tokens || (out_type != WEAVE_BF16 && out_type != WEAVE_F32) ||
        (x_type != WEAVE_BF16 && x_type != WEAVE_F32 && x_type != WEAVE_INT8) || (x_type == WEAVE_INT8) != (x_scale != nullptr))
        return WEAVE_ERR_INVALID_ARG;
    if (T == 0) return WEAVE_OK;
    if (!x || !out || !aligned(x, 16) || !aligned(out, 16) || !aligned(x_scale, 4)) return WEAVE_ERR_INVALID_ARG;
    const int K = h->cfg.in_features, N = h->cfg.out_features;
    const size_t out_size = out_type == WEAVE_F32 ? 4 : 2, x_size = x_type == WEAVE_INT8 ? 1 : x_type == WEAVE_BF16 ? 2 : 4;
    const Range outs[1] = {{out, (size_t)T * N * out_size}};
    const Range ins[5] = {{x, (size_t)T * K * x_size}, {x_scale, x_scale ? (size_t)T * 4 : 0}, {h->cfg.weight, (size_t)N * K},
                          {h->cfg.scale, (size_t)N * 4}, {h->ws, h->L.total}};
    if (!outputs_clear(outs, 1, ins, 5) || !on_its_device(h->e)) return WEAVE_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t err;
    int8_t *xq = reinterpret_cast<int8_t *>(h->ws + h->L.xq);
    float *xs = reinterpret_cast<float *>(h->ws + h->L.x_scale);
    const bool round = x_type != WEAVE_INT8;
    const void *q = round ? xq : x;
    if (round) x_scale = xs;
    const bool direct = (size_t)N * out_size % 16 != 0;
    const LinearPlan plan = plan_linear(h->e, K, N, T, round);
    if (plan.small) {
        SmallArgs a;
        a.products = 0;
        if (!small_product(h->e, a, WEAVE_INT8, h->cfg.weight, q, N, false, K, T, x_scale, h->cfg.scale, out, out_type == WEAVE_F32,
                           round ? small_copies(h->e, T, K) : 1))
            return WEAVE_ERR_CUDA;
        if (round) small_round(a, x, x_type, xq, xs);
        err = launch_small<true>(h->e, a, T, stream);
        return err == cudaSuccess ? WEAVE_OK : cuda_fail(h->e, err);
    }
    if (round) {
        err = launch_quant(x, x_type, T, K, xq, xs, kPlain, stream);
        if (err != cudaSuccess) return cuda_fail(h->e, err);
    }
    GemmArgs g;
    const int wide = plan.w.width;
    const int rows_a = gemm_rows(T);
    g.direct = direct;
    g.out_f32 = out_type == WEAVE_F32;
    g.row_scale = x_scale;
    g.col_scale = h->cfg.scale;
    if (!map_k(h->e, g.job[0].a, WEAVE_INT8, q, T, K, rows_a) || !map_k(h->e, g.job[0].b[0], WEAVE_INT8, h->cfg.weight, N, K, wide / 2)) return WEAVE_ERR_CUDA;
    g.job[0].b[1] = g.job[0].b[0];
    gemm_job(g.job[0], T, N, K, 128, wide, false, false, out, N, plan.w.splits);
    err = launch_gemm<kEpiScaled, true>(h->e, g, 1, wide * 64, round ? kBehind : kPlain, stream);
    return err == cudaSuccess ? WEAVE_OK : cuda_fail(h->e, err);
}

int weave_int8_linear_debug_plan(const weave_int8_linear_config *cfg, int x_type, int T, int n_sm, weave_ffn_product *out, int max_products)
{
    if (!int8_shape_ok(cfg) || (x_type != WEAVE_BF16 && x_type != WEAVE_F32 && x_type != WEAVE_INT8) || T < 1 || T > cfg->max_tokens ||
        n_sm < 2 || max_products < 0)
        return WEAVE_ERR_INVALID_ARG;
    const int K = cfg->in_features, N = cfg->out_features;
    const Engine e = engine_planned(n_sm, int8_layout(cfg).partial_bytes);
    Products p = {out, max_products, 0};
    const LinearPlan plan = plan_linear(e, K, N, T, x_type != WEAVE_INT8);
    if (plan.small) p.small(e, N, false, K, 128, T);
    else p.pairs(T, N, plan.w.width, 1, plan.w.splits, false);
    return p.n;
}

int weave_int8_linear_status(weave_int8_linear_t h) { return h ? engine_status(h->e, h->L.control) : WEAVE_ERR_INVALID_ARG; }

int weave_int8_linear_set_timeout_ms(weave_int8_linear_t h, int ms)
{
    if (!h || ms <= 0) return WEAVE_ERR_INVALID_ARG;
    h->e.timeout_ns = (unsigned long long)ms * 1000000ull;
    return WEAVE_OK;
}

int weave_int8_linear_last_cuda_error(weave_int8_linear_t h) { return h ? h->e.last_cuda_error : 0; }

int weave_int8_linear_destroy(weave_int8_linear_t h)
{
    delete h;
    return WEAVE_OK;
}

}  // extern "C"
