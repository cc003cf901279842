/*
 * weave_ffn.h - C ABI of the dense gated feed-forward block (one expert of weave_moe.h without a router, or a model's
 * dense layers): its forward pass and its gradient in bf16, and its forward pass in 8-bit integers together with the
 * 8-bit matrix product and the rounding of rows that it is made of.
 *
 * The conventions are those of weave_moe.h: plain C, no exceptions, 0 = WEAVE_OK or a negative WEAVE_ERR_* code that
 * weave_moe_strerror() names; the caller owns every buffer (the library never allocates device memory) and keeps the
 * weights, their scales and the workspace alive until the handle is destroyed; device pointers belong to the device
 * that was current at creation, which has to be current in every call; matrices are row-major and dense, 16-byte
 * aligned; calls are asynchronous on the given stream and may be captured into a CUDA graph.
 *   - Calls on one handle use its one workspace: one at a time may be in flight, in the order of one stream or ordered
 *     by the caller.  That holds for replays of graphs that were captured from the same handle, too.
 *   - The weights may be changed between calls (by work that the stream orders before the next call); the handle keeps
 *     nothing computed from them.
 *   - An output must not overlap an input, a weight or its scales, another output or the workspace (WEAVE_ERR_INVALID_ARG).
 *   - T = 0 is allowed: no rows are read or written (a backward call then fills the weight gradients with zeros).
 */
#ifndef WEAVE_FFN_H
#define WEAVE_FFN_H

#include "weave_moe.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct weave_ffn *weave_ffn_t;

/* Types of matrix elements in the calls below. */
enum { WEAVE_BF16 = 0, WEAVE_F32 = 1, WEAVE_INT8 = 2 };

typedef struct weave_ffn_config {
    int hidden;          /* H: width of x and of the result; a multiple of 8 (WEAVE_INT8: of 16), at most 65536   */
    int ffn;             /* I: inner width, same rule                                                             */
    int max_tokens;      /* largest T of a call (sizes the workspace), at most 4194304                            */
    int weight_type;     /* WEAVE_BF16 or WEAVE_INT8                                                              */
    int backward;        /* 1 = weave_ffn_backward() may be called (WEAVE_BF16 only)                              */
    const void *gate_up; /* device [2I][H]: rows [0,I) gate projection (gets SiLU), rows [I,2I) up projection     */
    const void *down;    /* device [H][I]                                                                         */
    const float *gate_up_scale; /* WEAVE_INT8: device fp32 [2I], one scale per row; else NULL                     */
    const float *down_scale;    /* WEAVE_INT8: device fp32 [H]; else NULL                                         */
    void *workspace;     /* device scratch of at least weave_ffn_workspace_bytes(); 1024-byte aligned             */
    size_t workspace_bytes;
} weave_ffn_config;

/* Bytes of device scratch a handle with this config needs (pure host arithmetic on the five integers; 0 = bad shape): h for
 * max_tokens rows, [dg du] beside it for the gradient, and 9.25 MB for partial sums where a product may cut its K into parts
 * (max_tokens above 32 or the gradient, and H up to 4736 or I up to 2368). */
size_t weave_ffn_workspace_bytes(const weave_ffn_config *cfg);

/* Validates the config and zeroes the control words, behind all work given to the device before (synchronous, so not to be called
 * while a stream is being captured).  Tensor maps are encoded by each call, on the host: their boxes depend on T. */
int weave_ffn_create(const weave_ffn_config *cfg, weave_ffn_t *out_handle);

/* out[t] = Wd ( silu(Wg x[t]) (.) Wu x[t] ), x and out bf16 [T][H], 0 <= T <= max_tokens.
 * WEAVE_BF16: products are summed up in fp32, the gated product is rounded to bf16 (a relative 2^-8 of each value at
 * most), the result as well.
 * WEAVE_INT8: x is rounded to 8-bit integers with one scale per token (weave_int8_quantize()), so is the gated product
 * behind its rounding to bf16; sums of integer products are exact. */
int weave_ffn_forward(weave_ffn_t h, const void *x, void *out, int T, void *cuda_stream);

/* The gradients of x, gate_up and down for the gradient dy of out: dx bf16 [T][H], dgate_up bf16 [2I][H], ddown bf16
 * [H][I], all overwritten.  x is what the forward call was given; nothing else is kept between the two: the gate and up
 * projections are computed again, together with dy's product with down, in the kernel that needs them.  Each result is
 * a product of fp32 sums, rounded once; its operands h, d(gate) and d(up) are rounded to bf16 once before it. */
int weave_ffn_backward(weave_ffn_t h, const void *x, const void *dy, void *dx, void *dgate_up, void *ddown, int T,
                       void *cuda_stream);

/* Waits for all work on the device (graphs of the handle's calls may have been replayed on any stream), returns the device
 * status word (WEAVE_OK, or WEAVE_ERR_TIMEOUT if a bounded in-kernel wait gave up, after which results are undefined) and
 * clears it. */
int weave_ffn_status(weave_ffn_t h);
/* Upper bound in milliseconds for any single in-kernel wait (default 4000). */
int weave_ffn_set_timeout_ms(weave_ffn_t h, int ms);
/* Test hook: how a call of T tokens is carried out on a device of n_sm SMs (host arithmetic alone, by the routines that the
 * call itself uses; of the config the integers are read).  Writes up to max_products records, in the order of the products
 * (backward: dh; g and u; dx; dgate_up; ddown), and returns how many there are. */
typedef struct weave_ffn_product {
    int kernel;          /* 0 = on pairs of SMs, 1 = the one launch for up to 128 tokens                          */
    int mma_n;           /* N of its tensor-core products                                                        */
    int tail_n;          /* ... of those behind the last whole block of K, 0 where K has no such tail            */
    int width;           /* columns of the result in a tile                                                      */
    int parts;           /* parts of K summed up by different pairs                                              */
    int blocks;          /* blocks of K side by side in a step (kernel 1)                                        */
    int tiles;           /* kernel 0: of the result; kernel 1: of a thread block                                 */
    int mn_run, mn_atom; /* where B's N runs along its rows: elements of it in a CTA, and in a swizzle atom; else 0 */
} weave_ffn_product;
int weave_ffn_debug_plan(const weave_ffn_config *cfg, int backward, int T, int n_sm, weave_ffn_product *out, int max_products);
/* Test hook for the give-up paths (-1 = off, the default).  In the one launch for up to 128 tokens thread block `cta` never
 * arrives at a grid barrier, so that the bounded waits of all expire; in the launches on pairs of SMs the pair that it belongs to
 * waits for bytes that nobody sends.  The call ends with WEAVE_ERR_TIMEOUT; nothing faults or traps. */
int weave_ffn_debug_withhold_arrival(weave_ffn_t h, int cta);
int weave_ffn_last_cuda_error(weave_ffn_t h);
/* Releases host state.  Does not touch device memory. */
int weave_ffn_destroy(weave_ffn_t h);

/* ---- 8-bit integers with scales ------------------------------------------------------------- */

/* Rows to 8-bit integers: scale[r] = max|x[r]| / 127 in fp32, q[r][c] = the integer nearest to x[r][c] / scale[r]
 * (decided exactly, ties to even, within +-127).  x: device, x_type WEAVE_BF16 or WEAVE_F32, [rows][cols]; q: int8
 * [rows][cols]; scale: fp32 [rows]; cols from 1 to 16777216.
 * A row of zeros has scale 0 and zeros; a row with an inf or a NaN
 * has scale inf or NaN and zeros, so that what is computed from it is NaN.  Serves activations (rows = tokens) and
 * weights (rows = output channels).  No handle, no workspace. */
int weave_int8_quantize(const void *x, int x_type, int rows, int cols, void *q, float *scale, void *cuda_stream);

typedef struct weave_int8_linear *weave_int8_linear_t;

typedef struct weave_int8_linear_config {
    int in_features;     /* K: a multiple of 16, at most 65536 (sums stay below 2^31)                             */
    int out_features;    /* N: any number up to 4194304                                                           */
    int max_tokens;      /* largest T of a call, at most 4194304                                                  */
    const void *weight;  /* device int8 [N][K]                                                                    */
    const float *scale;  /* device fp32 [N]                                                                       */
    void *workspace;     /* device scratch of at least weave_int8_linear_workspace_bytes(); 1024-byte aligned     */
    size_t workspace_bytes;
} weave_int8_linear_config;

size_t weave_int8_linear_workspace_bytes(const weave_int8_linear_config *cfg);
int weave_int8_linear_create(const weave_int8_linear_config *cfg, weave_int8_linear_t *out_handle);

/* out[t][n] = (sum_k q[t][k] weight[n][k]) * (x_scale[t] * scale[n]): the sum in int32, exact; the two products in fp32;
 * out_type WEAVE_BF16 or WEAVE_F32, [T][N].
 * x_type WEAVE_INT8: x is q and x_scale its scales.  x_type WEAVE_BF16 or WEAVE_F32: x is rounded by
 * weave_int8_quantize()'s rule first, into the workspace, and x_scale is NULL. */
int weave_int8_linear_forward(weave_int8_linear_t h, const void *x, int x_type, const float *x_scale, void *out,
                              int out_type, int T, void *cuda_stream);
int weave_int8_linear_status(weave_int8_linear_t h);
int weave_int8_linear_set_timeout_ms(weave_int8_linear_t h, int ms);
/* Test hook: as weave_ffn_debug_plan(). */
int weave_int8_linear_debug_plan(const weave_int8_linear_config *cfg, int x_type, int T, int n_sm, weave_ffn_product *out,
                                 int max_products);
int weave_int8_linear_last_cuda_error(weave_int8_linear_t h);
int weave_int8_linear_destroy(weave_int8_linear_t h);

#ifdef __cplusplus
}
#endif
#endif /* WEAVE_FFN_H */
