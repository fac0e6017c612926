/* sdden.h -- C ABI of the target predictions D(y, k) used by the synthetic workloads.
 *
 * The method treats the target's drift as a black-box network (Sec. 3.1: the drift is given by a
 * trained network) that is evaluated on all drafted states of a window in one batched
 * call (Alg. "Speculative Sampling for DDM", the (Par.) line).  These are the stand-ins with a
 * plain definition; each maps rows X [R,d] with a per-row chain step krow [R] to out [R,d]:
 *
 *   gmm      E[x0 | x_t] of a diagonal-covariance Gaussian mixture (Bayes' rule over components)
 *   lowrank  E[x0 | x_t] of N(mu, U U^T + s2 I): two skinny fp32 GEMMs in the eigenbasis of
 *            U U^T with a per-row diagonal gain in between
 *   mlp      3-layer SiLU MLP on [x ; sinusoidal(k)], bf16 weights, fp32 accumulation (bf16 MFMA)
 *   mlp4     the same network with its matrices in 4 bits: a draft model of few bytes
 *   gated    pre-norm residual gated blocks, bf16 weights, fp32 residual stream
 *
 * and, below them, the layers these are made of as calls of their own, with the backward passes that fit them.
 *
 * Conventions as in sd.h: "dev" pointers are caller-owned device memory, "host" pointers are read
 * during the create call only.  Rows with krow < 0 or krow >= T are skipped: nothing is computed
 * for them and their output row is left untouched.  `alpha_bar_state` (host, length T+1) is the signal level of
 * chain state k: x = sqrt(ab) x0 + sqrt(1-ab) eps.  sdden_eval only enqueues kernels on `stream`.
 */
#ifndef SDDEN_H
#define SDDEN_H

#include <stddef.h>
#include <stdint.h>

#include "sd.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct sdden sdden;     /* opaque; owns device copies of its parameters and tables */

/* means, stds [M,d], logw [M] (log mixture weights), alpha_bar_state [T+1]: host. */
int sdden_gmm_create(int32_t M, int32_t d, const float* means, const float* stds,
                     const float* logw, int32_t T, const float* alpha_bar_state, sdden** out);

/* mu [d], U [d,r] row-major, alpha_bar_state [T+1]: host.  Builds the eigenbasis Q [d,r] of U U^T
 * and the per-step gain tables on the host in fp64. */
int sdden_lowrank_create(int32_t d, int32_t r, const float* mu, const float* U, float s2,
                         int32_t T, const float* alpha_bar_state, sdden** out);

/* W1 [(d+E),H], W2 [H,H], W3 [H,d]: bf16 bit patterns, row = input feature; b1,b2 [H], b3 [d]:
 * host.  Time embedding of width E: emb[i] = sin(k w_i), emb[E/2+i] = cos(k w_i),
 * w_i = 10000^(-2i/E); its product with the last E rows of W1 is folded into a per-step bias
 * table at create time.  Rmax: rows reserved right away (as by sdden_reserve).
 * d and H must be multiples of 256.  The denoiser keeps every weight twice on the device, 4 (2 d H + H H) bytes in all: in
 * the layout of the kernels for many rows and in that of the kernels for few. */
int sdden_mlp_create(int32_t d, int32_t H, int32_t E, const uint16_t* W1, const float* b1,
                     const uint16_t* W2, const float* b2, const uint16_t* W3, const float* b3,
                     int32_t T, int32_t Rmax, sdden** out);

/* The same network with W1's first d rows, W2 and W3 kept in 4 bits with one bf16 scale per `group` inputs of an output (group:
 * 32, 64 or a multiple of 128): scale = bf16(max |w| / 7), q = round(w / scale) + 8, quantised here from the bf16 weights; the
 * time embedding and the biases stay as they are.  Rows and activations are bf16 as in sdden_mlp_create.  Any d and H up to 2^20.
 * 4.1 to 4.5 bits per weight on the device.  Meant for the draft side of the independent drafter with few chains: a quarter of the
 * target's bytes, which is what calls of up to about 32 rows wait for; from 64 rows on the bf16 network is as fast or faster.
 * A prediction does not depend on the call it is part of.  Weights to be quantised that are not finite are refused (SD_ERR_ARG). */
int sdden_mlp4_create(int32_t d, int32_t H, int32_t E, int32_t group, const uint16_t* W1, const float* b1, const uint16_t* W2,
                      const float* b2, const uint16_t* W3, const float* b3, int32_t T, int32_t Rmax, sdden** out);

/* A network of residual gated blocks:  h_0 = x + be + emb(k) We,  h_{l+1} = h_l + FF_l(LN_l(h_l)),  D(x, k) = h_blocks, with the
 * layer norm and the gated block described further down.  We [E,d] bf16 (row = input feature), be [d]; norm_weight, norm_bias
 * [blocks,d] fp32; Wg, Wu [blocks,H,d] and Wd [blocks,d,H] bf16, row = OUTPUT feature: host.  d and H multiples of 8.  The
 * residual stream is fp32; the norm's output and the hidden rows are rounded to bf16. */
int sdden_gated_create(int32_t d, int32_t H, int32_t E, int32_t blocks, int32_t act, const uint16_t* We, const float* be,
                       const float* norm_weight, const float* norm_bias, float eps, const uint16_t* Wg, const uint16_t* Wu,
                       const uint16_t* Wd, int32_t T, int32_t Rmax, sdden** out);

/* Setup call: allocate the per-call scratch (row lists, intermediate activations) that
 * evaluations of up to Rmax rows need.  The gmm denoiser needs none; the others return
 * SD_ERR_WORKSPACE from sdden_eval when R exceeds what was reserved.  May be called again with a
 * larger Rmax (not while evaluations are in flight). */
int sdden_reserve(sdden* den, int32_t Rmax);

/* out[r] = D(X[r], krow[r]) for every r < R with 0 <= krow[r] < T.
 * X [R,d], krow [R], out [R,d]: dev, 16-byte aligned; X and out must not overlap.
 * Enqueues kernels on `stream` only: no allocation, no synchronisation. */
int sdden_eval(sdden* den, int32_t R, const float* X, const int32_t* krow, float* out,
               void* stream);

/* sdden_eval for a caller that also holds the rows as bf16 (bit patterns, round-to-nearest-even of
 * the same fp32 values; sd_draft can write this image next to the fp32 drafts, see
 * sd_set_draft_mirror in sd.h).  The MLP reads its first layer's input from Xbf16 and skips its
 * own conversion pass; the other denoisers ignore it.  Rows with krow < 0 need no valid image. */
int sdden_eval_mirror(sdden* den, int32_t R, const float* X, const uint16_t* Xbf16,
                      const int32_t* krow, float* out, void* stream);

/* The while-loop of the sampler for each chain in one launch, where the denoiser is cheap enough to be evaluated inside
 * the kernel that owns the chain (gmm with at most 64 components): windows back to back until step T, each
 * what (sdden_eval, sd_draft, sdden_eval, sd_verify, sd_advance) computes under the context's draft mode, carry rule,
 * temperature and seed.  Chains do not interact, so none waits for another's window; a window's positions are predicted
 * in order and only up to its first rejection.
 * in : y [B,d], n [B], chain_id [B]; draft_den: the draft network (EXPLICIT mode: the independent draft model), else
 *      ignored; D_frozen [B,d]: the carried prediction (FROZEN_REUSED), else ignored                         (dev)
 * out: out [*, d], row index = chain_id; B_active: dev int32, set to 0; counters: dev int64[5] or NULL, accumulated as in
 *      sd_advance (windows: those of the chain that needed most).  A chain handed over at step T leaves its state in
 *      `out` and counts one chain-window, as there.
 * SD_ERR_UNSUPPORTED, with nothing enqueued, when this denoiser (or draft_den) has no such form or fewer steps than
 * the chains, is being timed (sdden_profile) or runs under a device-resident count: the caller then makes the separate
 * calls.  Calls on one context must be ordered, as for sd_langevin_window. */
int sdden_run(sdden* den, sdden* draft_den, sd_ctx* ctx, int32_t B, const float* y, const int32_t* n,
              const int64_t* chain_id, const float* D_frozen, float* out, int32_t* B_active, int64_t* counters,
              void* stream);

/* Optional device-resident row limit: when `count` (dev int32) is set, only rows
 * r < min(R, *count * rows_per_chain) are evaluated, which lets a fixed launch sequence follow
 * the batch as sd_advance shrinks it (see sd_set_active_count).  NULL removes the limit. */
int sdden_set_active_count(sdden* den, const int32_t* count /*dev*/, int32_t rows_per_chain);

/* Measurement aid: time the `which`-th kernel of every following sdden_eval with HIP events on
 * the evaluation's stream (gmm: 1 = posterior mean; lowrank: 1, 2 = the two GEMMs; mlp, mlp4: 1..3 = the
 * three GEMMs; gated: 1 = the norms, 2, 3 = the blocks' first and last products; 0 = off, the default).  sdden_profile_collect waits for the recorded events, returns
 * the summed kernel time in ms and the number of timed launches, and starts a new collection.
 * Event objects are created on demand while profiling is on (never otherwise).
 * sdden_profile_min_rows restricts the timing to calls with R >= min_rows (default 0: every call),
 * e.g. to the batched evaluation of the drafted states rather than the window-start call. */
int sdden_profile(sdden* den, int32_t which);
int sdden_profile_min_rows(sdden* den, int32_t min_rows);
int sdden_profile_collect(sdden* den, double* total_ms, int64_t* launches);

/* Measurement aid (mlp only): which kernel serves the 256 x 256 GEMM tile of the batched call.
 * 0 = the default (alternating-phase kernel); 1 = the earlier hand-scheduled kernel, kept so that
 * the two can be timed side by side on the same data (results agree).  2, 3, 4 = the default
 * kernel with its fragment reads / its direct loads / both left out: TIMING ONLY, the results are
 * wrong -- they locate what bounds the kernel (4 = the MFMA and barrier schedule alone); 5 = the
 * default kernel without the fragment reads of the weight tile only (a third of its LDS reads),
 * TIMING ONLY as well. */
int sdden_mlp_select_gemm(sdden* den, int32_t variant);

int sdden_destroy(sdden* den);
/* Text of the last error of `den`, or with NULL of this thread's last call that had no denoiser (creates, layers, 4-bit matrices). */
const char* sdden_last_error(const sdden* den);

/* ---- Layers of row networks ------------------------------------------------------------------------------------------
 * What a denoiser of pre-norm residual blocks, h <- h + FF(LN(h)), is made of, forward for evaluating it and backward for
 * fitting it (or a draft model of it).  Plain calls without a handle: every buffer is the caller's device memory, kernels are
 * enqueued on `stream` only, nothing is allocated, synchronised or kept between calls, so any number may run at once on buffers
 * of their own, and all of them may be captured into a graph.  Matrices are row-major; a `*_stride` is the number of elements
 * between two rows.  Buffers must not overlap.  Errors: SD_ERR_* with the text in sdden_last_error(NULL), which is kept per
 * thread; nothing is enqueued then.  R = 0 is no error: no row is written, weight gradients become zero.  R <= 2^30. */
#define SDDEN_F32 0
#define SDDEN_BF16 1
#define SDDEN_SILU 0              /* f(g) = g / (1 + exp(-g))                                     */
#define SDDEN_GELU 1              /* f(g) = g P(g), P the normal distribution function            */

/* Layer norm:  y = (x - mean) rstd * weight + bias,  rstd = 1 / sqrt(mean((x - mean)^2) + eps), statistics in fp32.
 * x [R,d] of x_type, y [R,d] of y_type (any mix), weight and bias [d] fp32 or NULL (1 and 0), mean and rstd [R] fp32: both
 * written for the backward pass, or both NULL.  y keeps its digits in rows far from zero; the backward pass takes the mean as fp32 holds
 * it, so x - mean is off there by up to 2^-25 |mean|.  Any d from 1 to 2^30, any stride >= d, any alignment of the element type; 16-byte
 * accesses are used where d, the strides and the pointers allow them. */
int sdden_layernorm_forward(int32_t R, int32_t d, const void* x, int32_t x_type, int64_t x_stride, const float* weight,
                            const float* bias, float eps, void* y, int32_t y_type, int64_t y_stride, float* mean, float* rstd,
                            void* stream);

/* Its backward pass from dy [R,d] of dy_type and the forward pass's x, mean and rstd:
 *   dx = rstd (g - mean(g) - xh mean(g xh)) + dres,  g = dy * weight,  xh = (x - mean) rstd      (x_type)
 *   dweight = sum over rows dy xh,  dbias = sum over rows dy                                      (fp32 [d], each may be NULL)
 * dres [R,d] of x_type: a gradient added to dx (the one that reaches x around the block, on the residual path), or NULL.
 * workspace: sdden_layernorm_workspace_bytes(R, d) bytes where dweight or dbias is asked for, else NULL is enough.  Sums over rows
 * are taken in a fixed order: the same call gives the same bits. */
size_t sdden_layernorm_workspace_bytes(int32_t R, int32_t d);
int sdden_layernorm_backward(int32_t R, int32_t d, const void* dy, int32_t dy_type, int64_t dy_stride, const void* x, int32_t x_type,
                             int64_t x_stride, const float* weight, const float* mean, const float* rstd, const void* dres,
                             int64_t dres_stride, void* dx, int64_t dx_stride, float* dweight, float* dbias, void* workspace,
                             size_t workspace_bytes, void* stream);

/* Gated feed-forward block:  hidden = f(X Wg^T) * (X Wu^T),  Y = hidden Wd^T + res.
 * X [R,d], Wg and Wu [H,d], Wd [d,H], hidden [R,H]: bf16 bit patterns, the weights contiguous with one row per OUTPUT feature
 * (sdden_mlp_create takes its weights the other way round).  Y and res [R,d] of y_type with the same stride; res may be NULL.
 * hidden is scratch of an evaluation and an input of the backward pass; it is the one intermediate that is rounded to bf16,
 * as the second product takes it.  gates [2,R,H] fp32: g = X Wg^T and u = X Wu^T for the backward pass (kept in fp32, so that
 * gradients see no second rounding), or NULL.  d, H and the strides are multiples of 8 (16 bytes) up to 2^23; buffers are 16-byte
 * aligned. */
int sdden_gated_forward(int32_t R, int32_t d, int32_t H, int32_t act, const uint16_t* X, int64_t x_stride, const uint16_t* Wg,
                        const uint16_t* Wu, const uint16_t* Wd, const void* res, void* Y, int32_t y_type, int64_t y_stride,
                        uint16_t* hidden, float* gates, void* stream);

/* Its backward pass from dY [R,d] (bf16) and the forward pass's X, gates and hidden.  With dA = dY Wd, dG = dA u f'(g) and
 * dU = dA f(g), the last two rounded to bf16 for the products that take them:
 *   dX = dG Wg + dU Wu  (bf16 [R,d], or NULL);  dWg = dG^T X, dWu = dU^T X [H,d], dWd = dY^T hidden [d,H], of dw_type (all
 *   three, or all NULL).
 * The gradient of res is dY itself.  workspace: sdden_gated_workspace_bytes(R, d, H) bytes, 16-byte aligned. */
size_t sdden_gated_workspace_bytes(int32_t R, int32_t d, int32_t H);
int sdden_gated_backward(int32_t R, int32_t d, int32_t H, int32_t act, const uint16_t* dY, int64_t dy_stride, const uint16_t* X,
                         int64_t x_stride, const uint16_t* Wg, const uint16_t* Wu, const uint16_t* Wd, const float* gates,
                         const uint16_t* hidden, uint16_t* dX, int64_t dx_stride, void* dWg, void* dWu, void* dWd,
                         int32_t dw_type, void* workspace, size_t workspace_bytes, void* stream);


/* A matrix kept in 4 bits with one scale per group of inputs, and its product with rows:
 *   Y[r,n] = sum_k X[r,k] (q[n,k] - 8) scale[n, k / group]  (+ bias[n])
 * sdden_q4_create: q [N, ceil(K/2)] (row = output, two inputs per byte, the even one in the low half; values 0..15) and
 * scale [N, ceil(K/group)] bf16 bit patterns: host, read during the call, which lays the matrix out on the current device in the
 * kernels' order and waits for that.  group: 32, 64 or a multiple of 128 (K: one scale per row); N, K <= 2^20, any size.
 * sdden_q4_eval: X [R,K] and Y [R,N] of SDDEN_F32 or SDDEN_BF16 with any stride, bias [N] fp32 or NULL: dev, on the matrix's
 * device.  bf16 and fp32 rows enter exactly, an fp32 value as the sum of three bf16 ones (from |x| = 2^-103 on; of smaller values what
 * lies below 2^-126 may be lost).  Sums are fp32, the output is rounded once.  The sum of a group of inputs (a block of 128 of a
 * larger group) starts from -8 sum(x) and is scaled when it is complete, so 24 sum |x| over it has to stay below 2^128: it does
 * where |x| < 2^116; beyond that a result may be infinite or NaN although its value is not.  A row with an infinity or a NaN
 * gives NaN.  Sums are taken in one order for every R: a row's result does not depend on the call it is part of.  The handle is read only: any number of calls may use it at once, on any streams of its
 * device, also captured ones, as long as it lives.  Errors: text in sdden_last_error(NULL). */
typedef struct sdden_q4 sdden_q4;
int sdden_q4_create(int32_t N, int32_t K, int32_t group, const uint8_t* q, const uint16_t* scale, sdden_q4** out);
int sdden_q4_eval(const sdden_q4* m, int32_t R, const void* X, int32_t x_type, int64_t x_stride, const float* bias, void* Y,
                  int32_t y_type, int64_t y_stride, void* stream);
int sdden_q4_destroy(sdden_q4* m);

#ifdef __cplusplus
}
#endif
#endif /* SDDEN_H */
