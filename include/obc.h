/*
 * libobc -- the layer-wise ExactOBS / OBQ solver of "Optimal Brain Compression"
 * (arxiv 2208.11580) for one AMD MI355X (gfx950).
 *
 * Problem (Sec. 3, eq. (2)): for a layer with weights W (d_row x d_col) and calibration
 * inputs X (d_col x N) find compressed weights W^ minimising ||W X - W^ X||^2 under a
 * sparsity or quantization constraint.  The path is
 *
 *     X --obc_hessian--> H = 2 X X^T + lambda I --obc_invert--> H^-1
 *       --obc_prune_rows / obc_quant_rows--> per-row order P, loss changes L, weights
 *       --obc_global_select--> per-row counts and layer mask
 *       --obc_gather_trace (from the pruning trace) or obc_reconstruct_rows (closed form)--> W^
 *
 * Conventions
 *  - Every array argument is a DEVICE pointer owned by the caller, row-major and
 *    contiguous unless a leading dimension is given.  `const` inputs are never written.
 *    The library allocates no large memory: scratch is a caller-provided workspace whose
 *    size comes from the matching *_workspace_bytes query (host call, no GPU work).
 *  - All work is enqueued on the HIP stream given to obc_create and is asynchronous with
 *    respect to the host, except obc_invert, obc_refit and obc_check, which wait for the stream,
 *    and obc_prune_rows / obc_quant_rows when given a live mask of more than 192 columns, which wait once
 *    at their start (the smallest number of already-pruned weights over the rows is read back).
 *  - Every call returns 0 (OBC_OK) or a negative OBC_ERR_* code; nothing throws or aborts
 *    across this boundary.  obc_last_error gives a text for the last failure on a context.
 *    Conditions only a kernel can see (a non-positive or non-finite pivot [H^-1]_pp) are
 *    latched on the device and reported by obc_check.
 *  - Results are deterministic: the same call on the same inputs gives bit-identical outputs.  (The two
 *    row-solver strategies round differently, and a workspace below the query makes OBC_STRATEGY_AUTO take
 *    the other one, see there.)
 *  - Matrices and results are fp32.  obc_invert, obc_refit and obc_reconstruct_rows factorise in fp64
 *    internally and round the result; the row solvers keep a row's weights and the diagonal of its
 *    inverse in fp64 and the matrix itself in fp32.
 */
#ifndef OBC_H
#define OBC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define OBC_OK 0
#define OBC_ERR_BAD_ARG (-1)   /* null pointer, negative size, value out of range */
#define OBC_ERR_BAD_SHAPE (-2) /* sizes inconsistent with each other (d % M != 0, k > d, ...) */
#define OBC_ERR_NOT_SPD (-3)   /* obc_invert met a non-positive Cholesky pivot */
#define OBC_ERR_WORKSPACE (-4) /* workspace missing or smaller than the query says (or than a row needs) */
#define OBC_ERR_NUMERIC (-5)   /* a row solver met a non-positive / non-finite [H^-1]_pp */
#define OBC_ERR_HIP (-6)       /* a HIP runtime call failed */

/* Row-solver strategies (argument `strategy` below).  AUTO picks the blocked solver up to
 * d_col = 4608 and the streamed rank-1 solver beyond (as far as its per-row vectors fit in LDS,
 * d_col <= ~5600; larger d_col returns OBC_ERR_BAD_SHAPE).  Where a row's matrix fits in LDS
 * (d_col <= ~190) AUTO needs no workspace: it takes the rank-1 solver when it is given less than the
 * query says (up to d_col = 64 the query says 256 bytes and the blocked solver needs none), or when
 * that would be more than 4 GiB. */
#define OBC_STRATEGY_AUTO 0
#define OBC_STRATEGY_RANK1 1   /* literal Algorithm 1: one rank-1 elimination per step */
#define OBC_STRATEGY_BLOCKED 2 /* same arithmetic result, eliminations applied in blocks */

typedef struct obc_ctx obc_ctx;

/* Create a context bound to `hip_stream` (a hipStream_t; NULL = the default stream) on the
 * current device.  The context owns only a few bytes of device memory (the error latch). */
int obc_create(obc_ctx **ctx, void *hip_stream);
int obc_destroy(obc_ctx *ctx);
const char *obc_last_error(const obc_ctx *ctx);
const char *obc_version(void);

/* Wait for the context's stream and return the first error a kernel latched since the last
 * obc_check (OBC_ERR_NUMERIC, OBC_ERR_NOT_SPD; OBC_ERR_BAD_ARG from obc_pack4, obc_distill, obc_score,
 * obc_embed, obc_embed_grad and obc_adamw) or
 * OBC_OK; clears the latch. */
int obc_check(obc_ctx *ctx);

/* ---- Measurement support (not part of the method) ---------------------------------------
 * Between obc_profile_begin and obc_profile_end every launch of the row solvers' kernels is
 * bracketed by HIP events on the context's stream.  obc_profile_end waits for the stream and
 * fills one obc_kernel_stat per kernel class: launches, summed duration, and the algorithmic
 * bytes / flops of those launches (what the method needs moved / computed under the schedule
 * the kernel implements: the flush reads and writes one triangle of the surviving m x m part of
 * each row's (symmetric) inverse once per block of B steps, or once for several such blocks above 2304
 * columns, 8 m(m+1)/2 bytes and m(m+1) flops per step per row; a panel reads one matrix row per step and
 * the vectors of the blocks since the last flush, 4 m bytes each; the rank-1 kernel moves 8 m^2 bytes
 * per step). */
#define OBC_KERNEL_PANEL 0
#define OBC_KERNEL_FLUSH 1
#define OBC_KERNEL_RANK1 2
#define OBC_KERNEL_CLASSES 3
typedef struct obc_kernel_stat {
    int launches;
    double ms;
    double bytes;
    double flops;
} obc_kernel_stat;
int obc_profile_begin(obc_ctx *ctx);
int obc_profile_end(obc_ctx *ctx, obc_kernel_stat stats[OBC_KERNEL_CLASSES]);

/* What this GPU's memory system gives the plainest kernels (16-byte accesses, every compute unit
 * busy): kind 0 reads `bytes` from src, 1 writes `bytes` to dst, 2 copies src to dst; streaming != 0
 * makes the stores non-temporal (as the row solver's matrix stores are).  Runs one warm-up pass and
 * `reps` timed passes on the context's stream, waits, and returns the mean milliseconds per pass:
 * the measured ceiling that HBM-bound kernels are compared with.  bytes must be a multiple of 16,
 * the buffers 16-byte aligned; for kind 0 the buffer must hold words whose lowest bit is clear
 * (e.g. all zero).  Synchronous. */
int obc_membench(obc_ctx *ctx, int kind, int streaming, const void *src, void *dst, size_t bytes,
                 int reps, double *ms_per_pass);

/* What the matrix cores of this GPU sustain on nothing but independent MFMA instructions, four
 * wavefronts on every SIMD: kind 0 = v_mfma_f32_32x32x2_f32 (the first flush's instruction; the others'
 * v_mfma_f32_4x4x1, of the same nominal rate, sustains 151 TFLOP/s where this one does 155), kind 1 =
 * v_mfma_f64_16x16x4_f64 (the factorisation's).  Every wavefront issues 4 * iters instructions per
 * pass; one warm-up pass and `reps` timed ones on the context's stream.  Returns the mean
 * milliseconds per pass and the flops of a pass.  Synchronous. */
int obc_mfmabench(obc_ctx *ctx, int kind, int iters, int reps, double *ms_per_pass, double *flops_per_pass);

/* ---- Sec. 4: H = 2 X X^T, "Implementation Details": dampening -------------------------
 * X: d x N fp32 with leading dimension ldx >= N (element (j, n) at X[j*ldx + n]).
 * H: d x d fp32.  accumulate == 0: H = 2 X X^T;  accumulate != 0: H += 2 X X^T (calibration
 * data arriving in batches; samples only ever need to be accumulated once).
 * damp_rel >= 0: after the product, add damp_rel * mean(diag(H)) to the diagonal (call with
 * damp_rel < 0 for all batches but the last).  The sum over samples is not divided by N.  A workspace
 * that is enough for N samples is enough for fewer (obc_cross likewise). */
int obc_hessian_workspace_bytes(int d, int64_t N, size_t *bytes);
int obc_hessian(obc_ctx *ctx, const float *X, int d, int64_t N, int64_t ldx, float damp_rel,
                int accumulate, float *H, void *ws, size_t ws_bytes);

/* ---- Sec. 4 Step 1: the inverse every row starts from ---------------------------------
 * In-place inverse of the symmetric positive definite d x d matrix H through its Cholesky
 * factor (fp64 inside, result rounded to fp32 and exactly symmetric).  Synchronous.
 * Returns OBC_ERR_NOT_SPD (H is then undefined) when a pivot is not positive. */
int obc_invert_workspace_bytes(int d, size_t *bytes);
int obc_invert(obc_ctx *ctx, float *H_inout, int d, void *ws, size_t ws_bytes);

/* ---- Algorithm 1 (+ N:M rule of Sec. 4) and Algorithm 3 --------------------------------
 * Workspace for obc_prune_rows / obc_quant_rows on R rows of width d. */
int obc_rows_workspace_bytes(int R, int d, int strategy, size_t *bytes);

/* Prune every row of W independently with Algorithm 1, each on a private copy of Hinv.
 *   W        R x d   weights (input)
 *   Hinv     d x d   symmetric inverse Hessian shared by all rows (input)
 *   k_steps  greedy steps per row, 0 <= k_steps <= d (N:M: <= d (M-N)/M)
 *   nm_n, nm_m   N:M pattern: a weight is eligible while its block of nm_m consecutive
 *            indices has fewer than nm_m - nm_n pruned weights; nm_m == 0: unstructured
 *   stop_counts  nullable, R: row i stops after min(k_steps, stop_counts[i]) steps (replay of
 *            the counts chosen by obc_global_select); entries of order/loss beyond are untouched
 *   live     nullable, R x d: 0 marks a weight that is already pruned (Sec. 4 "Implementation
 *            Details": an already sparse matrix is handled on the dense sub-problem of its
 *            non-zeros).  Those indices are first removed from the row's inverse (Lemma 1, no
 *            weight change, nothing recorded), keep weight 0, and the k_steps greedy steps run
 *            on the survivors (a row with fewer survivors stops when none is left; entries of
 *            order / loss beyond are untouched).  Not combined with the N:M rule.
 *   order    R x k_steps int32 out: index pruned at each step
 *   loss     R x k_steps fp32 out: loss change w_p^2 / (2 [H^-1]_pp) of each step
 *   W_out    R x d out: the row after its last step (pruned weights exactly 0)
 *   trace    nullable, R x k_steps x d out: the row after every step (the "pruning trace" of
 *            Sec. 4 Step 2, kept in HBM here); entries of steps a row does not take (stop_counts,
 *            fewer survivors than k_steps) are zero
 * Ties in the argmin go to the lowest index. */
int obc_prune_rows(obc_ctx *ctx, const float *W, const float *Hinv, int R, int d, int k_steps,
                   int nm_n, int nm_m, const int32_t *stop_counts, const uint8_t *live, int32_t *order,
                   float *loss, float *W_out, float *trace, int strategy, void *ws, size_t ws_bytes);

/* Block pruning (Sec. 4 "Block-Sparsity", eq. (5)): Algorithm 1 on blocks of c consecutive
 * weights (block b = indices b c .. b c + c - 1; d must be a multiple of c, 1 <= c <= 8).  Each
 * step takes the live block P with the smallest w_P^T ((H^-1)_P)^-1 w_P, moves the remaining
 * weights by -H^-1[:,P] ((H^-1)_P)^-1 w_P and removes P from the inverse (Lemma 1 for every p in
 * P).  Arguments as obc_prune_rows, counted in blocks:
 *   k_blocks     steps per row (<= d / c); stop_counts nullable, per-row step limits in blocks
 *   order, loss  R x k_blocks out: block index per step and its loss change
 *                w_P^T ((H^-1)_P)^-1 w_P / 2
 *   trace        nullable, R x k_blocks x d out: the row after every block step
 * The traces feed obc_global_select (with d := k_blocks) and obc_gather_trace unchanged.
 * Workspace: obc_blocks_workspace_bytes.  strategy: OBC_STRATEGY_BLOCKED handles c = 4 (and
 * c = 1, which is obc_prune_rows) and returns OBC_ERR_BAD_ARG otherwise; OBC_STRATEGY_AUTO uses
 * it for those and the rank-1 solver for every other block size. */
int obc_blocks_workspace_bytes(int R, int d, int c, int strategy, size_t *bytes);
int obc_prune_blocks(obc_ctx *ctx, const float *W, const float *Hinv, int R, int d, int c, int k_blocks,
                     const int32_t *stop_counts, int32_t *order, float *loss, float *W_out, float *trace,
                     int strategy, void *ws, size_t ws_bytes);

/* Flags of obc_quant_rows. */
#define OBC_QUANT_OUTLIERS 1   /* Sec. 5 "Quantization Outliers": while any live weight of the row has
                                  a quantization error |q(w) - w| > delta / 2, the greedy choice runs
                                  over those weights only (same score, same tie rule) */

/* Quantize every row with Algorithm 3 on the caller's per-row uniform grid
 *   q(w) = offset[i] + delta[i] * clamp(rne((w - offset[i]) / delta[i]), 0, maxq)
 * (rne = round half to even; the kernels evaluate the quotient in fp64 as a product with the fp64
 * reciprocal of delta[i], in the candidate scores and when the chosen weight is written alike).
 *   flags    0 or OBC_QUANT_OUTLIERS
 *   live     nullable, R x d: 0 marks an already pruned weight; those are first removed from the
 *            row's inverse (Lemma 1, no weight change) so that OBQ runs on the dense sub-problem
 *            of the survivors; they keep weight 0 and get code -1.
 *   order, loss   R x d: entries [0, #live_i) are written for row i
 *   codes    R x d int32 out: grid code of each weight at the moment it was chosen
 *   W_out    R x d out: dequantized weights offset + delta * code */
int obc_quant_rows(obc_ctx *ctx, const float *W, const float *Hinv, int R, int d,
                   const float *delta, const float *offset, int maxq, const uint8_t *live, int flags,
                   int32_t *order, float *loss, int32_t *codes, float *W_out, int strategy,
                   void *ws, size_t ws_bytes);

/* Per-row grid over the live weights (live nullable = all live).
 *   symmetric == 0: asymmetric min-max grid, offset = min, delta = (max - min) / maxq
 *   symmetric != 0: grid symmetric about zero, offset = -max|w|, delta = 2 max|w| / maxq
 * delta = 1 when the range is empty (constant row, all-zero row, no live weight). */
int obc_minmax_grid(obc_ctx *ctx, const float *W, const uint8_t *live, int R, int d, int maxq,
                    int symmetric, float *delta, float *offset);

/* ---- Appendix "Sequential Quantization with OBQ": re-fit of the dense weights ------------
 * When the layer's inputs X come from the already compressed model, the dense weights are first
 * re-optimised for them by the closed form of linear regression, W^T = (X X^T)^-1 X Y^T (Y = the
 * dense model's outputs of this layer, d_row x N); then their gradient is zero again and OBQ
 * applies.  With H = 2 X X^T (+ dampening, as obc_hessian forms it) and C = 2 Y X^T this is
 * W = C H^-1: the minimiser of the quadratic whose Hessian the row solvers use.  C is accumulated
 * over batches like H. */

/* Workspace of obc_cross. */
int obc_cross_workspace_bytes(int d_row, int d_col, int64_t N, size_t *bytes);

/* C (d_row x d_col, device, row-major) = 2 Y X^T, or C += 2 Y X^T when accumulate != 0.
 *   X  device, d_col x N, leading dimension ldx >= N;  Y  device, d_row x N, ldy >= N.
 * Matrix cores, the precision of fp32 products and sums, fixed summation order (deterministic).  Errors as
 * obc_hessian. */
int obc_cross(obc_ctx *ctx, const float *X, const float *Y, int d_col, int d_row, int64_t N, int64_t ldx,
              int64_t ldy, int accumulate, float *C, void *ws, size_t ws_bytes);

/* Workspace of obc_refit. */
int obc_refit_workspace_bytes(int d_col, int d_row, size_t *bytes);

/* W_out (d_row x d_col, device) = C H^-1 through the fp64 Cholesky factor of H (H^-1 itself is
 * never rounded to fp32 on the way).
 *   H   device, d_col x d_col, the dampened Hessian; left untouched when invert_in_place == 0,
 *       replaced by its inverse exactly as obc_invert does otherwise (the factorisation is shared)
 *   C   device, d_row x d_col, from obc_cross
 * Synchronises.  OBC_ERR_NOT_SPD as obc_invert. */
int obc_refit(obc_ctx *ctx, float *H, int d_col, const float *C, int d_row, float *W_out,
              int invert_in_place, void *ws, size_t ws_bytes);

/* ---- Appendix Algorithm 2: the global step ---------------------------------------------
 * From the per-row loss traces (loss, order: R x d as written by obc_prune_rows with
 * k_steps == d) find how many weights each row gives up when k weights are pruned from the
 * layer: k times, the row whose next loss change is smallest advances (lowest row on ties).
 *   counts   R int32 out;  mask  R x d uint8 out, 1 = pruned. */
int obc_global_select_workspace_bytes(int R, int d, size_t *bytes);
int obc_global_select(obc_ctx *ctx, const float *loss, const int32_t *order, int R, int d,
                      int64_t k, int32_t *counts, uint8_t *mask, void *ws, size_t ws_bytes);

/* The same global step for callers that cannot allocate device memory or hand over a workspace
 * (code under HIP graph capture, tight serving loops, harnesses that forbid allocation): the
 * scratch is a device array built into the library, OBC_SELECT_STATIC_SCRATCH_BYTES per GPU, held
 * from the library's load to the end of the process.  Arguments, results and errors as
 * obc_global_select; layers beyond OBC_SELECT_STATIC_MAX_WEIGHTS weights or
 * OBC_SELECT_STATIC_MAX_ROWS rows are refused with OBC_ERR_WORKSPACE.  The call allocates and
 * frees nothing, waits for nothing and clears its scratch with kernels.  All calls on one GPU
 * share that GPU's array: calls that overlap in time on one GPU (two streams, two contexts) race;
 * calls on one stream are ordered and safe. */
#define OBC_SELECT_STATIC_MAX_WEIGHTS 2359296 /* R * d, e.g. 512 x 4608, 768 x 3072, 3072 x 768 */
#define OBC_SELECT_STATIC_MAX_ROWS 8192
#define OBC_SELECT_STATIC_SCRATCH_BYTES (4 * OBC_SELECT_STATIC_MAX_WEIGHTS + 2 * 4 * OBC_SELECT_STATIC_MAX_ROWS + 2048)
int obc_global_select_static(obc_ctx *ctx, const float *loss, const int32_t *order, int R, int d,
                             int64_t k, int32_t *counts, uint8_t *mask);

/* ---- Sec. 4 Step 2: weights of the chosen mask from the pruning trace -------------------
 * W_out[i] = trace[i][counts[i]-1] (the row after counts[i] steps), or W[i] when counts[i] == 0.
 * trace is R x k_steps x d with k_steps >= max counts. */
int obc_gather_trace(obc_ctx *ctx, const float *W, const float *trace, const int32_t *counts,
                     int R, int d, int k_steps, float *W_out);

/* ---- Sec. 4 Step 2: weights of a mask by the group-OBS closed form ------------------------
 * For every row, with P the indices the mask marks as pruned,
 *     W_out = w - H^-1[:, P] ((H^-1)[P, P])^-1 w_P,    W_out[P] = 0 exactly
 * (the sign as in eq. (5)), from the ORIGINAL weights W and inverse Hessian Hinv: neither a trace nor a
 * second run of the greedy loop is needed (the paper's cheaper way to a row's weights once the global
 * step has fixed its mask).  The solve runs in fp64 through a Cholesky factorisation per row.
 *   mask        R x d uint8, non-zero = pruned (as obc_global_select writes it)
 *   max_pruned  upper bound on the pruned weights of any row, 0 <= max_pruned <= d; it sizes the
 *               workspace (8 max_pruned^2 bytes per row, roughly).  A row with more pruned weights
 *               than that is returned unchanged (a copy of W) and OBC_ERR_WORKSPACE is latched for
 *               obc_check; a non-positive pivot latches OBC_ERR_NUMERIC.
 * Asynchronous. */
int obc_reconstruct_workspace_bytes(int R, int d, int max_pruned, size_t *bytes);
int obc_reconstruct_rows(obc_ctx *ctx, const float *W, const float *Hinv, const uint8_t *mask, int R, int d,
                         int max_pruned, float *W_out, void *ws, size_t ws_bytes);

/* ---- Running compressed layers of language models -----------------------------------------
 * A layer's codes on a grid of at most 16 values, packed to 4 bits with a step and an offset per row
 * and group of `group` consecutive columns, and the operators around it: its product with activations
 * (single tokens to prompts), the gradient of its inputs, the root-mean-square norm before it, and the
 * loss against the dense model's answers by which what stays uncompressed is tuned.  All asynchronous.
 * Element types of activations, gradients and logits: */
#define OBC_F32 0
#define OBC_F16 1
#define OBC_BF16 2
#define OBC_I8 3   /* 8-bit integers with an fp32 scale per row */

/* Flags of obc_group_grid. */
#define OBC_GRID_SYMMETRIC 1 /* symmetric about zero: offset = -max|w|, delta = 2 max|w| / maxq */
#define OBC_GRID_ZERO 2      /* zero is one of the grid's values (layers that are pruned and quantized) */

/* Grid of every row and group over its live weights (live nullable = all live): min-max, or as `flags`
 * say; 1 <= maxq <= 15.  group: 32, 64 or a multiple of 128; 0 or >= d: one group per row.
 *   delta, offset   R x ceil(d / group) out; values of half precision, rounded so that the grid still
 *                   covers the weights, as obc_pack4 keeps them.  With one group per row they are what
 *                   obc_quant_rows takes.  delta = 1 where the range is empty.
 * A group whose weights half precision cannot hold latches OBC_ERR_NUMERIC. */
int obc_group_grid(obc_ctx *ctx, const float *W, const uint8_t *live, int R, int d, int group, int maxq,
                   int flags, float *delta, float *offset);

/* Pack R x d codes (int32, 0 .. 15, as obc_quant_rows writes them) with their grid for the products:
 * weight = offset + delta * code.  delta and offset (R x ceil(d / group)) are rounded to half precision
 * (obc_group_grid's already are).  A code of -1 is a pruned weight: it takes the code whose value is
 * exactly 0.  A code out of range, or of -1 on a grid without a zero, latches OBC_ERR_BAD_ARG; a step or
 * offset beyond half precision or not finite latches OBC_ERR_NUMERIC.  `packed` (obc_pack4_bytes, aligned
 * to 16 bytes) is opaque: codes in the order of the matrix instructions' operands. */
int obc_pack4_bytes(int R, int d, int group, size_t *bytes);
int obc_pack4(obc_ctx *ctx, const int32_t *codes, const float *delta, const float *offset, int R, int d,
              int group, void *packed);

/* y = x W^T for T tokens: y[t, r] = sum_c x[t, c] (offset + delta code)[r, c], T x R.
 *   x   T x d, leading dimension ldx >= d, of x_type; OBC_I8: x stands for x_scale[t] * x[t, c]
 *       (x_scale: T fp32; null for the other types)
 *   y   T x R, leading dimension ldy >= R, of y_type (OBC_F32, OBC_F16 or OBC_BF16)
 * Products are exact and sums have the precision of fp32 (OBC_I8: integer sums over up to 128 columns of a group, exact;
 * those are joined in fp32); one rounding, to y's type.  Codes enter the sums as up to 31 times an input: these are to stay
 * below fp32's 3.4e38.  Rows need no alignment beyond their elements'.  Fixed summation order for a given T, R, d and group.
 * A non-finite input makes its token's outputs non-finite (inf or NaN).  y may not overlap x.  Where a row has several
 * groups, ceil(d / 128) * (group / 128) has to be below 2^32 (OBC_ERR_BAD_SHAPE).
 * ws: obc_product4_workspace_bytes for this T (0 up to 16 tokens, but for few rows of many columns). */
int obc_product4_workspace_bytes(int T, int R, int d, int group, int x_type, size_t *bytes);
int obc_product4(obc_ctx *ctx, const void *packed, int R, int d, int group, const void *x, int x_type,
                 const float *x_scale, int T, int64_t ldx, void *y, int y_type, int64_t ldy, void *ws,
                 size_t ws_bytes);

/* dx = dy W for T tokens, the gradient of obc_product4's inputs: dx[t, c] = sum_r dy[t, r] W[r, c].
 *   dy  T x R, leading dimension lddy >= R;  dx  T x d, leading dimension lddx >= d; both of `type`
 *       (OBC_F32, OBC_F16 or OBC_BF16)
 * 16-bit types: weights to 22 bits, products and sums fp32, one rounding of the result.  OBC_F32: the precision of
 * fp32 throughout.  Fixed summation order for a given T, R, d and group.  A non-finite dy makes its token's outputs
 * non-finite.  dx may not overlap dy. */
int obc_product4_grad_workspace_bytes(int T, int R, int d, int group, int type, size_t *bytes);
int obc_product4_grad(obc_ctx *ctx, const void *packed, int R, int d, int group, const void *dy, int type, int T,
                      int64_t lddy, void *dx, int64_t lddx, void *ws, size_t ws_bytes);

/* Root-mean-square norm of T rows with the residual's addition:
 *   h = x + residual,  y = h / sqrt(mean(h^2) + eps) * gain
 *   x, residual, h   T x d, contiguous, of x_type (OBC_F32, OBC_F16, OBC_BF16); residual nullable (h = x); h
 *            nullable (not written), h == x or h == residual allowed.  The norm is of the unrounded sum.
 *   gain     d, fp32
 *   y        T x d of y_type: x_type or OBC_I8; OBC_I8: y stands for y_scale[t] * y[t, c], y_scale[t] =
 *            max|y| / 127 (1 for a row of zeros; NaN, and codes 0, for a row with a NaN or an infinity, also where
 *            the gain brings it in)
 *   y_scale  T fp32 out, with OBC_I8;  rstd  nullable, T fp32 out: 1 / sqrt(mean(h^2) + eps)
 * Squares are summed in fp32: values beyond about 1e19 give a row of zeros, in 8 bits scale NaN and codes 0.
 * 1 <= d <= 65536. */
int obc_rmsnorm(obc_ctx *ctx, const void *x, const void *residual, int x_type, const float *gain, float eps, int T,
                int d, void *h, void *y, int y_type, float *y_scale, float *rstd);

/* Its backward pass (8-bit outputs: straight through the rounding), from the saved sum h and rstd:
 *   dx = dh + rstd (gain dy - xhat mean(gain dy xhat)),  dgain = sum_t dy xhat,   xhat = h rstd
 *   h, dy, dh, dx   T x d, contiguous, of `type`; dh: the gradient that reaches h on the residual path, nullable.
 *                   dx is the gradient of x and of residual alike; dx == dy or dx == dh allowed
 *   dgain    d fp32 out
 * Fixed summation order. */
int obc_rmsnorm_grad_workspace_bytes(int T, int d, size_t *bytes);
int obc_rmsnorm_grad(obc_ctx *ctx, const void *h, const float *gain, const float *rstd, const void *dy, const void *dh,
                     int type, int T, int d, void *dx, float *dgain, void *ws, size_t ws_bytes);

/* Distillation from a teacher's top logits.  For every row t with its valid entries j (top_index >= 0)
 *   p_j = softmax over the valid entries of top_logit / temperature,  q = softmax over the row of z / temperature
 *   loss[t] = weight[t] temperature^2 sum_j p_j (log p_j - log q[top_index_j])
 *   dz[t, v] = weight[t] temperature (q[v] - sum of p_j over the entries with top_index_j = v)
 * dz is the gradient of the losses' sum.
 *   z          T x V logits of `type`, leading dimension ldz >= V
 *   top_index  T x k int32, negative: no entry (rows may hold any number from 0 to k); top_logit  T x k fp32
 *   weight     nullable (1), T fp32.  A row of weight 0 or without an entry has loss 0 and a gradient of zeros,
 *              whatever its logits are.  An entry with a logit of -inf counts as none.
 *   loss       T fp32 out;  dz  nullable, T x V out of `type`, leading dimension lddz; dz == z allowed (lddz == ldz)
 * An index >= V latches OBC_ERR_BAD_ARG and counts as no entry.  0 <= k <= 1024, temperature > 0. */
int obc_distill(obc_ctx *ctx, const void *z, int type, int T, int V, int64_t ldz, const int32_t *top_index,
                const float *top_logit, int k, float temperature, const float *weight, float *loss, void *dz,
                int64_t lddz);

/* ---- Judging and tuning compressed models -------------------------------------------------
 * The dense model's side of the distillation and the judgement of the compressed one's answers, and what is tuned around the
 * packed layers: layer norms, embedding tables, and the step that applies their gradients.  All asynchronous. */

/* Scores of T rows of logits at a temperature, with d = z / temperature:
 *   lse[t] = log sum_v exp(d[v]),  logp[t] = d[target[t]] - lse[t],  entropy[t] = -sum_v p[v] log p[v],  p = exp(d - lse)
 *   top_index, top_logit   the k largest logits z, largest first, the lowest index first among equal ones; top_logit holds them
 *                          as they are, so that they are what obc_distill takes
 *   z          T x V of `type`, leading dimension ldz >= V;  target  nullable, T int32: negative: none, logp 0
 *   logp (goes with target), entropy, lse   nullable, T fp32 out
 *   top_index, top_logit   T x k int32 and fp32 out; null with k = 0.  0 <= k <= 1024, V <= 2^30
 * A logit of -inf has probability 0, adds nothing and is never among the largest; entries that are left over have index -1 and
 * logit -inf.  A row of -inf alone has lse and logp -inf and entropy 0.  A row with a NaN or +inf has NaN for all its numbers and
 * indices of -1 (a logp of 0 where it has no target).  A target >= V latches OBC_ERR_BAD_ARG and counts as none. */
int obc_score_workspace_bytes(int T, int V, int type, int k, size_t *bytes);
int obc_score(obc_ctx *ctx, const void *z, int type, int T, int V, int64_t ldz, const int32_t *target, float temperature, int k,
              float *logp, float *entropy, float *lse, int32_t *top_index, float *top_logit, void *ws, size_t ws_bytes);

/* Layer norm of T rows with the residual's addition:
 *   h = x + residual,  y = (h - mean(h)) rstd gain + bias,  rstd = 1 / sqrt(mean((h - mean(h))^2) + eps)
 *   gain, bias   d, fp32; bias nullable (0);  mean, rstd  nullable, T fp32 out
 * The rest as in obc_rmsnorm.  Sums are fp32: a row with deviations beyond about 1e19 gives its bias or NaN, in 8 bits scale NaN and
 * codes 0. */
int obc_layernorm(obc_ctx *ctx, const void *x, const void *residual, int x_type, const float *gain, const float *bias, float eps, int T,
                  int d, void *h, void *y, int y_type, float *y_scale, float *mean, float *rstd);

/* Its backward pass (8-bit outputs: straight through the rounding), from the saved sum h, mean and rstd:
 *   w = gain dy,  dx = dh + rstd (w - mean(w) - xhat mean(w xhat)),  dgain = sum_t dy xhat,  dbias = sum_t dy,
 *   xhat = (h - mean) rstd
 *   dgain, dbias   d fp32 out; dbias nullable.  The rest as in obc_rmsnorm_grad. */
int obc_layernorm_grad_workspace_bytes(int T, int d, size_t *bytes);
int obc_layernorm_grad(obc_ctx *ctx, const void *h, const float *gain, const float *mean, const float *rstd, const void *dy,
                       const void *dh, int type, int T, int d, void *dx, float *dgain, float *dbias, void *ws, size_t ws_bytes);

/* y[t] = scale table[ids[t]] for T tokens, T x d.
 *   table   V x d of `type`, leading dimension ldt >= d;  y  of y_type, leading dimension ldy >= d (OBC_F32, OBC_F16, OBC_BF16 each)
 *   ids     T int32; negative: no token, a row of zeros
 * The product is fp32, rounded once.  An id >= V latches OBC_ERR_BAD_ARG and counts as no token.  y may not overlap
 * the table.  1 <= d <= 2^20. */
int obc_embed(obc_ctx *ctx, const void *table, int type, int V, int d, int64_t ldt, const int32_t *ids, int T, float scale, void *y,
              int y_type, int64_t ldy);

/* The table's gradient: dtable[v] = scale sum over the tokens t with ids[t] = v of dy[t]; every row is written, with zeros where it
 * has no token.  accumulate != 0: dtable[v] += that, rows without a token are not touched.
 *   dy      T x d of `type`, leading dimension lddy >= d;  dtable  V x d of dtable_type, leading dimension lddt >= d
 * Sums are fp32, over an id's tokens in a fixed order; one rounding.  Ids as in obc_embed.  dtable may not
 * overlap dy.  T <= 2^26. */
int obc_embed_grad_workspace_bytes(int T, int V, int d, size_t *bytes);
int obc_embed_grad(obc_ctx *ctx, const int32_t *ids, int T, const void *dy, int type, int64_t lddy, float scale, int V, int d,
                   int accumulate, void *dtable, int dtable_type, int64_t lddt, void *ws, size_t ws_bytes);

/* A tensor of obc_adamw_plan: n elements each, contiguous.  Inputs and outputs may be the same arrays (the usual case) or others.  An
 * output overlaps no other output and no input, but that it may be, from its first byte to its last, an input of the same tensor. */
typedef struct obc_adamw_tensor {
    const void *p;                  /* parameters, of `type` */
    void *p_out;
    const void *g;                  /* gradients, of `type` */
    const void *m;                  /* first moment: fp32, or 8-bit numbers (sign, 4 bits of exponent, 3 of mantissa: up to 448) */
    void *m_out;
    const void *v;                  /* second moment: fp32, or its root in 8-bit numbers */
    void *v_out;
    const float *m_scale, *v_scale; /* 8 bits: ceil(n / 256) factors of 256 consecutive numbers each */
    float *m_scale_out, *v_scale_out;
    const float *master;            /* nullable: the parameters in fp32, which p is a rounded copy of */
    float *master_out;
    int64_t n;
    float decay;
} obc_adamw_tensor;

/* Lay out `count` tensors for obc_adamw, which takes them in one launch.
 *   tensors     HOST array; it may go when the call returns
 *   bits        of the moments: 32 or 8
 *   plan        obc_adamw_plan_bytes on the device, aligned to 16 bytes, opaque; written on the context's stream
 *   workgroups  HOST out, for obc_adamw.  (2^24 - 1 at most, of 2048 elements of a tensor each.)
 * Overlaps as said above are refused; gradients may be listed more than once. */
int obc_adamw_plan_bytes(int count, size_t *bytes);
int obc_adamw_plan(obc_ctx *ctx, const obc_adamw_tensor *tensors, int count, int type, int bits, void *plan, int64_t *workgroups);

/* One step of AdamW over a plan's tensors:
 *   g' = g grad_scale,  m = beta1 m + (1 - beta1) g',  v = beta2 v + (1 - beta2) g'^2
 *   p = p (1 - lr decay) - lr m / (1 - beta1^step) / (sqrt(v / (1 - beta2^step)) + eps)
 * in fp32, on master where there is one; p is rounded to nearest from that.
 *   count, workgroups, type, bits   the plan's
 *   step        1 for the first; step_at (device, nullable) is read in its place.  lr_at (device, nullable) in lr's place.
 *               Neither is changed.  A step_at below 1 latches OBC_ERR_BAD_ARG and leaves all values as they are.
 *   grad_scale  device, nullable (1): a loss scale's reciprocal or a clipping factor.  Infinite or NaN: all values stay as they are.
 * Moments of 8 bits: m and sqrt(v) are divided by their block's scale, its largest magnitude / 448, and rounded up or down with the
 * chances that keep them on average, by a hash of seed, step, the tensor's place in the list and the element's in the tensor (in 64
 * bits where fp32 is within 6 units of its last place of deciding otherwise); sqrt(v) > 0 is never rounded to 0.  A block whose
 * largest is below 1e-30 becomes zeros.  A block with a NaN or an infinity gets scale NaN.
 * 0 <= beta < 1, eps >= 2^-120.  (Moments of 32 bits: a v that fp32's least number, 2^-149, does not reach is zero.)  Results do not depend on
 * how tensors are listed, but for the hash. */
int obc_adamw(obc_ctx *ctx, const void *plan, int count, int64_t workgroups, int type, int bits, int64_t step, const int64_t *step_at,
              float lr, const float *lr_at, double beta1, double beta2, float eps, const float *grad_scale, uint32_t seed);

#ifdef __cplusplus
}
#endif
#endif /* OBC_H */
