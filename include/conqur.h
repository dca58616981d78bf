/*
 * conqur.h -- C ABI of the MI355X (gfx950) hot path of ConQuR's online rotation
 * calibration: rotate -> row-normalise -> hypercube-corner assign -> accumulate
 * the cross-covariance -> closed-form orthogonal Procrustes (polar) update, plus
 * the per-token symmetric fake-quantisation error of the rotated activations.
 *
 * Conventions (all matrices row-major, activations are rows, App. A "X_hat = X R"):
 *   y_i  = x_i R                      the rotation maps row vectors; it is the
 *                                     transpose of the R of Sec. 3 (which writes R x)
 *   M    = sum_i (x_i/||x_i||)^T c_i  c_i = sgn(y_i)/sqrt(dh), sgn(0) = +1 (Eq. 2);
 *                                     the transpose of Sec. 3.3's C = Z^T X~
 *   R    <- polar(M) = U V^T          Sec. 3.3, for M = U S V^T
 * With heads = h > 1 the row of width d is h independent blocks of width dh = d/h,
 * each with its own rotation, statistics and update (App. A: the block-diagonal
 * per-head rotation; Sec. 3.4 "a Procrustes problem per head").
 *
 * Pointers are tagged HOST or DEVICE below.  Every call returns a conqur_status;
 * nothing throws across the boundary.  Calls enqueue their kernels on the stream
 * given at init and return without waiting unless a HOST output is requested.
 * A context is not thread safe.  The library never falls back to the CPU: every
 * step below runs in HIP kernels, and a call fails with CONQUR_EHIP if the device
 * or a launch fails.
 */
#ifndef CONQUR_H
#define CONQUR_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct conqur_ctx conqur_ctx; /* opaque; owns R, the rotate operand, M and all workspaces (device) */

typedef enum {
  CONQUR_OK = 0,
  CONQUR_EINVAL = 1,    /* bad argument, shape, stride or alignment; nothing was enqueued        */
  CONQUR_ESTATE = 2,    /* call not valid in this state (update with no accumulated row)         */
  CONQUR_ENOMEM = 3,    /* device or host allocation failed                                      */
  CONQUR_EHIP = 4,      /* a HIP call failed; conqur_last_error() holds the HIP error string      */
  CONQUR_ENOCONV = 5,   /* polar iteration hit polar_max_iters; R holds the last iterate and the
                           reported orthogonality error says how far it is from orthogonal        */
  CONQUR_ENONFINITE = 6 /* (reported by update) rows with NaN/Inf were met and skipped           */
} conqur_status;

typedef enum { CONQUR_F32 = 0, CONQUR_BF16 = 1 } conqur_dtype;

typedef struct {
  uint32_t d;               /* row width of X; d % heads == 0, (d/heads) % 16 == 0, d/heads <= 8192 */
  uint32_t heads;           /* 1 = one d x d rotation; h > 1 = h independent (d/h) x (d/h) problems */
  uint32_t act_dtype;       /* conqur_dtype of X; the rotate operand is R rounded to this type      */
  uint32_t max_tokens;      /* largest T passed to step_batch / quant_error (sizes the workspaces);
                               (d/heads) * round_up(max_tokens, 64) < 2^30                           */
  float prox_lambda;        /* R <- polar(M + lambda * tau * R_prev), tau = ||M||_F / sqrt(dh): the proximal
                               reading that makes the update unique when M is rank deficient.  0 asks for
                               the paper's update R <- polar(M) (Sec. 3.3) and is taken as the limit
                               lambda -> 0+ at fp32 resolution: values below 2^-20 are raised to 2^-20
                               (that ties R to R_prev on the null space of M, where every completion is
                               optimal, and breaks exact degeneracies a polynomial iteration would keep;
                               it moves <R, M> by less than 1e-6 relative)                            */
  float polar_tol;          /* stop when ||X^T X - I||_F <= tol; 0 selects 9.5e-5                    */
  uint32_t polar_max_iters; /* 0 selects 200                                                        */
  uint32_t polar_precision; /* arithmetic of the main polar iterations: 0 = single fp16 operands (fast; 11
                               significant bits: meets the orthogonality and objective tolerances, R itself
                               deviates a little on directions with small singular values, where a step's
                               rounding is amplified by 1/sigma), 1 = two bf16 planes per operand (about 16
                               significant bits), 2 = three planes (fp32-equivalent products).
                               The closing iterations always run fp32-equivalent.                     */
  uint32_t polar_verify;    /* orthogonality of the final iterate: 0 = bounded from the last measured
                               residual (exact-arithmetic residual of the closing step, from ||D^3||_F,
                               plus a rounding allowance; one bf16 GEMM), 1 = measured by one more
                               fp32-equivalent Gram matrix (costs about six bf16 GEMMs)               */
  int32_t device;           /* HIP device ordinal                                                   */
  void* stream;             /* hipStream_t the caller owns (NULL = the device's default stream)      */
} conqur_config;

/* Per-head statistics of the rows accumulated since the last update (HOST struct). */
typedef struct {
  uint64_t rows;    /* rows that entered M                                                         */
  uint64_t skipped; /* rows skipped: all-zero or non-finite head slice                             */
  double l1;        /* L = sum_i ||y_i||_1 / ||x_i||_2                                               */
  double objective; /* Eq. 1 summed over those rows, sum_i || y_i/||x_i|| - c_i ||^2, evaluated through
                       the l1 identity of Sec. 3.2 as 2*rows - 2*L/sqrt(dh)                          */
} conqur_batch_stats;

/* Per-head result of one Procrustes update (HOST struct). */
typedef struct {
  uint32_t iters;       /* polar iterations run (main + closing)                                   */
  uint32_t accurate;    /* how many of them were closing iterations (fp32-equivalent Gram)         */
  double orth_err;      /* ||R^T R - I||_F of the stored fp32 R: measured on the device, or an upper
                           estimate of it (see polar_verify)                                         */
  double inner;         /* <R_new, M>, the Procrustes objective value (nuclear norm at the optimum)  */
  double m_fro;         /* ||M||_F                                                                  */
  double ms;            /* device time of this update in milliseconds (all heads together): from the start of
                           its first launch to the report of its results, by the device's 100 MHz clock.
                           conqur_get_timing's event times hold the launch's latency and its end as
                           well, 2 to 5 us more                                                       */
  uint32_t orth_measured; /* 1: orth_err was measured; 0: it is the estimate                          */
  uint32_t reserved;
  double l1;            /* L of the rows this update consumed (as conqur_batch_stats.l1 just before it)   */
  double mfma_flop;     /* multiply-add work the update's matrix products issued, in FLOP, all heads
                           together (tiles that ran x tile area x contraction length x 2: symmetric
                           products run on the tiles on and above the diagonal only, split-plane
                           products count once per plane pair); the algorithmic figure is
                           4 dh^3 heads per iteration                                                 */
} conqur_update_stats;

/*
 * Create a context (Alg. 1 "initial rotation").  R0_host: HOST, heads*dh*dh floats,
 * head-major, each block row-major and orthogonal (not checked).  Copied; the caller
 * keeps ownership.  On success *out receives the context.  Allocates all device
 * memory the other calls need; those calls allocate nothing.
 */
conqur_status conqur_init(const conqur_config* cfg, const float* R0_host, conqur_ctx** out);

/*
 * One batch of the statistics loop (Alg. 1 inner loop; Sec. 3.4): for every row
 * x_i of X and every head, rotate with the operand copy of R, take the corner of
 * the rotated row (Eq. 2), and add (x_i/||x_i||)^T c_i to M.  May be called many
 * times before one update (Alg. 1 pools all sites of a mini-batch).
 * X_dev: DEVICE, T rows of row_stride_elems elements of act_dtype, of which the
 * first d are used; 16-byte aligned base and row pitch.  1 <= T <= max_tokens,
 * T * row_stride_elems < 2^30 (CONQUR_EINVAL otherwise).  The caller keeps ownership of X and may reuse it once the stream has passed
 * this call's kernels.  Asynchronous; never touches the host.
 */
conqur_status conqur_step_batch(conqur_ctx* ctx, const void* X_dev, uint64_t T, uint64_t row_stride_elems);

/*
 * The same for the heads [head0, head0 + nheads) only: X_dev holds T rows whose first
 * nheads * dh columns belong to those heads.  One context can so carry the per-head
 * rotations of several layers (Alg. 1 keeps one R_2 per layer, App. A one block per
 * head): every layer's batch goes to its own range, and a single
 * conqur_update_rotation then updates all of them in batched launches that fill the
 * device, which one layer's heads alone do not.  A partial range needs heads of width
 * 128 and bf16 activations (CONQUR_EINVAL otherwise); the full range is
 * conqur_step_batch.  Every head must have received rows before the update
 * (CONQUR_ESTATE otherwise).  After a partial range conqur_get_last_corners has nothing
 * to return (CONQUR_ESTATE).
 */
conqur_status conqur_step_batch_heads(conqur_ctx* ctx, const void* X_dev, uint64_t T, uint64_t row_stride_elems,
                                      uint32_t head0, uint32_t nheads);

/*
 * Read the per-head statistics accumulated since the last update.  stats_host:
 * HOST array of `heads` entries.  Synchronises the stream.
 */
conqur_status conqur_get_batch_stats(conqur_ctx* ctx, conqur_batch_stats* stats_host);

/*
 * Orthogonal Procrustes update (Sec. 3.3): R <- polar(M + prox_lambda*tau*R) per
 * head, computed on the device by a GEMM-only Newton-Schulz iteration; refreshes
 * the rotate operand and clears M and the batch statistics (Alg. 1 starts every
 * mini-batch with empty statistics).  stats_host: HOST array of `heads` entries or
 * NULL.  Synchronises the stream (the iteration count is data dependent).
 * Returns CONQUR_ESTATE if no row was accumulated, CONQUR_ENOCONV if the cap was
 * hit (R is still replaced; stats->orth_err tells how good it is), and
 * CONQUR_ENONFINITE (after a successful update) if rows were skipped as non-finite.
 * CONQUR_ENONFINITE is also returned when M itself is not finite; rotation, operand and
 * statistics are then left as they were (conqur_last_error tells which of the two it is).
 */
conqur_status conqur_update_rotation(conqur_ctx* ctx, conqur_update_stats* stats_host);

/*
 * Score the current rotation (App. B symmetric quantiser; Sec. 4.3 error metric):
 * Y = X R_op per head, stored in act_dtype, then per token (one scale over the whole
 * row of width d) D = max|y| / (2^(bits-1) - 1), q = D * round_half_even(y / D)
 * clamped to the level range.  sse_host = sum (y - q)^2, energy_host = sum y^2
 * (both HOST doubles).  X_dev as in conqur_step_batch.  bits in [2, 8].  Does not
 * change the calibration state.  Synchronises the stream.
 */
conqur_status conqur_quant_error(conqur_ctx* ctx, const void* X_dev, uint64_t T, uint64_t row_stride_elems,
                                 uint32_t bits, double* sse_host, double* energy_host);

/*
 * The same score with the per-token asymmetric (zero-point) quantiser (App. B, "zeropoint
 * quantizer"; App. C evaluates activations with clipping ratio 0.9): per token, over the
 * whole row, lo = clip_ratio * min_j y_j, hi = clip_ratio * max_j y_j, D = (hi - lo) /
 * (2^bits - 1), integer zero point zeta = -round_half_even(lo / D), code = round_half_even(y / D)
 * + zeta clamped to [0, 2^bits - 1], q = D * (code - zeta); a constant row has the single
 * level lo.  clip_ratio in (0, 1] (1: the appendix's quantiser).  Arguments, outputs,
 * synchronisation and errors as conqur_quant_error.
 */
conqur_status conqur_quant_error_zp(conqur_ctx* ctx, const void* X_dev, uint64_t T, uint64_t row_stride_elems,
                                    uint32_t bits, float clip_ratio, double* sse_host, double* energy_host);

/*
 * The rotated rows themselves: Y = X R_op per head (R_op = R rounded to act_dtype;
 * fp32-equivalent products for fp32), stored in act_dtype -- Eq. 1's R x~ before
 * normalisation; with the rows of a weight matrix as X this folds the learned rotation
 * into that matrix (App. A).  X_dev as in conqur_step_batch (T <= max_tokens rows per
 * call).  Y_dev: DEVICE, T rows of y_row_stride_elems elements of act_dtype
 * (d <= y_row_stride_elems < 2^21, else CONQUR_EINVAL), owned by the caller, must not
 * overlap X.  Asynchronous on the context's stream; does not change the calibration
 * state.  Every call that rotates rows (this one, the scores, the diagnostics, the
 * quantised rows, the statistics steps of the general path) gives the same rows the same
 * sums in calls of the same size.  Calls of up to 16 rows (32 with fp32 activations or dh <= 4096)
 * add up the dh products of an entry in another order than larger calls: a row rotated in
 * either may differ in the last bit of its fp32 sums, hence in the rounding of an entry
 * or in the corner sign of one that is zero to rounding.
 */
conqur_status conqur_rotate(conqur_ctx* ctx, const void* X_dev, uint64_t T, uint64_t row_stride_elems, void* Y_dev,
                            uint64_t y_row_stride_elems);

/*
 * The fake-quantised rotated rows: Yq = Q(X R_op), what a linear layer receives when its
 * input is quantised after the current rotation has been applied (quantisation-aware
 * calibration, Sec. 3.4).  Y = X R_op as in conqur_rotate; each row of width d is then
 * quantised per token with the symmetric quantiser of conqur_quant_error (zero_point =
 * 0; clip_ratio ignored) or the zero-point quantiser of conqur_quant_error_zp
 * (zero_point = 1, clip_ratio in (0, 1]) and written as the level values q (not the
 * integer codes), rounded once into act_dtype.  Yq_dev: DEVICE, T rows of
 * yq_row_stride_elems >= d elements of act_dtype, base and row pitch multiples of 16
 * bytes, owned by the caller, must not overlap X.  Asynchronous on the context's stream;
 * does not change the calibration state.  Errors: CONQUR_EINVAL (bits outside [2, 8],
 * zero_point > 1, clip_ratio outside (0, 1], NULL / misaligned Yq_dev, bad X
 * arguments), CONQUR_EHIP.
 */
conqur_status conqur_rotate_quant(conqur_ctx* ctx, const void* X_dev, uint64_t T, uint64_t row_stride_elems, uint32_t bits,
                                  uint32_t zero_point, float clip_ratio, void* Yq_dev, uint64_t yq_row_stride_elems);

/*
 * Quantisation-aware calibration (Sec. 3.4, second paragraph: during calibration the input of every
 * linear layer is quantised after the current rotation has been applied, so that later sites see
 * the activations inference will give them): conqur_step_batch and conqur_rotate_quant of the same
 * batch in ONE call and from ONE rotation of X.  The site's statistics are accumulated exactly as
 * conqur_step_batch does, and Yq_dev receives Q(X R_op) exactly as conqur_rotate_quant writes it --
 * the quantised input of the layer behind the site.  Arguments and errors as for those two calls.
 * (Heads of width 128 with bf16 activations rotate twice internally: their fused step keeps the
 * rotated rows on the compute unit.)  Asynchronous on the context's stream.
 */
conqur_status conqur_step_batch_quant(conqur_ctx* ctx, const void* X_dev, uint64_t T, uint64_t row_stride_elems, uint32_t bits,
                                      uint32_t zero_point, float clip_ratio, void* Yq_dev, uint64_t yq_row_stride_elems);

/*
 * Per-row diagnostics of the rotated activations: Y = X R_op per head, stored in
 * act_dtype, then per token over the whole row of width d
 *   pr  = ||y||_2^4 / (d ||y||_4^4)   normalised participation ratio (Sec. 4.2), in [1/d, 1]
 *   rho = ||y||_inf^2 / ||y||_2^2     dynamic-range ratio of the SQNR bound (App. B), in [1/d, 1]
 * pr_host / rho_host: HOST, T floats each, either may be NULL; a row with zero or
 * non-finite energy gets 0.  X_dev as in conqur_step_batch.  Does not change the
 * calibration state.  Synchronises the stream.
 */
conqur_status conqur_row_diagnostics(conqur_ctx* ctx, const void* X_dev, uint64_t T, uint64_t row_stride_elems,
                                     float* pr_host, float* rho_host);

/*
 * Copy state to the host / replace it (checkpointing, and teacher-forced parity
 * tests).  R_host, M_host: HOST, heads*dh*dh floats or NULL.  n_rows_host: HOST,
 * `heads` entries or NULL: the rows that entered M since the last update (as
 * conqur_batch_stats.rows).  set_state(R) also refreshes the rotate operand;
 * set_state(M) marks the statistics as holding rows, so that an update may follow; the
 * row and skipped counters and the l1 term then still describe the rows stepped through
 * the library, not the M that was written.  Both synchronise the stream.
 */
conqur_status conqur_get_state(conqur_ctx* ctx, float* R_host, float* M_host, uint64_t* n_rows_host);
conqur_status conqur_set_state(conqur_ctx* ctx, const float* R_host, const float* M_host);

/*
 * Keep (enable != 0) or drop (0, the default) the corner signs of every later
 * conqur_step_batch for conqur_get_last_corners.  Only the fused per-head step
 * (heads of width 128, bf16 activations) honours the switch -- there the signs never
 * leave the compute unit otherwise and storing them doubles the step's HBM traffic;
 * the general path produces them anyway as an operand of the accumulate GEMM.
 */
conqur_status conqur_set_taps(conqur_ctx* ctx, int enable);

/*
 * Debug / parity taps of the last conqur_step_batch: the corner signs as int8
 * (+1 / -1; HOST, T*d, row-major like X) and the per-row norms (HOST, heads*T,
 * head-major; 0 marks a skipped row).  Either may be NULL.  Synchronises.
 * CONQUR_ESTATE if the signs are asked for and the last step did not keep them
 * (see conqur_set_taps).
 */
conqur_status conqur_get_last_corners(conqur_ctx* ctx, int8_t* signs_host, float* norms_host);

/*
 * For callers that cannot allocate device memory or wait for the stream (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the score of
 * conqur_quant_error (zero_point = 0; clip_ratio ignored) or conqur_quant_error_zp (zero_point
 * = 1) on rows that are ALREADY rotated -- Y_dev is what conqur_rotate wrote -- with the two
 * results left in device memory.  No context: the per-row results the score kernels exchange
 * live in a static device array of the library (2 floats per row, 512 KiB, held by every GPU
 * the library has run on until the process ends), so the call allocates nothing, copies
 * nothing to the host and returns without waiting.  Runs on the CURRENT device; `stream` must
 * belong to it (NULL = its default stream).  The array's address is looked up once per device,
 * by conqur_init or by the first call on that device: make that first call outside any graph
 * capture.  Y_dev: DEVICE, T rows of row_stride_elems >= d elements of dtype (conqur_dtype),
 * 16-byte aligned base and row pitch; 1 <= T <= 65536 rows per call (more: CONQUR_EINVAL, split
 * the rows over several calls and add the results); d a multiple of 16, at most 65536.
 * out_dev: DEVICE, 2 doubles, overwritten with { sum (y - q)^2, sum y^2 } once the stream has
 * passed the call's kernels.  All calls on one GPU share the array, which keeps the last
 * call's per-row values: calls that overlap in time on one GPU (different streams) race; calls
 * on one stream are ordered and safe.  Errors: CONQUR_EINVAL (arguments as above, bits outside
 * [2, 8], zero_point > 1, clip_ratio outside (0, 1]), CONQUR_EHIP.
 */
conqur_status conqur_score_rows_static(const void* Y_dev, uint32_t dtype, uint64_t T, uint64_t d, uint64_t row_stride_elems,
                                       uint32_t bits, uint32_t zero_point, float clip_ratio, double* out_dev, void* stream);

/* ---- One attention layer around the calibrated heads -------------------------------------------
 * What stands between a layer's projections and the rows that o_proj (and the per-head rotations above) receive: positions
 * and norms of queries and keys, a paged cache that holds keys and values in 16 bits or in the zero-point codes of 8 or 4
 * bits, and the attention of new tokens over it.  These calls need no context.  They run on the CURRENT device, on `stream`
 * (NULL = its default stream), which must belong to it; they allocate nothing, copy nothing to the host and return without
 * waiting, so they may be captured into a HIP graph.  All memory they name is DEVICE memory of the caller's, except where
 * HOST is said; it must stay until the stream has passed the call.  `conqur_rotary_call` and its like are HOST structs, read
 * before the call returns.  Errors: CONQUR_EINVAL (nothing was enqueued), CONQUR_EHIP.                                    */

/* Rows of several heads: entry e of head h of token t lies at data + t * token_stride + h * head_stride + e, in elements of the
 * call's dtype.  Inputs may have any strides from 0 (one row for all) to below 2^40; an output's rows must not overlap (an
 * output may be its own input).  heads = 0: absent, the rest is ignored.  A base and strides that are multiples of 16 bytes are the fast case; any
 * multiple of the element's size is allowed.                                                                            */
typedef struct {
  void* data;
  int64_t token_stride;
  int64_t head_stride;
  uint64_t heads;
} conqur_heads;

/* Which entries of a head's rotated part form pair j: (j, j + part/2), or (2j, 2j + 1). */
typedef enum { CONQUR_HALF = 0, CONQUR_INTERLEAVED = 1 } conqur_rotary_layout;

/* How the frequencies theta^(-2j/part) are stretched by `factor` for contexts longer than the trained one:
 *   LINEAR  all divided by factor
 *   BASE    theta is replaced by theta * factor^(part / (part - 2)): the lowest is divided by factor, the highest kept
 *   BANDS   pairs that make more than `high` turns within `context` tokens are kept, those that make fewer than `low` are divided by
 *           factor, and between them the share kept is linear in the number of turns
 *   RAMP    as BANDS, but the share kept is linear in the number of the pair, between the (rounded) pairs that make `high` and
 *           `low` turns; the result is multiplied by 0.1 ln(factor) + 1 (queries and keys alike)                          */
typedef enum {
  CONQUR_SCALE_NONE = 0,
  CONQUR_SCALE_LINEAR = 1,
  CONQUR_SCALE_BASE = 2,
  CONQUR_SCALE_BANDS = 3,
  CONQUR_SCALE_RAMP = 4
} conqur_rotary_scaling;

/*
 * The frequencies of a rotary plan, computed on the HOST: turns_host (HOST, part/2 doubles) receives the turns (angle / 2 pi) that
 * one position adds to each pair, magnitude_host (HOST) the factor on the rotated entries.  part: even, 2 to 512.  theta > 1;
 * factor >= 1 (ignored for NONE); 0 < low < high and context > 0 for BANDS and RAMP (ignored otherwise); BASE needs part >= 4.
 */
conqur_status conqur_rotary_frequencies(uint32_t part, uint32_t scaling, double theta, double factor, double low, double high, double context,
                                        double* turns_host, float* magnitude_host);

typedef struct {
  conqur_heads q, k;            /* queries and keys, [tokens][heads][width]; either may be absent                        */
  conqur_heads q_out, k_out;    /* results, the same numbers of heads                                                     */
  conqur_heads q_grad, k_grad;  /* conqur_qk_norm_rotary_backward only: gradients of the results                          */
  const void* q_weight;         /* norms only: `width` weights of the queries' norm, in the call's dtype                  */
  const void* k_weight;         /* ... of the keys'                                                                       */
  const int64_t* positions;     /* one per token, any value whose product with a frequency a double holds to 2^-24 turns  */
  const double* turns;          /* part/2 frequencies as conqur_rotary_frequencies gives them                             */
  uint64_t tokens;              /* below 2^31; 0: nothing is done                                                         */
  uint32_t width;               /* entries of a head, even, 2 to 512                                                      */
  uint32_t part;                /* entries that are rotated, the first of a head: even, 2 to width; the others are copied */
  uint32_t layout;              /* conqur_rotary_layout                                                                   */
  uint32_t dtype;               /* conqur_dtype of the rows and the weights                                               */
  uint32_t transposed;          /* 1 (conqur_rotary only): the transposed rotation, which takes gradients back            */
  float magnitude;              /* factor on the rotated entries                                                          */
  float eps;                    /* norms only, >= 0                                                                       */
  uint32_t reserved;
} conqur_rotary_call;

/*
 * Rotary positions: y_a = m (x_a cos t - x_b sin t), y_b = m (x_b cos t + x_a sin t) for every pair (a, b), t = position *
 * frequency (whole turns are dropped in 64 bits, so that far positions keep 32-bit angles).  32-bit arithmetic, one rounding.
 */
conqur_status conqur_rotary(const conqur_rotary_call* call, void* stream);

/*
 * Norms of queries and keys over each head, and the rotation, in one pass: y = rotary(w x / sqrt(mean x^2 + eps)), 32-bit arithmetic,
 * one rounding at the end.  With eps = 0 a row of zeros gives NaN.
 */
conqur_status conqur_qk_norm_rotary(const conqur_rotary_call* call, void* stream);

/*
 * Its gradients: q, k are the inputs of the forward call, q_grad, k_grad the gradients of its results, q_out, k_out receive the gradients
 * of q and k (an out may be the grad or the input itself), q_weight_grad and k_weight_grad (`width` floats each, overwritten) those
 * of the weights, summed over tokens and heads in 32 bits in an order that depends on the sizes alone.  workspace: 16-byte aligned,
 * at least conqur_qk_norm_rotary_workspace(width) bytes; its content does not matter.  Calls that overlap in time need one each.
 */
uint64_t conqur_qk_norm_rotary_workspace(uint32_t width);
conqur_status conqur_qk_norm_rotary_backward(const conqur_rotary_call* call, float* q_weight_grad, float* k_weight_grad, void* workspace,
                                             uint64_t workspace_bytes, void* stream);

/*
 * A paged cache of keys and values.  Page p, head h, slot t, entry e:
 *   bits 16  k: bf16 [pages][heads][page_tokens][width]      v: bf16 [pages][heads][width][page_tokens]
 *   bits 8   k: one byte [pages][heads][page_tokens][width]  v: one byte [pages][heads][width][page_tokens]
 *   bits 4   k: [pages][heads][page_tokens][width/2], v: [pages][heads][width/2][page_tokens]; byte j holds the codes of entries j (low
 *            half) and j + width/2 (high half)
 * Values lie with the tokens side by side because attention contracts over tokens.  With codes, k_scale and v_scale hold two floats
 * { step, offset } for [pages][heads][page_tokens]: the value is step * code + offset.  One range per token and head, by the zero-point
 * quantiser's definition (conqur_quant_error_zp, ratio 1) over the head's entries: step = (hi - lo) / (2^bits - 1), code = clamp(rint(y / step) + zeta),
 * zeta = -rint(lo / step), offset = -step * zeta; a constant row has step 0, code 0 and offset lo.  y / step is a division here, where the scores
 * multiply by the rounded 1 / step: next to a tie the codes may differ, not the error.  All pools 16-byte aligned.
 * A sequence's token i lies in slot i % page_tokens of page table[i / page_tokens].  A table entry outside [0, pages) names no
 * page: tokens there are not written and not seen.
 */
typedef struct {
  void* k;
  void* v;
  float* k_scale;        /* NULL for bits 16 */
  float* v_scale;
  uint64_t pages;        /* below 2^31 */
  uint32_t heads;        /* up to 65535 */
  uint32_t width;        /* 64 or 128 */
  uint32_t page_tokens;  /* a power of two, 16 to 256 */
  uint32_t bits;         /* 16, 8 or 4 */
} conqur_cache;

/* New tokens of several sequences, packed: sequence b's are [start[b], start[b + 1]) of the call's rows and become the tokens prefix[b],
 * prefix[b] + 1, ... of that sequence.  Entries are clamped to [0, tokens]; a negative count means none; tokens beyond the table's
 * row (table_columns * page_tokens) are dropped.  conqur_cache_append with more than 512 sequences: no start may lie below one before it
 * (where one does, which tokens are written is unspecified).                                                            */
typedef struct {
  const int32_t* start;      /* sequences + 1 */
  const int32_t* prefix;     /* sequences: tokens committed already, >= 0 */
  const int32_t* table;      /* [sequences][table_stride], the first table_columns of a row used */
  int64_t table_stride;
  uint32_t table_columns;
  uint32_t sequences;        /* 1 to 65535 */
} conqur_batch;

typedef struct {
  conqur_cache cache;
  conqur_batch batch;
  conqur_heads k, v;                /* bf16, [tokens][cache.heads][width] */
  conqur_heads k_values, v_values;  /* optional (heads 0: not wanted; codes only): what the cache holds of them, rounded to bf16 */
  uint64_t tokens;                  /* rows of k and v, below 2^31; 0: nothing is done */
} conqur_append_call;

/*
 * Put new keys and values into the cache, and optionally write out the values that it holds of them (what a quantisation-aware stream goes
 * on with, Sec. 3.4).  Tokens of no sequence leave their rows of k_values / v_values as they are.  A row with a NaN or an infinity, or
 * whose hi - lo is beyond fp32, gets an unspecified pair and codes.  Two sequences must not share a page that either appends to.
 */
conqur_status conqur_cache_append(const conqur_append_call* call, void* stream);

typedef struct {
  conqur_cache cache;
  conqur_batch batch;
  conqur_heads q, out;       /* bf16, [tokens][heads][width]; heads a multiple of cache.heads, at most 64 times it: query head j reads
                                head j / (heads / cache.heads) of the cache.  out may be q                                */
  const uint64_t* mask;      /* one per token: bit j is set if the token sees new token j of its sequence.  NULL: a chain, every token sees
                                itself and those before it                                                                */
  uint64_t tokens;           /* rows of q, below 2^31; 0: nothing is done */
  uint64_t max_context;      /* largest prefix + count of a sequence, below 2^31 (at most table_columns * page_tokens is used); tokens of a
                                sequence beyond it are not seen                                                           */
  void* workspace;           /* 16-byte aligned, conqur_tree_attention_workspace bytes; its content does not matter.  Calls that overlap
                                in time need one each                                                                     */
  uint64_t workspace_bytes;
  uint32_t max_query;        /* largest count of new tokens of a sequence, 1 to 64; tokens beyond it get no result (their rows of
                                `out` stay as they are)                                                                   */
  float scale;               /* on the scores, finite */
} conqur_tree_call;

/*
 * Attention of new tokens over a cache that holds them already (conqur_cache_append first): token i of a sequence sees all `prefix`
 * committed tokens and those new ones that its mask names, for drafted tokens its ancestors in their tree and itself; one token per
 * sequence is plain decoding.  out = sum_j p_j v_j / sum_j p_j, p_j = exp(scale (q k_j - max)), over the tokens seen; what is not
 * seen has no influence, whatever it holds.  A token that sees nothing, or whose every score is -inf, gets zeros.  Scores, maxima, sums and
 * results in 32 bits; the weights p (times the step, with codes) are rounded to bf16 as factors of the second product.
 */
uint64_t conqur_tree_attention_workspace(const conqur_tree_call* call);
conqur_status conqur_tree_attention(const conqur_tree_call* call, void* stream);

/* Device times (ms) of the most recent call of each kind, measured with HIP events on the
 * context's stream.  level 0: off.  level 1: one event pair around each whole call (what a
 * caller's pipeline sees: the call's kernels run back to back).  level 2: additionally one
 * pair per stage -- the records between the kernels keep one kernel's launch from
 * overlapping the previous kernel's tail, so the stages sum to more than the whole call --
 * and the clock probes of conqur_get_clock_probe.  out_host: HOST, 12 floats:
 * [0] step: prepare (norms + transposed operand)  [1] step: rotate+corner GEMM (a per-head step of one launch: all of it)
 * [2] step: accumulate GEMM                       [3] step: statistics reduction
 * [4] update: whole polar update                  [5] quant: rotate GEMM
 * [6] quant: error kernel                         [7] whole conqur_step_batch
 * [8] whole conqur_quant_error (device part)      [9..11] reserved (0)
 * Entries whose events were not recorded at the current level are 0.                       */
conqur_status conqur_set_timing(conqur_ctx* ctx, int level);
conqur_status conqur_get_timing(conqur_ctx* ctx, float* out_host);

/* Clock probe of the two GEMM launches of the most recent conqur_step_batch that ran with timing
 * level 2: means over the launch's workgroups.  out_host: HOST, 8 floats:
 * [0] shader clock (MHz) sustained during the rotate+corner GEMM's main loop  [1] its main-loop time (us)
 * [2] its prologue (first operand tiles arriving) (us)      [3] its epilogue (us)
 * [4..7] the same for the accumulate GEMM.  Zeros if no probe was taken.  Synchronises.           */
conqur_status conqur_get_clock_probe(conqur_ctx* ctx, float* out_host);

/* Environment: CONQUR_TRACE (set to anything) makes conqur_update_rotation print one line per polar step to stderr
 * (interval, coefficients, measured and predicted residuals) and measure a few quantities it otherwise skips; results
 * are unchanged.  Nothing else is read from the environment. */

/* Last error text of this context (HOST string owned by the context; "" if none). */
const char* conqur_last_error(const conqur_ctx* ctx);

/* Release the context and all device memory it owns.  NULL is allowed. */
void conqur_destroy(conqur_ctx* ctx);

/* Library version string, e.g. "conqur-gfx950 0.1". */
const char* conqur_version(void);

#ifdef __cplusplus
}
#endif
#endif /* CONQUR_H */
