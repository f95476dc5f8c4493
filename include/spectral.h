/*
 * spectral.h -- C ABI of the per-head spectral-norm estimator and the
 * per-layer FP8 E4M3 scale factor for MI355X (gfx950).
 *
 * What it computes (arXiv 2602.18851):
 *   For every layer l and query head h, sigma_h estimates
 *   ||W^Q_h W^{K T}_{g(h)}||_2 by implicit power iteration (Sec. 4.1 and
 *   App. E, "Power Iteration for Spectral Norm Estimation"): with one
 *   persistent vector v per head,
 *       z = W^{K T} v,  u' = W^Q z,  sigma = ||u'||,  u = u'/sigma,
 *       y = W^{Q T} u,  v' = W^K y,  v = v'/||v'||,
 *   never forming the d x d product.  Grouped-query attention uses the
 *   unexpanded key weights (Sec. 4.2, Prop. "Implicit GQA power iteration"):
 *   query head h reads key head g(h) = floor(h / g), g = n_q / n_kv, and each
 *   key head's weights are read once per sweep for its whole group.
 *   The per-layer scale is Eq. "scale" (Sec. 3.4):
 *       scale_l = alpha * max_h sigma_h * (d / sqrt(d_h)) / (eta_fp8 * r_max).
 *
 * Weight layout (per layer, PyTorch Linear): wq is [n_q*d_h rows][ld],
 * wk is [n_kv*d_h rows][ld], row-major, only the first d_model columns of a
 * row are read.  Rows of head h are h*d_h .. h*d_h+d_h-1, i.e. the transpose
 * of the paper's W^Q_h in R^{d x d_h}.
 *
 * Memory and ownership: every pointer passed to spectral_step is device
 * memory owned by the caller and must stay valid until the work queued on the
 * context's stream has finished.  The library owns only the context and its
 * workspace (allocated in spectral_init, freed in spectral_destroy).
 *
 * Errors: functions return SN_OK (0) or a negative code; spectral_last_error
 * returns a thread-local message for the last failure on the calling thread.
 * Argument and shape errors are detected before anything is queued.
 * Numerical degeneracy is reported per head through sigma and iters.
 *
 * Threading: a context may be used by one host thread at a time.  Distinct
 * contexts are independent.
 */
#ifndef SPECTRAL_H
#define SPECTRAL_H

#include <stdint.h>

#if defined(__GNUC__)
#define SN_API __attribute__((visibility("default")))
#else
#define SN_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

#define SN_OK 0
#define SN_EINVAL (-1)   /* bad shape, parameter, size or alignment            */
#define SN_ENULL (-2)    /* a required pointer is NULL                          */
#define SN_EDTYPE (-3)   /* dtype is neither SN_F32 nor SN_BF16                 */
#define SN_EHIP (-4)     /* a HIP runtime call failed (message has its text)    */
#define SN_ESTATE (-5)   /* context not usable (e.g. no device)                 */

/* Weights, tokens and heads are SN_F32 or SN_BF16; 8-bit matrices (see
 * spectral_quantize_fp8) OCP E4M3FN or E5M2 codes. */
typedef enum { SN_F32 = 0, SN_BF16 = 1, SN_E4M3 = 2, SN_E5M2 = 3, SN_I8 = 4 } sn_dtype;

typedef struct {
  int32_t n_layers;    /* L >= 1                                                  */
  int32_t d_model;     /* d >= 1: model width (LayerNorm/RMSNorm width, Sec. 3.1) */
  int32_t n_q_heads;   /* n_q >= 1                                                */
  int32_t n_kv_heads;  /* n_kv >= 1, divides n_q (n_kv == n_q: multi-head)        */
  int32_t head_dim;    /* d_h: one of 8, 16, 32, 64, 128; d_h * ld * element size
                          must stay below 2^31 bytes                              */
  int32_t dtype;       /* sn_dtype of the weights; vectors are always float32     */
  int64_t ld;          /* row stride of wq and wk in elements; 0 means d_model.
                          ld * element size must be a multiple of 16 bytes.       */
} sn_shape;

typedef struct {
  float alpha;         /* calibration factor alpha > 0 (Eq. "calibrated_bound")   */
  float eta_fp8;       /* FP8 margin, 0 < eta_fp8 (the paper uses 0.8)            */
  float r_max;         /* largest finite FP8 magnitude, 448 for OCP E4M3          */
  float tol;           /* 0: run exactly n_iter iterations.  > 0: stop a head
                          after step k >= 2 once |sigma_k - sigma_{k-1}| <=
                          tol * sigma_k, with n_iter as the cap.  Where such
                          calls run sweeps (see spectral_step) and head_dim >=
                          16, the workspace then also holds the Gram matrices
                          of the tail (4096 or one per query and key head, of
                          2 d_h (d_h + 16) bytes).                                */
  int32_t q_strips;    /* column strips per head in the W_Q sweep; 0 = automatic  */
  int32_t k_strips;    /* column strips per KV head in the W_K sweep; 0 = auto.
                          A count given here keeps spectral_step on the sweeps
                          (without SN_FLAG_GRAM).                               */
  int32_t flags;       /* SN_FLAG_* bits; 0 for the defaults                      */
} sn_params;

/* Run the W_K sweeps of grouped heads on the vector ALUs even where the
 * matrix-core kernel applies (bf16 weights, d_h 64 or 128, >= 3 query heads
 * per KV head).  Results agree to rounding; the flag exists for comparison. */
#define SN_FLAG_VALU_K_SWEEP 1

/* Gram form of the same iteration, for every call of the context (without
 * the flag spectral_step chooses; see there).  For one head, ||W^Q z||^2 = z^T G_Q z
 * with G_Q = Q_h Q_h^T (d_h x d_h), and ||W^K y||^2 = y^T G_K y with
 * G_K = K_j K_j^T, so the step maps of Sec. 4.1 factor through the two Gram
 * matrices:  y = G_Q z / sigma,  z_next = G_K y / ||v'||.  One
 * sweep over all weights forms G_Q for every query head and G_K for every
 * key head on the matrix cores, the iteration runs in d_h-space, and one
 * final W_K sweep (plus one W_Q sweep when u is requested) maps the last y
 * (z) back to v (u).  The iterates, sigma, u and v are those of the sweeps
 * up to rounding; W_K is read twice and W_Q once (twice with u) per call
 * instead of once each per iteration.  The products are summed and iterated
 * in double (head_dim 128 with bf16 weights and 3 or more query heads per
 * key head, whose sweeps take vectors in two bf16 halves: iterated in
 * float).  A head whose rows cancel in Q^T z or K^T y over its steps
 * (sigma^2 or ||v'||^2 of the last one below 1/4 of its terms' squares, or
 * below 0.58 in the mean of all), where the products in d_h-space would lose
 * digits, or whose Gram matrices lie near the ends of the float range, is
 * iterated on its weights instead, by one workgroup. Needs head_dim >= 16.
 * The workspace of any context with head_dim >= 16 holds the Gram partials,
 * 4 d_h (d_h + 16) bytes per query or key head and column strip, for as many
 * key heads at a time as fit 128 MiB; the flag adds nothing to it. */
#define SN_FLAG_GRAM 2

/* Reserve the workspace of the layer-level form (spectral_step_layer): the
 * row-sweep partials, one d_h-vector per query head, the column sums (one row
 * of d_model rounded up to 64 per layer and row split, up to n_q splits on
 * small shapes) and per-layer vectors; with grouped heads and up to 1024 key
 * rows (n_kv * head_dim) per layer also the sums of each group's query rows
 * in float32, for as many layers at a time as fit 1 GiB (spectral_init goes
 * without them where they cannot be allocated; calls then read the weights
 * twice per iteration).  spectral_workspace_bytes gives the total.  spectral_step itself is
 * unaffected. */
#define SN_FLAG_LAYER 4


typedef struct sn_ctx sn_ctx;

/* Creates a context for one model shape on the current HIP device and
 * allocates its workspace and a device table of the layer pointers.
 * hip_stream is a hipStream_t (NULL = the default stream) on which every
 * later spectral_step is queued.  On success *ctx receives the handle.
 * Errors: SN_ENULL, SN_EINVAL, SN_EDTYPE, SN_EHIP. */
SN_API int spectral_init(sn_ctx** ctx, const sn_shape* shape, const sn_params* params,
                         void* hip_stream);

/* One estimation call over all layers and heads (Sec. 4.1; App. E).
 *   wq_layers  host array of n_layers device pointers, layer l -> wq of l
 *              (16-byte aligned).
 *   wk_layers  host array of n_layers device pointers to wk.
 *   v          device float32 [n_layers][n_q][d_model], in/out: the
 *              persistent right vectors.  Read as the start vectors (any
 *              nonzero finite vectors; normalised on entry), overwritten with
 *              the unit vector after the last step of each head.
 *   u          device float32 [n_layers][n_q][d_model] or NULL: receives the
 *              unit left vector u of each head's last step.
 *   n_iter     >= 1: iterations (tol == 0) or the cap (tol > 0).
 *   sigma      device float32 [n_layers][n_q]: the estimate of the last step,
 *              sigma = ||M v|| taken before v moves.
 *   scale      device float32 [n_layers]: Eq. "scale" with max_h sigma_h;
 *              NaN if any head of the layer is NaN.
 *   iters      device int32 [n_layers][n_q] or NULL: steps run per head;
 *              -1 if the start vector is zero or not finite (sigma = NaN,
 *              v unchanged, u = 0); -2 if M v = 0 (sigma = 0, v normalised
 *              start vector, u = 0).
 * With head_dim >= 16, automatic strips and no SN_FLAG_VALU_K_SWEEP, calls
 * of a fixed count n_iter >= 2, and calls with tol > 0 and n_iter > 2 over
 * 64 MiB of weights or more, run the Gram form (see SN_FLAG_GRAM), whose
 * iterates are those of the sweeps up to rounding; the others run sweeps
 * over the weights, two per iteration.
 * The call is queued asynchronously on the context's stream and never waits
 * on the host.  On the sweeps, with tol > 0 and head_dim >= 16, the first two steps (the
 * fewest the stopping rule allows) run as sweeps over all heads; then one
 * fixed sequence of launches lists the heads still running on the device,
 * forms their Gram matrices G_Q = Q_h Q_h^T and G_K = K_j K_j^T (see
 * SN_FLAG_GRAM), continues their iteration in d_h-space to the tolerance or
 * the cap, and maps the last vectors back to v (and u) with sweeps over the
 * listed heads only; the iterates are those of the sweeps up to rounding.
 * (With head_dim 8 every step runs as sweeps over all heads; stopped heads
 * leave them at once.)  The layer pointers reach the kernels through a
 * device table written by a small kernel whose launch arguments carry them:
 * an eager call rewrites it only when the pointers change; a call being
 * captured into a HIP graph always writes its own copy, so every replay
 * uses the pointers of its capture (graphs captured from one context must
 * not replay concurrently).  Every form and mode can be captured.  Weights
 * and vectors must not alias the outputs.  Errors: SN_ENULL, SN_EINVAL,
 * SN_EHIP. */
SN_API int spectral_step(sn_ctx* ctx, const void* const* wq_layers, const void* const* wk_layers,
                         float* v, float* u, int32_t n_iter, float* sigma, float* scale,
                         int32_t* iters);

/* Allocation-free variant of spectral_step, for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc).  It needs no context: shape, params
 * (SN_FLAG_LAYER ignored) and hip_stream as for spectral_init, the other
 * arguments as for spectral_step, whose results it gives bit for bit.  Its
 * workspace and layer-pointer table live in a static device array of
 * 32 MiB that each device holds from the first call on it until the process
 * ends; a shape whose workspace without the Gram form's matrices, plus 4
 * n_layers pointers rounded up to 256 bytes, does not fit is rejected with
 * SN_EINVAL before anything is queued.  The Gram form takes what is left, in
 * launches over as many key heads as fit; a shape of which not even one key
 * head fits runs the sweeps, here and with a context.  The call allocates nothing (no
 * hipMalloc, hipFree, event or allocating library routine).  Every call on
 * a device shares that device's array, which keeps the last call's
 * contents: calls that overlap on one device (queued on different streams,
 * or from several threads without ordering) race and give wrong results.
 * Errors: SN_ENULL, SN_EINVAL, SN_EDTYPE, SN_ESTATE, SN_EHIP. */
SN_API int spectral_step_noalloc(const sn_shape* shape, const sn_params* params, const void* const* wq_layers,
                                 const void* const* wk_layers, float* v, float* u, int32_t n_iter, float* sigma,
                                 float* scale, int32_t* iters, void* hip_stream);

/* The layer-level estimator exactly as the paper prints it (App. E,
 * "Implicit GQA Power Iteration"; g = 1 is the multi-head algorithm of
 * Sec. 4.1): one pair u, v in R^d per layer for the concatenated
 * W^Q = [W^Q_1 .. W^Q_{n_q}] and the key weights expanded implicitly,
 *     z = RepeatBlocks(W^{K T} v, g),  u' = W^Q z,  sigma = ||u'||,
 *     y = W^{Q T} u,  v' = W^K SumGroups(y, g),  v = v'/||v'||,
 * so sigma estimates || sum_h W^Q_h W^{K T}_{g(h)} ||_2 for the whole layer
 * (not max_h of the per-head norms that spectral_step returns).  Needs a
 * context created with SN_FLAG_LAYER (else SN_ESTATE).
 *   wq_layers, wk_layers  as for spectral_step.
 *   v      device float32 [n_layers][d_model], in/out: the persistent right
 *          vector of each layer (normalised on entry, unit vector on exit).
 *   u      device float32 [n_layers][d_model] or NULL: the unit left vector.
 *   n_iter >= 1 iterations (fixed count; params.tol does not apply).
 *   sigma  device float32 [n_layers]: the estimate of the last step.
 *   scale  device float32 [n_layers]: Eq. "scale" with that sigma.
 * A layer whose start vector is zero or not finite gets sigma = scale = NaN,
 * v unchanged and u = 0; one with M v = 0 gets sigma = scale = 0, v the
 * normalised start vector and u = 0.  Queued on the context's stream; never
 * waits.  Errors: SN_ENULL, SN_EINVAL, SN_ESTATE, SN_EHIP. */
SN_API int spectral_step_layer(sn_ctx* ctx, const void* const* wq_layers, const void* const* wk_layers,
                               float* v, float* u, int32_t n_iter, float* sigma, float* scale);

/* ---- FP8 E4M3 consumer of the scale ----------------------------------
 *
 * Stage 3 of the geometry-aware forward pass (Sec. 3.4, Algorithm
 * "Geometry-Aware Attention Forward Pass") up to the quantised logits, for
 * every layer l and query head h:
 *     Q = X_l W^Q,  K = X_l W^K,  S_h = Q_h K_{g(h)}^T / sqrt(d_h),
 *     S~_h = S_h / scale_l  ->  OCP E4M3FN codes (round to nearest even;
 *                              |S~| > 464 gives NaN, 0x7F | sign),
 * with the statistics of Sec. 1 (overflow when |S~| > 448) and Table
 * "pretrained" (largest scaled logit).  Key heads are not expanded.  The
 * projections accumulate in fp32 and the logits are formed to about 2^-15
 * relative precision (three bf16 matrix-core products on hi/lo halves).
 * Needs bf16 weights and tokens and head_dim 16, 32, 64 or 128.
 *
 * spectral_logits_workspace_bytes: device scratch the call needs: a table
 * of 3 n_layers device pointers (padded to 256 bytes), then the Q and K of
 * every layer as hi and lo bf16 planes (n_layers * seq_len * (n_q + n_kv) *
 * head_dim * 4 bytes).  One launch of each kernel covers all layers.
 *
 * spectral_logits_fp8:
 *   x_layers   host array of n_layers device pointers: tokens of layer l,
 *              bf16 [seq_len][ld_x] (ld_x = 0: d_model), 16-byte aligned.
 *   wq_layers, wk_layers  as for spectral_step.
 *   scale      device float32 [n_layers] (e.g. spectral_step's output).
 *   workspace  device scratch of >= workspace_bytes bytes, 256-byte aligned,
 *              owned by the caller; contents are overwritten.
 *   codes      device uint8 [n_layers][n_q][seq_len][seq_len] or NULL
 *              (16-byte aligned): E4M3 codes of S~, row i, column j.
 *   max_abs    device float32 [n_layers][n_q]: max |S~| per head.
 *   n_over     device int32 [n_layers][n_q]: #{(i, j): |S~_ij| > 448}.
 * A scaled logit that is not finite (a NaN or zero scale) counts as an
 * overflow and makes max_abs non-finite (NaN for a NaN scale).
 * Queued on the context's stream; allocates nothing; seq_len <= 46340, and
 * one layer's W_Q (n_q * head_dim rows of ld bf16) below 4 GiB (else
 * SN_EINVAL).  The layer pointer table is written into the workspace by a
 * kernel whose launch arguments carry the pointers, so the call can be
 * captured into a HIP graph.
 * Errors: SN_ENULL, SN_EINVAL, SN_EDTYPE, SN_ESTATE. */
SN_API int spectral_logits_workspace_bytes(const sn_shape* shape, int32_t seq_len, int64_t* bytes);
SN_API int spectral_logits_fp8(sn_ctx* ctx, const void* const* x_layers, int64_t ld_x, int32_t seq_len,
                               const void* const* wq_layers, const void* const* wk_layers, const float* scale,
                               void* workspace, int64_t workspace_bytes, uint8_t* codes, float* max_abs,
                               int32_t* n_over);

/* ---- 8-bit matrices with a scale for each block of 128 ----------------
 *
 * A matrix X [rows][cols] in 8 bits is codes [rows][ld] (ld a multiple of 16,
 * at least cols) and float32 scales, one for each 128 consecutive columns of
 * a row ("rows", block_rows 1) or of 128 consecutive rows ("tiles",
 * block_rows 128):  X[r][c] = code[r][c] * scale[c / 128][r / block_rows].
 * Blocks at the edges are smaller.  Scales are stored column block first.
 *
 * spectral_quantize_fp8 forms them from x, in either direction or both from
 * one reading of x.  A block's scale is the smallest power of two, 2^-126 at
 * least, with max |x| / scale <= R (448 for SN_E4M3, 57344 for SN_E5M2), so
 * x / scale is exact and a code is x / scale rounded once, to nearest even.  A
 * block that holds an infinity or a NaN gets scale and codes NaN.
 *   x          device [rows][ld_x] (ld_x = 0: cols) of dtype SN_F32 or
 *              SN_BF16, any alignment of the type.
 *   format     SN_E4M3 or SN_E5M2.
 *   tiles      0: a scale per row and 128 columns (in the transpose: per
 *              column of x and 128 rows); 1: per 128 x 128 tile.
 *   row_codes  device [rows][ld_row] or NULL: codes of x; row_scale
 *              [ceil(cols / 128)][rows or ceil(rows / 128)].
 *   col_codes  device [cols][ld_col] or NULL: codes of x transposed; col_scale
 *              [ceil(rows / 128)][cols or ceil(cols / 128)].
 * Code rows are 16-byte aligned; ld_row and ld_col are multiples of 16 not
 * below cols and rows.  Codes are written up to the next multiple of 16
 * columns, zeros past the last.  One of row_codes and col_codes is required,
 * each with its scale.  Outputs must not overlap x or each other.  rows x cols
 * stays below 2^24 tiles of 128 x 128; rows = 0 or cols = 0 does nothing.  Errors:
 * SN_ENULL, SN_EINVAL, SN_EDTYPE, SN_ESTATE, SN_EHIP.
 *
 * These calls and spectral_rotary need no context: they queue on hip_stream
 * (NULL: the default stream), which has to belong to the current HIP device (else
 * SN_ESTATE), allocate nothing, never wait, and can be captured into a HIP
 * graph.  The pointers are of that device; this is not checked. */
SN_API int spectral_quantize_fp8(const void* x, int64_t rows, int64_t cols, int64_t ld_x, int32_t dtype,
                                 int32_t format, int32_t tiles, uint8_t* row_codes, int64_t ld_row,
                                 float* row_scale, uint8_t* col_codes, int64_t ld_col, float* col_scale,
                                 void* hip_stream);

/* C = A B^T of two such matrices, A [m][k] and B [n][k]:
 *     C[i][j] = sum_b sA[b][i / ra] sB[b][j / rb] sum_{c in block b} A[i][c] B[j][c],
 * the inner sums on the matrix cores, the outer in float32, rounded once to
 * C's type.  With C in SN_F32 the products are exact and summed in float32.  With
 * C in SN_BF16 the matrix cores may add them in eights, each kept to 2^-13 of its
 * eight's largest (a normal block's sum to 1.5e-5 of itself), at twice the rate;
 * where the terms cancel to less than 2^-5 of their size and that shows, take
 * SN_F32 and round.  Which kernel runs (spectral_matmul_fp8_kernel), and so the
 * last bits of a row of C, depends on m, n and k; the same call gives the same bits.
 * The three products of a linear layer y = x W^T are of this form:
 * y from x by rows and W by tiles, dx = dy W from dy by rows and W's
 * transpose by tiles, dW = dy^T x from the transposes of dy and x.
 * The products sA sB are formed in float32, before they meet the inner sums: they
 * have to stay below its largest value, and below 2^-126 (its smallest normal
 * value) they lose digits, below 2^-149 their block's share of C.  Every row of
 * codes, the last one too, holds k rounded up to 16 bytes; those past
 * column k are not used. */
typedef struct {
  int64_t m, n, k;          /* >= 0 (k = 0: C is zero); m x n below 2^22 tiles of
                               128 x 128, k below 2^22 - 128                          */
  int32_t a_type;           /* SN_E4M3, SN_E5M2; or SN_F32, SN_BF16: A is a plain
                               matrix [m][ld_a] that the call quantises by rows to
                               E4M3 on its way, bit for bit as
                               spectral_quantize_fp8 does                             */
  int32_t b_type;           /* SN_E4M3 or SN_E5M2                                     */
  int32_t c_type;           /* SN_F32 or SN_BF16                                      */
  int32_t a_block_rows;     /* rows that share a scale, 1 or 128 (plain A: 1)         */
  int32_t b_block_rows;
  int64_t ld_a, ld_b, ld_c; /* row strides in elements; 0 means k (plain A), k
                               rounded up to 16 (codes), n (C).  Code rows are
                               multiples of 16 bytes and below 2^22.                  */
  int64_t sa_block, sa_row; /* strides of sA in elements, from a column block to the
                               next and from a row (tile) to the next; both 0: dense;
                               one scale for all of A: both SN_STRIDE_ZERO            */
  int64_t sb_block, sb_row;
} sn_matmul;

#define SN_STRIDE_ZERO (-((int64_t)1 << 62))

/* Device scratch (256-byte aligned) that the call needs, possibly 0: the codes
 * and scales of a plain A, and float32 parts of C where the sum over k is
 * split over workgroups.  Errors: SN_ENULL, SN_EINVAL, SN_EDTYPE. */
SN_API int spectral_matmul_fp8_workspace_bytes(const sn_matmul* p, int64_t* bytes);

/* Which kernel the call runs (beside launches that quantise a plain A
 * first or join parts), for labelling profiles and for tests: its kind, into how
 * many parts the sum over k is split, and its launch; zeros where m or n is 0.
 * Errors: SN_ENULL, SN_EINVAL, SN_EDTYPE. */
typedef enum {
  SN_MATMUL_FEW_ROWS = 1, /* B once, from memory to registers             */
  SN_MATMUL_TILE_4 = 2,   /* tiles of 128 x 128 by 4 waves                */
  SN_MATMUL_TILE_8 = 3,   /* ... by 8 waves, one to a compute unit        */
  SN_MATMUL_WIDE = 4,     /* 256 x 128, large results in SN_F32           */
  SN_MATMUL_BIG = 5,      /* 256 x 256, large results in SN_BF16 (8-bit
                             integers: in either type)                   */
  SN_MATMUL_SMALL = 6     /* 64 x 64, 8-bit integers                      */
} sn_matmul_kernel;
SN_API int spectral_matmul_fp8_kernel(const sn_matmul* p, int32_t* kernel, int32_t* parts, int64_t* workgroups,
                                      int32_t* threads);

/* Codes are 16-byte aligned, scales and C aligned to their type; sa is NULL
 * for a plain A.  C must not overlap the inputs.  Calls that can run at the
 * same time need workspaces of their own, graphs captured from them too.
 * Errors: SN_ENULL, SN_EINVAL, SN_EDTYPE, SN_ESTATE, SN_EHIP. */
SN_API int spectral_matmul_fp8(const sn_matmul* p, const void* a, const float* sa, const void* b, const float* sb,
                               void* c, void* workspace, int64_t workspace_bytes, void* hip_stream);

/* ---- 8-bit integers with a scale for each row -------------------------
 *
 * A matrix X [rows][cols] in 8-bit integers is codes [rows][ld] (ld a multiple of
 * 16, at least cols) and a float32 scale for each row (a token of activations, an
 * output channel of a weight):  X[r][c] = code[r][c] * scale[r].
 *
 * spectral_quantize_int8 forms them from x: a row's scale is max |x| / 127,
 * rounded to float32, 2^-126 at least; a code is x / scale rounded to the nearest
 * whole number, ties to even, from -127 to 127.  A row that holds an
 * infinity or a NaN gets scale NaN and codes zero.
 *   x      device [rows][ld_x] (ld_x = 0: cols) of dtype SN_F32 or SN_BF16, any
 *          alignment of the type.
 *   codes  device [rows][ld], rows 16-byte aligned; written up to the next
 *          multiple of 16 columns, zeros past the last.
 *   scale  device [rows].
 * Outputs must not overlap x or each other.  rows = 0 does nothing.  Errors:
 * SN_ENULL, SN_EINVAL, SN_EDTYPE, SN_ESTATE, SN_EHIP.  These calls and those of
 * the cache below need no context either: see spectral_quantize_fp8. */
SN_API int spectral_quantize_int8(const void* x, int64_t rows, int64_t cols, int64_t ld_x, int32_t dtype,
                                  int8_t* codes, int64_t ld, float* scale, void* hip_stream);

/* C = A B^T of two such matrices, A [m][k] and B [n][k]:
 *     C[i][j] = sA[i] sB[j] sum_c A[i][c] B[j][c],
 * the sum exact in 32 bits, rounded to float32 and multiplied by the product of the scales (rounded
 * too); then rounded to C's type.  Every kernel gives the same bits.  Scales are any float32;
 * their product may leave float32's range where C does not.  Codes may be
 * -128.  Every row of codes, the last one too, holds k rounded up to 16 bytes;
 * those past column k are not used. */
typedef struct {
  int64_t m, n, k;          /* >= 0 (k = 0: the sums are zero); m x n below 2^22 tiles of
                               128 x 128, k below 2^17                              */
  int32_t a_type;           /* SN_I8; or SN_F32, SN_BF16: A is a plain matrix [m][ld_a]
                               that the call quantises on its way, bit for bit as
                               spectral_quantize_int8 does                          */
  int32_t c_type;           /* SN_F32 or SN_BF16                                    */
  int64_t ld_a, ld_b, ld_c; /* row strides in elements; 0 means k (plain A), k
                               rounded up to 16 (codes), n (C).  Code rows are
                               multiples of 16 bytes and below 2^22.                */
  int64_t sa_row, sb_row;   /* strides of the scales in elements; 0: one after the
                               other; one scale for all rows: SN_STRIDE_ZERO        */
} sn_matmul_int8;

/* Device scratch (256-byte aligned) that the call needs, possibly 0: the codes
 * and scales of a plain A, and parts of the sums where they are split over
 * workgroups.  Errors: SN_ENULL, SN_EINVAL, SN_EDTYPE. */
SN_API int spectral_matmul_int8_workspace_bytes(const sn_matmul_int8* p, int64_t* bytes);

/* Which kernel the call runs, as spectral_matmul_fp8_kernel. */
SN_API int spectral_matmul_int8_kernel(const sn_matmul_int8* p, int32_t* kernel, int32_t* parts, int64_t* workgroups,
                                       int32_t* threads);

/* Codes are 16-byte aligned, scales and C aligned to their type; sa is NULL
 * for a plain A.  C must not overlap the inputs.  Calls that can run at the
 * same time need workspaces of their own, graphs captured from them too.
 * Errors: SN_ENULL, SN_EINVAL, SN_EDTYPE, SN_ESTATE, SN_EHIP. */
SN_API int spectral_matmul_int8(const sn_matmul_int8* p, const void* a, const float* sa, const int8_t* b,
                                const float* sb, void* c, void* workspace, int64_t workspace_bytes, void* hip_stream);

/* ---- a cache of keys and values in 8 bits -------------------------------
 *
 * Places of tokens, in pages: codes [pages][heads][page][head_dim] and float32
 * scales [pages][heads][page], of keys and of values.  A row, the head_dim elements
 * of one place and head, has one scale, a power of two from 2^-126 on (or NaN):
 * element e is code[e] * scale.  Slot n is place n % page of page n / page.
 * Other scales are not looked for: spectral_cache_read multiplies by whatever is there,
 * spectral_cache_attend takes its power of two alone, and 1.5 is 1 to it. */
typedef struct {
  void* k;             /* codes of keys, 16-byte aligned                             */
  float* k_scale;      /* their scales, 16-byte aligned                              */
  void* v;             /* the same of values                                         */
  float* v_scale;
  int64_t pages;       /* >= 0, below 2^31                                           */
  int32_t heads;       /* 1 .. 65536                                                 */
  int32_t page;        /* places of a page, a power of two, 16 .. 65536; heads * page
                          below 2^31                                                 */
  int32_t head_dim;    /* a multiple of 16, 16 .. 256                                */
  int32_t format;      /* SN_E4M3 or SN_E5M2                                         */
  int64_t code_page;   /* elements from a page's codes to the next one's, and from its
                          scales; multiples of 16 and 4; 0: dense                    */
  int64_t scale_page;
} sn_cache;

/* Writes the keys and values of tokens to their slots: a row's scale is the smallest
 * power of two, 2^-126 at least, with max |x| / scale <= R (448 or 57344), and a
 * code x / scale rounded to nearest even; a row that holds an infinity or a
 * NaN gets scale and codes NaN.
 *   dtype  SN_F32 or SN_BF16: of k and v, element e of head h of token t at
 *          t * token + h * head + e (strides in elements, any alignment of the type).
 *   slots  device int64 [tokens]; a token whose slot is not in [0, pages * page) is
 *          padding and not written.  The others differ: of tokens with the same slot the
 *          place holds some mixture.
 * spectral_cache_read is the way back: code * scale rounded to dtype; zeros for a
 * slot outside.  Its results' rows must not overlap (else SN_EINVAL).  tokens = 0 does
 * nothing; tokens * heads stays below 2^31.  Errors: SN_ENULL, SN_EINVAL, SN_EDTYPE,
 * SN_ESTATE, SN_EHIP. */
SN_API int spectral_cache_write(const sn_cache* cache, int32_t dtype, int64_t tokens, const void* k, int64_t k_token,
                                int64_t k_head, const void* v, int64_t v_token, int64_t v_head, const int64_t* slots,
                                void* hip_stream);
SN_API int spectral_cache_read(const sn_cache* cache, int32_t dtype, int64_t tokens, const int64_t* slots, void* k,
                               int64_t k_token, int64_t k_head, void* v, int64_t v_token, int64_t v_head,
                               void* hip_stream);

/* Attention of the last `drafts` tokens of each sequence over the cache, theirs
 * among it:  out = softmax(scale q K^T) V  over the places that a token sees.  A
 * sequence of n places has them in the pages of its row of the table, in order; the last
 * `drafts` of them are the drafted tokens' (with fewer places, the first drafted
 * tokens have none).  Every token sees all places before these, and of these
 *   masks NULL: those of the drafted tokens up to itself;
 *   else: drafted token j where bit j of its mask is set (a tree: its ancestors and itself).
 * A token that sees nothing gets zeros.  A place whose page is not in [0, pages)
 * is not seen.  Query head h reads head h / (q_heads / heads) of the cache.  What a
 * place holds that a token does not see, NaN and infinities too, does not
 * reach its result.  A NaN that it sees, as spectral_cache_write makes of a row that is
 * not finite, does: of a key it makes the whole result NaN, of a value its element.
 * Infinities are codes of SN_E5M2 that spectral_cache_write never stores, and elements that it
 * rounds to 2^128 (|x| from 1.9375 2^127 on, with SN_E5M2 1.875).  Of a value that is seen they
 * make its element NaN or an infinity; of a key the whole result NaN or, where the
 * logit is minus infinity, a weight of zero.
 *   q        device, element e of head h of drafted token i of sequence b at
 *            b * q_batch + i * q_draft + h * q_head + e; out the same.
 *   table    device int32 [batch][table_ld] (0: table_cols), page numbers.
 *   lengths  device int32 [batch], taken between 0 and table_cols * page.
 *   masks    device int64 [batch][drafts] (mask_batch elements apart; 0: one
 *            for all sequences), or NULL.
 * Queries in SN_F32 are held to 2^-24 and the weights to 2^-24 of a row's
 * largest; with SN_BF16 the weights to 2^-16.  Sums are float32.  The
 * same call gives the same bits.  Calls that can run at the same time need
 * workspaces of their own, graphs captured from them too; the workspace depends on the sizes
 * here, not on lengths, which a graph may change between replays.  batch = 0 does nothing.  batch *
 * table_cols * page * heads stays below 2^36 (with drafts * q_heads / heads above 64 or so: by
 * their 64th or 256th part less). */
typedef struct {
  int32_t dtype;       /* SN_F32 or SN_BF16, of q and out                            */
  int32_t batch;       /* 0 .. 2^20                                                  */
  int32_t drafts;      /* 1 .. 64 tokens of each sequence                            */
  int32_t q_heads;     /* a multiple of the cache's heads                            */
  int32_t table_cols;  /* pages of the longest sequence; times page below 2^31 - 128 */
  float scale;         /* positive, below 2e38                                       */
  int64_t q_batch, q_draft, q_head;
  int64_t out_batch, out_draft, out_head;
  int64_t table_ld, mask_batch;
} sn_attend;

/* Device scratch (256-byte aligned) that the call needs, possibly 0: parts of results, and above 256 sequences
 * how they are shared out.  Errors: SN_ENULL, SN_EINVAL, SN_EDTYPE. */
SN_API int spectral_cache_attend_workspace_bytes(const sn_cache* cache, const sn_attend* p, int64_t* bytes);

/* Errors: SN_ENULL, SN_EINVAL, SN_EDTYPE, SN_ESTATE, SN_EHIP. */
SN_API int spectral_cache_attend(const sn_cache* cache, const sn_attend* p, const void* q, const int32_t* table,
                                 const int32_t* lengths, const int64_t* masks, void* out, void* workspace,
                                 int64_t workspace_bytes, void* hip_stream);

/* ---- rotary positions -------------------------------------------------
 *
 * Turns pairs (x0, x1) of the first rot_dim elements of every head by the
 * angle p f_i of the token's position p and the pair's frequency f_i:
 *     (x0 cos - x1 sin, x0 sin + x1 cos) * amplitude,
 * and leaves the rest as it is.  Rotations are orthogonal, so the bounds on the
 * logits hold unchanged (Sec. 3.3).  inverse != 0 turns back, which with the
 * same amplitude is the gradient. */
typedef enum { SN_ROTARY_HALF = 0,         /* pair i is elements i and i + rot_dim / 2 */
               SN_ROTARY_INTERLEAVED = 1   /* pair i is elements 2 i and 2 i + 1       */
} sn_rotary_layout;

/* f_i = base^(-2 i / rot_dim), for positions beyond a trained length T:
 *   SN_ROTARY_LINEAR  f_i / factor
 *   SN_ROTARY_BASE    base * factor^(rot_dim / (rot_dim - 2)) in the place of base
 *   SN_ROTARY_INDEX   f_i (1 - r) + f_i / factor r, r from 0 to 1 in i between
 *                     floor(j(high)) (0 at least) and ceil(j(low)) (rot_dim - 1
 *                     at most), j(t) = rot_dim ln(T / (2 pi t)) / (2 ln base)
 *                     the index with t turns over T; amplitude 1 + 0.1 ln factor
 *   SN_ROTARY_TURNS   the same mix with 1 - r from 0 to 1 in the turns T f_i / 2 pi
 *                     between low and high; amplitude 1 */
typedef enum { SN_ROTARY_NONE = 0, SN_ROTARY_LINEAR = 1, SN_ROTARY_BASE = 2, SN_ROTARY_INDEX = 3,
               SN_ROTARY_TURNS = 4 } sn_rotary_scaling;

typedef struct {
  int32_t head_dim;   /* 2 .. 1024                                             */
  int32_t rot_dim;    /* even, 2 .. min(head_dim, 256)                         */
  int32_t layout;     /* sn_rotary_layout                                      */
  int32_t scaling;    /* sn_rotary_scaling                                     */
  double base;        /* > 1                                                   */
  double factor;      /* >= 1; not used without scaling                        */
  double low, high;   /* 0 < low < high, turns over T; INDEX and TURNS only    */
  int64_t trained;    /* T >= 1; INDEX and TURNS only                          */
} sn_rotary;

/* The rot_dim / 2 angles per position (radians) and the amplitude, to float32, of
 * a plan (host doubles).  Errors: SN_ENULL, SN_EINVAL. */
SN_API int spectral_rotary_frequencies(const sn_rotary* p, double* freq, double* amplitude);

/* One tensor of heads: element e of head h of token t is at
 * t * token + h * head + e (strides in elements, any alignment of the type). */
typedef struct {
  const void* x;
  void* out;                     /* may be x itself, with the same strides; must not overlap it otherwise */
  int64_t heads;                 /* >= 0 */
  int64_t x_token, x_head;
  int64_t out_token, out_head;   /* heads within tokens (out_token >= heads * out_head) or tokens within heads
                                    (out_head >= n_tokens * out_token) */
} sn_heads;

#define SN_ROTARY_COPY_PADDING (1 << 30)

/* Turns n_heads tensors (1 or 2: queries and keys) of the same tokens in one launch.
 *   dtype      SN_F32 or SN_BF16; turned in float32 and rounded once.
 *   positions  device int64 [n_tokens], or NULL: token t is at first + t.
 *              Angles are formed and reduced in double, exact to |p| 2^-48, and
 *              their cosines and sines, times the amplitude, rounded to float32 once.  A
 *              token at a negative position is padding: its rows of out are left as
 *              they were or, with SN_ROTARY_COPY_PADDING, are x's own, not turned.
 *   inverse    0, or 1 to turn back; SN_ROTARY_COPY_PADDING may be added.
 * n_tokens = 0 does nothing.  Errors: SN_ENULL, SN_EINVAL, SN_EDTYPE, SN_ESTATE, SN_EHIP. */
SN_API int spectral_rotary(const sn_rotary* p, int32_t dtype, int64_t n_tokens, const int64_t* positions,
                           int64_t first, int32_t inverse, const sn_heads* heads, int32_t n_heads, void* hip_stream);

/* spectral_logits_fp8 with queries and keys turned by their positions before
 * the logits: S_h[i][j] = (R_i Q_h[i]) . (R_j K_{g(h)}[j]) / sqrt(d_h), on the
 * projections as the consumer holds them, float32 sums split into two bf16 halves (2^-17
 * of the value), and held so again after the turn.  rotary->head_dim is the context's.  positions: device int64
 * [seq_len], the same for every layer, or NULL (row i at position i); a row at a
 * negative position is not turned, nor, without amplitude, is one at zero.  All else
 * as spectral_logits_fp8. */
SN_API int spectral_logits_fp8_rotary(sn_ctx* ctx, const void* const* x_layers, int64_t ld_x, int32_t seq_len,
                                      const void* const* wq_layers, const void* const* wk_layers,
                                      const float* scale, const sn_rotary* rotary, const int64_t* positions,
                                      void* workspace, int64_t workspace_bytes, uint8_t* codes, float* max_abs,
                                      int32_t* n_over);

/* Redirects later calls to another hipStream_t.  Unless either stream is
 * being captured, the new stream is first made to wait for all work queued
 * on the previous one (they share the workspace and the pointer table). */
SN_API int spectral_set_stream(sn_ctx* ctx, void* hip_stream);

/* Frees the context and its workspace (waits for its queued work first). */
SN_API void spectral_destroy(sn_ctx* ctx);

/* Thread-local text of the last error ("" if none). */
SN_API const char* spectral_last_error(void);

/* Bytes of device workspace spectral_init allocates for this shape. */
SN_API int spectral_workspace_bytes(const sn_shape* shape, const sn_params* params,
                                    int64_t* bytes);

/* Per-kernel timing.  With enable != 0 every later launch is bracketed by
 * HIP events on the context's stream.  spectral_profile_read waits for the
 * stream and returns, per kernel kind (0 = first W_K sweep from v, 1 = W_Q
 * sweep, 2 = W_K sweep, 3 = finalize, 4 = Gram matrices of key heads (and of
 * split query heads), or of the tail, 5 = d_h-space iteration, with the Gram
 * matrices of the heads whose own workgroup forms them, 6 = final sweeps of
 * the Gram form, 7 = row sweeps of the layer-level form (one-pass: its W_K
 * sweeps), 8 = its column sweeps (one-pass: those over W_Q or the group
 * sums), 9 = its group sums, reductions and finalize, 10 = projections of
 * the logit consumer (and its rotary positions), 11 = its logit kernels, 12 = the running-head lists of
 * tolerance mode), the summed device time in
 * milliseconds and the number of launches since the previous read, then
 * resets both.  ms and launches point to SN_PROFILE_KINDS host elements
 * each. */
#define SN_PROFILE_KINDS 13
SN_API int spectral_profile(sn_ctx* ctx, int32_t enable);
SN_API int spectral_profile_read(sn_ctx* ctx, double* ms, int64_t* launches);

/* ---- host-side calibration helpers (no GPU involved) ------------------
 *
 * spectral_alpha_select: the selection rule of Sec. 3.2.  gamma is the
 * smallest gamma > 1 with gamma - 1 - ln(gamma) >= (2 / d_h) ln(2 N L / delta)
 * (Eq. "gamma_selection"), and alpha_min = sqrt(2 gamma d_h) / d *
 * sqrt(ln(4 N L^2 / delta)) (Eq. "alpha_selection"), with N = n_heads_total
 * (layers x query heads) and L = seq_len.  Writes both to host doubles.
 * Errors: SN_ENULL, SN_EINVAL (sizes < 1, delta outside (0, 1)). */
SN_API int spectral_alpha_select(int32_t d_model, int32_t head_dim, int64_t n_heads_total, int64_t seq_len,
                                 double delta, double* gamma, double* alpha_min);

/* T1 = L exp(-(d_h / 2)(gamma - 1 - ln gamma)), T2 = 2 L^2 exp(-d^2 alpha^2 /
 * (2 gamma d_h)) of Prop. "Rank-aware overflow probability bound", for one
 * head.  Errors: SN_ENULL, SN_EINVAL (alpha <= 0, gamma <= 1, sizes < 1). */
SN_API int spectral_overflow_terms(int32_t d_model, int32_t head_dim, int64_t seq_len, double alpha,
                                   double gamma, double* t1, double* t2);

/* Auto-alpha (Sec. 3.5, App. M): alpha = Quantile_q(slack) * kappa over n
 * burn-in slack ratios (host array), the quantile interpolating linearly
 * between order statistics at position q (n - 1).  Errors: SN_ENULL,
 * SN_EINVAL (n < 1, q outside [0, 1], kappa < 1, a negative or non-finite
 * ratio). */
SN_API int spectral_auto_alpha(const double* slack, int64_t n, double quantile, double kappa, double* alpha);

/* Slack ratio r = max|S| / B_max with B_max = sigma_layer * d / sqrt(d_h)
 * (Sec. 3.5, Eq. "bound"). */
SN_API double spectral_slack_ratio(double max_abs_logit, double sigma_layer, int32_t d_model, int32_t head_dim);

#ifdef __cplusplus
}
#endif

#endif /* SPECTRAL_H */
