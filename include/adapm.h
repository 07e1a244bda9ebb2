/*
 * adapm.h - C ABI of the AdaPM optimizer step for AMD MI355X (gfx950).
 *
 * The library applies, to every parameter block of a model, one step of the
 * paper's update (Alg. 1 "Low Rank Update with Correction"): full momentum
 * (eq. 5), no momentum (Sec. 4.1 regime 1) or bias-corrected low-rank momentum
 * (eq. 2-4, tracked by the gradient-descent solver of Alg. 2 / App. B), a
 * per-element or blockwise second moment (Alg. 1 "v_t"; blockwise mean as in the
 * Adam-mini combination of Sec. 5.1.3), and the clipped update with decoupled
 * weight decay (Alg. 1 last line).
 *
 * Conventions
 *  - Every pointer named *_dev is DEVICE memory owned by the caller; every other
 *    pointer is HOST memory.  The library owns only the context object (a host
 *    plan plus small device-side tables, released by adapm_destroy).
 *  - A block is one parameter tensor, row-major rows x cols, rows = output units;
 *    1-D tensors use cols = 1.  Block base pointers must be 16-byte aligned.
 *  - adapm_step is asynchronous on the given HIP stream and updates params and state in
 *    place; grads are read-only.  It allocates nothing once adapm_state_init has run on
 *    the context (which places the launch plan on the device), unless per-launch timing
 *    is on, and it never waits for the device: the pointer tables live on the device in a
 *    few slots keyed by their contents (a caller that rotates up to four sets of tensors
 *    uploads each once; a new set is copied on the step's stream).  Issue the steps of one
 *    context on one stream, or order the streams yourself.
 *  - Functions return ADAPM_OK (0) or a negative status; nothing aborts or throws.
 *    adapm_last_error() gives a thread-local message for the last failure.
 *  - bf16 tensors are IEEE-like bfloat16 bit patterns; stores round to nearest even.
 */
#ifndef ADAPM_H
#define ADAPM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  ADAPM_OK = 0,
  ADAPM_EINVAL = -1,   /* bad argument / table entry */
  ADAPM_ENOMEM = -2,   /* host or device allocation of the context failed */
  ADAPM_EHIP = -3,     /* a HIP runtime call failed */
  ADAPM_ESTATE = -4    /* call order / step number inconsistent */
} adapm_status_t;

/* ADAPM_E4M3 (8 bits, largest value 448) is an output type of adapm_norm_forward only. */
typedef enum { ADAPM_F32 = 0, ADAPM_BF16 = 1, ADAPM_E4M3 = 2 } adapm_dtype_t;

/* Momentum regime of a block (Sec. 4.1): none / full (eq. 5) / low-rank (Alg. 1). */
typedef enum { ADAPM_MOM_NONE = 0, ADAPM_MOM_FULL = 1, ADAPM_MOM_LOWRANK = 2 } adapm_mom_t;

/* Granularity of the second moment: per element (Alg. 1), one value per group of
 * v_group_rows consecutive rows, or one value for the whole block (Sec. 5.1.3). */
typedef enum { ADAPM_V_ELEMENT = 0, ADAPM_V_ROWGROUP = 1, ADAPM_V_WHOLE = 2 } adapm_vmode_t;

/* Arithmetic of the low-rank contractions (G R^T, L^T G, Gram matrices, L R):
 *  F64     - operands exact, fp64 accumulation on the fp64 matrix cores;
 *  BF16X2  - bf16 MFMA with fp32 accumulation, every fp32 factor operand carried
 *            as a (hi, lo) pair of bf16 values (relative operand error 2^-17);
 *            requires bf16 gradients.  Implemented for rank <= 128 (a block runs in
 *            the kernels of the next rank class 32 / 64 / 128, its factors padded
 *            with zeros on chip) and cols >= 8; any other block silently uses F64;
 *  AUTO    - per block: F64 when the block's parameters are fp32, else BF16X2. */
typedef enum { ADAPM_CONTRACT_AUTO = 0, ADAPM_CONTRACT_F64 = 1, ADAPM_CONTRACT_BF16X2 = 2 } adapm_contract_t;

typedef struct {
  int64_t rows, cols;
  int32_t param_dtype, grad_dtype; /* adapm_dtype_t */
  int32_t mom_mode;                /* adapm_mom_t */
  int32_t rank;                    /* LOWRANK only: 1 <= rank <= min(rows, cols); cols >= 2 */
  int32_t v_mode;                  /* adapm_vmode_t */
  int32_t v_group_rows;            /* ROWGROUP: rows % v_group_rows == 0 */
  float lr_scale;                  /* 1.0; the paper uses 0.75 for no-momentum blocks (Sec. 5.1) */
  float weight_decay;              /* lambda of Alg. 1 for this block */
} adapm_block_t;

typedef struct {
  float beta1, beta2, eps;    /* 0.9, 0.95, 1e-8 (Sec. 5.1) */
  float clip;                 /* element-wise clamp of Alg. 1's last line; 1.0; +inf disables */
  int32_t adam_debias;        /* 0 = Alg. 1 as printed; 1 = divide by (1-beta^t) (Adam comparison only) */
  int32_t refresh_iters_K;    /* iterations of Alg. 2; 5 (App. B) */
  int32_t refresh_period_T;   /* 1 = Alg. 2 every step (Alg. 1 verbatim).  T > 1: Alg. 2 on steps with
                                 (step-1) % T == 0, followed by a product-preserving orthonormalisation
                                 of R; on other steps L is the least-squares fit with R held.  A block
                                 whose R R^T is not positive definite at that point (R has lost rank)
                                 keeps its (L, R) as Alg. 2 left them. */
  int32_t bias_correction;    /* 1 = eq. 4; 0 = ablation of Sec. 5.1.2 (use L_t R_t as the momentum) */
  int32_t contraction;        /* adapm_contract_t */
  int32_t refresh_normalise;  /* 0 = Alg. 2 as printed.  1 (an option beyond the paper): every iteration of Alg. 2
                                 divides its step size by max(||R R^T||_F, ||L^T L||_F), which makes the
                                 iteration invariant under a rescaling of the gradients (as printed it
                                 diverges for large and stalls for small gradients) */
  uint64_t seed;              /* seeded start R_0 of the low-rank factors; 0 = literal all-zero start (the factors then
                                 stay zero for ever; only with refresh_period_T = 1, else ADAPM_EINVAL) */
} adapm_hparams_t;

typedef struct adapm_ctx adapm_ctx;

/* Validate the table and hyper-parameters, fix the state / workspace layout and build
 * the launch plan on the current HIP device.  table[0..nblocks) and hp are read during
 * the call only.  On failure *out is NULL. */
adapm_status_t adapm_init(adapm_ctx** out, const adapm_block_t* table, int64_t nblocks,
                          const adapm_hparams_t* hp);

/* Size of the caller-allocated optimizer state: per block, in table order,
 * [L (rows x rank) | R (rank x cols)] or [m (rows x cols)] or nothing, then v;
 * fp32, each sub-buffer 256-byte aligned (Alg. 1, initialisation).  0 if ctx is NULL. */
size_t adapm_state_bytes(const adapm_ctx* ctx);

/* Size of the caller-allocated scratch buffer used inside adapm_step (previous
 * factors, thin products, Gram matrices, partial sums).  With refresh_period_T > 1 the
 * library also keeps bf16 copies of R there between two runs of Alg. 2: pass the same,
 * unmodified buffer on consecutive steps (a different workspace or state pointer is detected
 * and the copies are rebuilt from that state; overwriting the contents of either buffer
 * between steps is not, see adapm_state_loaded). */
size_t adapm_workspace_bytes(const adapm_ctx* ctx);

/* Byte offsets into the state buffer of block `block`'s sub-buffers; an absent
 * sub-buffer reports (size_t)-1.  Any of L, R, m, v may be NULL. */
adapm_status_t adapm_state_offsets(const adapm_ctx* ctx, int64_t block, size_t* L, size_t* R,
                                   size_t* m, size_t* v);

/* Zero the state and write the seeded R_0 (Alg. 1, initialisation, with L_0 R_0 = 0).
 * Asynchronous on `stream` (a hipStream_t, or NULL for the default stream). */
adapm_status_t adapm_state_init(adapm_ctx* ctx, void* state_dev, void* stream);

/* Tell the library that the caller has overwritten the state buffer (e.g. restored a
 * checkpoint into it): anything derived from the old contents is dropped, and the state is
 * taken to come from a run with the same hyper-parameters (with refresh_period_T > 1: R with
 * orthonormal rows).  Not needed after adapm_state_init. */
adapm_status_t adapm_state_loaded(adapm_ctx* ctx);

/* One optimizer step (Alg. 1) over all blocks.
 *  params_dev / grads_dev: HOST arrays of nblocks DEVICE pointers (table order);
 *  state_dev: adapm_state_bytes() bytes; workspace_dev: adapm_workspace_bytes() bytes
 *  (may be NULL if that size is 0); step: 1-based iteration count t; lr: eta_t.
 * Checks step >= 1, non-null and 16-byte aligned pointers; everything else was
 * validated at init.  With refresh_period_T > 1, a step that holds R on a state whose R has
 * not been orthonormalised (no step that runs Alg. 2 since adapm_state_init, and no
 * adapm_state_loaded) is ADAPM_ESTATE. */
adapm_status_t adapm_step(adapm_ctx* ctx, void* const* params_dev, const void* const* grads_dev,
                          void* state_dev, void* workspace_dev, int64_t step, float lr, void* stream);

/* adapm_step for callers that cannot allocate device memory (code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc): the same step with the library's OWN scratch buffer in place of
 * workspace_dev, a fixed array in device memory of adapm_static_scratch_bytes() bytes (64 MiB) that every GPU
 * the library runs on holds until the process ends.  The call allocates nothing (no hipMalloc / hipFree, no
 * event creation): the context must have been set up by adapm_state_init beforehand (else ADAPM_ESTATE) and
 * per-launch timing must be off.  A table whose adapm_workspace_bytes() exceeds the array is ADAPM_EINVAL.
 * All contexts on a GPU share that GPU's array, which keeps whatever the last call left there: the library
 * rebuilds what a context keeps in scratch between steps when another context has used the array in the
 * meantime, and nothing in it is expected to start at zero; calls that overlap in time on one GPU (different
 * streams, different host threads) race on it and are not allowed.  Everything else as adapm_step. */
adapm_status_t adapm_step_static(adapm_ctx* ctx, void* const* params_dev, const void* const* grads_dev,
                                 void* state_dev, int64_t step, float lr, void* stream);

/* Size of the library's own scratch array (see adapm_step_static). */
size_t adapm_static_scratch_bytes(void);

/* Global gradient-norm clipping of the paper's pre-training runs (Sec. 5.1, set-ups: threshold 1.0),
 * folded into the step.  After adapm_set_grad_clip(ctx, c) with c > 0, every adapm_step first sums the
 * squares of all gradients of the table on the device (fixed order, fp64 partial sums), derives
 *     factor = min(1, c / (||G||_2 + 1e-6))
 * there, and uses factor * G wherever the method uses G (second moment, momentum, Alg. 2, update); the
 * caller's gradients are not modified and nothing is read back.  c <= 0 or +inf switches it off (the
 * default); NaN is ADAPM_EINVAL.  Costs one extra pass over the gradients. */
adapm_status_t adapm_set_grad_clip(adapm_ctx* ctx, float max_norm);

/* Norm and factor of the last clipped adapm_step that used workspace_dev (device pointer; NULL: the
 * library's own scratch array, after adapm_step_static): copies two floats to the host and synchronises
 * `stream`.  Either output may be NULL. */
adapm_status_t adapm_last_grad_norm(adapm_ctx* ctx, const void* workspace_dev, void* stream, float* norm, float* scale);

/* Learning-rate schedule of the same runs (Sec. 5.1, set-ups: cosine decay with warm-up), a host helper
 * for the `lr` argument of adapm_step: linear from 0 to peak_lr over warmup_steps, half a cosine down to
 * min_lr at total_steps, min_lr afterwards.  step counts from 1. */
float adapm_lr_cosine_warmup(int64_t step, float peak_lr, float min_lr, int64_t warmup_steps, int64_t total_steps);

/* Arithmetic the planner chose for the contractions of a block (see adapm_contract_t):
 * ADAPM_CONTRACT_F64 or ADAPM_CONTRACT_BF16X2 for a low-rank block, -1 for a block without
 * low-rank momentum or an index out of range. */
int32_t adapm_block_contraction(const adapm_ctx* ctx, int64_t block);

/* Number of kernel launches the last adapm_step enqueued (0 before the first). */
int64_t adapm_last_launch_count(const adapm_ctx* ctx);

/* Compulsory HBM bytes of one step over the table: every input read once and every
 * output written once in its storage type.  refresh_step != 0 counts a step that runs
 * Alg. 2; 0 counts a step with R held (T > 1 only). */
double adapm_algorithmic_bytes(const adapm_ctx* ctx, int32_t refresh_step);

/* Multiply-add work of the low-rank contractions of one step, in flop (2 per multiply-add),
 * counted once per mathematical product (operand splitting not counted). */
double adapm_algorithmic_flops(const adapm_ctx* ctx, int32_t refresh_step);

/* Optional per-launch timing for benchmarks.  While enabled, adapm_step brackets every kernel
 * launch with a pair of HIP events on the caller's stream (this serialises nothing but adds two
 * event records per launch).  For callers that want the duration of each kernel class without an
 * external profiler. */
adapm_status_t adapm_profile_enable(adapm_ctx* ctx, int32_t on);

/* After the caller has synchronised the stream: entry `index` of the per-kernel-class totals
 * accumulated since the last read with index 0 (which folds and clears the pending records).
 * name receives a NUL-terminated label (at most name_cap bytes), total_ms the summed duration,
 * launches the number of launches.  Returns the number of entries. */
int64_t adapm_profile_read(adapm_ctx* ctx, int64_t index, char* name, size_t name_cap, double* total_ms,
                           int64_t* launches);

/* ---- The end of a model ---------------------------------------------------------------------------------------------
 *
 * What stands between the last layer and the gradients that adapm_step reads for the two blocks a table ends with, the
 * final norm vector and the output head:
 *
 *     h = residual + dropout(x),   y = norm(h) * weight,   loss = cross entropy of y W^T,   and the way back.
 *
 * These calls need no context.  Like adapm_step they are asynchronous on the given stream of the CURRENT device,
 * allocate nothing, never wait for the device and keep nothing between calls: they may be captured into a HIP graph, and
 * calls on different streams may overlap if their outputs and workspaces differ.  Sums are held in fp32 or fp64 and added
 * in a fixed order: the same inputs give the same bits.  rows = 0 is allowed everywhere. */

/* A matrix of activations or weights: row r starts at data + r * stride elements (stride >= the row's length; any
 * alignment to whole elements).  data = NULL: absent, where that is allowed. */
typedef struct {
  void* data;
  int64_t stride;
} adapm_rows_t;

/* Dropout by a counter-based generator (Philox4x32-10): whether element (row, column) is kept depends on seed, offset, row and
 * column alone, so the backward pass makes the same mask again and no mask is ever stored.  The probability is rounded
 * to a multiple of 2^-16 (at most 65535 / 65536); what is kept is divided by one minus that.  What is dropped becomes 0
 * whatever it was.  offset_dev (DEVICE, may be NULL) is added to offset: a captured graph whose replays have to draw new masks
 * reads its counter there. */
typedef struct {
  uint64_t seed, offset;
  const uint64_t* offset_dev;
  float p;                         /* 0 <= p < 1 */
  int32_t reserved;                /* 0 */
} adapm_dropout_t;

/* y = residual + dropout(x), rounded once; residual.data may be NULL.  The gradient of x is the same call on the gradient of
 * y, without residual.  y may be x or residual. */
adapm_status_t adapm_dropout(adapm_rows_t y, adapm_rows_t x, adapm_rows_t residual, int64_t rows, int64_t cols, int32_t dtype,
                             const adapm_dropout_t* drop, void* stream);

/* Root-mean-square norm with the residual's addition. */
typedef struct {
  int64_t rows, cols;              /* 1 <= cols <= 16384 */
  int32_t dtype;                   /* x, residual, h and all gradients but dweight: F32 or BF16 */
  int32_t weight_dtype;            /* F32 or BF16 */
  int32_t y_dtype;                 /* forward: dtype, or ADAPM_E4M3 */
  int32_t grad_dtype;              /* backward: dweight, F32 or BF16 */
  float eps;
  int32_t reserved;                /* 0 */
} adapm_norm_t;

/* h = residual + dropout(x) in dtype, rstd = 1 / sqrt(mean(h^2) + eps) (fp32, one a row), y = h * rstd * weight.
 * residual.data and drop may be NULL; with neither, h.data may be NULL and the h of the backward pass is x itself.
 * The squares and their sum are fp32: |h| up to 1e17 is in range in rows of any length (a sum past 3.4e38 gives rstd = 0, y = 0), and
 * with eps = 0 rows whose largest value is 1e-16 or more (a row of zeros is NaN then).
 * y_dtype = ADAPM_E4M3: y holds 8-bit values and y_scale[row] = max|row| / 448 (1 for a row of zeros, at least 2^-126 for any
 * other; NaN does not count) is what they are multiplied by.  h may be x or residual; y overlaps none of the others. */
adapm_status_t adapm_norm_forward(const adapm_norm_t* n, adapm_rows_t x, adapm_rows_t residual, adapm_rows_t h,
                                  const void* weight_dev, adapm_rows_t y, float* y_scale_dev, float* rstd_dev,
                                  const adapm_dropout_t* drop, void* stream);

/* Scratch of adapm_norm_backward; 0 if n is invalid. */
size_t adapm_norm_workspace_bytes(const adapm_norm_t* n);

/* dy: gradient of y; dh: gradient of h from elsewhere, the residual stream (data may be NULL).  Writes dresidual (the gradient of
 * h; data may be NULL), dx (dropout's factor times that) and dweight (cols values).  dx and dresidual may be dy or dh, but with
 * dropout not one another; workspace_dev: adapm_norm_workspace_bytes() bytes, 256-byte aligned. */
adapm_status_t adapm_norm_backward(const adapm_norm_t* n, adapm_rows_t dy, adapm_rows_t dh, adapm_rows_t h,
                                   const void* weight_dev, const float* rstd_dev, adapm_rows_t dx, adapm_rows_t dresidual,
                                   void* dweight_dev, const adapm_dropout_t* drop, void* workspace_dev, void* stream);

/* loss = f * sum_i w_i (lse_i - s_i,target(i)), s = x W^T: softmax cross entropy over a vocabulary whose logits are never
 * kept.  f = scale, divided by the number of rows that count with ADAPM_REDUCE_MEAN. */
typedef enum { ADAPM_REDUCE_SUM = 0, ADAPM_REDUCE_MEAN = 1 } adapm_reduction_t;
typedef struct {
  int64_t rows, vocab, cols;       /* x: rows x cols; W: vocab x cols; rows <= 2^22, vocab <= 2^21, cols <= 2^16;
                                      rows x vocab of 2^36 always fits, of more where one launch holds its tiles */
  int32_t dtype;                   /* x, W and their gradients: F32 or BF16 */
  int32_t reduction;               /* adapm_reduction_t */
  float scale;
  int32_t reserved;                /* 0 */
} adapm_head_t;

/* Scratch of adapm_head_loss (backward = 0) or adapm_head_backward (1); 0 if h is invalid.  weight: as in the call (W whose rows
 * are not whole, 16-byte aligned vectors is copied there).  It has room for a packed copy of x, since the device alone knows whether all
 * rows count and x can be read where it is. */
size_t adapm_head_workspace_bytes(const adapm_head_t* h, adapm_rows_t weight, int32_t backward);

/* targets[rows]: a row whose target lies outside [0, vocab) does not count: whatever it holds reaches nothing, its row_loss
 * and lse are 0.  row_weight[rows] (may be NULL: 1).  Writes loss (one float), row_loss[rows] (not weighted) and lse[rows], which
 * the backward pass needs.  If no row counts the loss is 0. */
adapm_status_t adapm_head_loss(const adapm_head_t* h, adapm_rows_t x, adapm_rows_t weight, const int64_t* targets_dev,
                               const float* row_weight_dev, float* loss_dev, float* row_loss_dev, float* lse_dev,
                               void* workspace_dev, size_t workspace_bytes, void* stream);

/* Gradients of upstream * loss (upstream_dev: one float, NULL: 1) by x and W, for the same arguments and the lse of
 * adapm_head_loss.  Either of dx and dweight may have data = NULL; rows that do not count get dx = 0, and dweight is 0 if
 * none does, whatever upstream is (inf and NaN too).  dx may be x; apart from that dx and dweight
 * overlap neither the inputs nor one another.  All vocab rows of dweight
 * are written: for the output head of a table that buffer is the block's gradient in adapm_step.  bf16: P = w (softmax - onehot) is
 * rounded to bf16 between the products, which makes the gradients' error 1.07 times that of their own rounding (root mean square), with
 * row weights 1.42 times.  Where up to 32 rows count, with row weights up to 1024, P is kept as two bf16 numbers: 1.00 times. */
adapm_status_t adapm_head_backward(const adapm_head_t* h, adapm_rows_t x, adapm_rows_t weight, const int64_t* targets_dev,
                                   const float* row_weight_dev, const float* lse_dev, const float* upstream_dev,
                                   adapm_rows_t dx, adapm_rows_t dweight, void* workspace_dev, size_t workspace_bytes,
                                   void* stream);

const char* adapm_last_error(void);

void adapm_destroy(adapm_ctx* ctx);

#ifdef __cplusplus
}
#endif
#endif /* ADAPM_H */
