/*
 * dartquant.h -- C ABI of the B200 (sm_100a) rotational-distribution-calibration
 * library.
 *
 * One calibration iteration is the loop body of Algorithm 1 of the DartQuant
 * paper: R <- Q factor of qr(Z) (QR-Orth, Sec. 4.3 / Algorithm 2), O <- X R,
 * L <- Whip(O) (Eq. 4), Z <- Z - eta dL/dZ.  Every step runs in CUDA kernels of
 * this library; there is no CPU fallback.
 *
 * Conventions
 *   - Pointers named d_* are DEVICE pointers, h_* are HOST pointers.
 *   - Matrices are row-major.  X is [batch][n_tokens][ldx] (one token per row),
 *     latents / rotations are [batch][d][d] fp32.
 *   - One process may use the library on several devices (a handle belongs to the device that was
 *     current at dq_calib_init; per-device kernel attributes are set on first use of each device).
 *   - Every call returns a dq_status; nothing throws, aborts or traps.  Device
 *     side problems (rank-deficient latent, non-finite loss, a wait that ran
 *     out) are recorded in a device status word read by dq_calib_status().  The
 *     first error wins and stays until dq_calib_set_latent or one of the
 *     dq_calib_set_* configuration calls clears it; while it is set, the kernels
 *     that update the latent (or the Cayley iterate) and the optimiser state
 *     change nothing, so the parameter stays at the last good iterate.
 *   - All work is enqueued on the stream given at init; calls are asynchronous
 *     with respect to the host unless stated otherwise.
 *   - Notation: R is always the rotation (the orthogonal factor of Z = R U),
 *     U the upper-triangular factor with positive diagonal.
 */
#ifndef DARTQUANT_H_
#define DARTQUANT_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct dq_calib dq_calib_t; /* opaque, owned by the library */

typedef enum {
  DQ_OK = 0,
  DQ_ERR_INVALID_ARG = 1, /* null pointer, non-positive size, bad enum          */
  DQ_ERR_UNSUPPORTED = 2, /* shape / dtype / path combination not implemented   */
  DQ_ERR_ALLOC = 3,       /* device allocation failed                           */
  DQ_ERR_CUDA = 4,        /* a CUDA runtime/driver call failed                  */
  DQ_ERR_SINGULAR = 5,    /* latent is (numerically) rank deficient: U^-T undefined */
  DQ_ERR_NONFINITE = 6,   /* loss became NaN/Inf                                */
  DQ_ERR_TIMEOUT = 7,     /* a bounded in-kernel wait gave up                   */
  DQ_ERR_NOT_CONVERGED = 8 /* DQ_QR_ITERATIVE: one step moved the latent too far     */
} dq_status;

enum { DQ_FP32 = 0, DQ_BF16 = 1 };             /* x_dtype                       */
enum { DQ_PATH_FP32 = 0, DQ_PATH_BF16_TC = 1 }; /* arithmetic of the X R / X^T G contractions */
enum { DQ_MEAN_TOKENS = 0, DQ_SUM_TOKENS = 1 }; /* reduction of Eq. 4 over token rows */
enum { DQ_SGD = 0, DQ_SGD_MOMENTUM = 1, DQ_ADAM = 2 }; /* optimiser (Algorithm 1, update step; Sec. 4.3: "SGD or Adam") */

typedef struct {
  int32_t d;         /* channels = size of the rotation; multiple of 64 (fp32 path) or 128 (tensor-core path); <= 8192 */
  int64_t n_tokens;  /* tokens per problem; any positive count (fp32 path) or a multiple of 256 (tensor-core path) */
  int32_t batch;     /* independent problems (e.g. attention heads); >= 1       */
  int32_t x_dtype;   /* DQ_FP32 | DQ_BF16                                       */
  int32_t path;      /* DQ_PATH_FP32: fp32 FMA contractions (needs DQ_FP32 X);
                        DQ_PATH_BF16_TC: bf16 tensor-core contractions with fp32 accumulation (needs DQ_BF16 X) */
  int32_t reduction; /* DQ_MEAN_TOKENS (default reading of Algorithm 1's loss step) | DQ_SUM_TOKENS */
  int32_t optimizer; /* DQ_SGD here; others via dq_calib_set_optimizer          */
  float lr;          /* eta                                                     */
  int64_t ldx;       /* row stride of X in elements (>= d; a multiple of 8 on the tensor-core path); problems are n_tokens*ldx apart */
} dq_calib_config;

/* Algorithm 1, hand-off before the loop: bind calibration activations and the initial
 * latent.  d_X is BORROWED (must outlive the handle; only dq_calib_run_epochs writes it).  d_Z0
 * ([batch][d][d] fp32) is COPIED.  cuda_stream is a cudaStream_t (NULL = legacy
 * default stream).  Allocates every workspace the step needs.
 * Errors: INVALID_ARG, UNSUPPORTED, ALLOC, CUDA.  *out is NULL on error. */
dq_status dq_calib_init(dq_calib_t** out, const dq_calib_config* cfg, const void* d_X,
                        const float* d_Z0, void* cuda_stream);

/* Algorithm 1's loop, exactly n_steps iterations.  d_loss_out (nullable) is a
 * device array [n_steps][batch] fp32; entry k is L(Z_k), the loss BEFORE the
 * k-th update.  No host synchronisation. */
dq_status dq_calib_step(dq_calib_t* h, int32_t n_steps, float* d_loss_out);

/* Sec. 4.3: the rotation of the CURRENT latent, i.e. the orthogonal factor of
 * Z = R U with diag(U) > 0 (recomputed if the latent changed since the last
 * factorisation).  d_R_out is caller-owned [batch][d][d] fp32. */
dq_status dq_calib_get_rotation(dq_calib_t* h, float* d_R_out);

/* Sec. 3 (Y = X R): apply a rotation to activations and materialise the result.
 * x_dtype selects both the storage type of X / Y and the arithmetic (DQ_FP32:
 * fp32 FMA; DQ_BF16: bf16 tensor cores, fp32 accumulation, bf16 output).
 * X is [n][ldx], Y is [n][ldy], R is [d][d] fp32, all device, no aliasing. */
dq_status dq_rotate_apply(const void* d_X, int32_t x_dtype, int64_t n, int32_t d, int64_t ldx,
                          const float* d_R, void* d_Y, int64_t ldy, void* cuda_stream);

/* (No counterpart in the paper: a packaging variant of dq_rotate_apply for bf16 activations.)
 * The same Y = X R, for callers that must not allocate device memory: a serving process that
 * handed all of HBM to its own arena at start-up (a later cudaMalloc would fail or fragment
 * it), or a latency-critical loop where the implicit device synchronisation of cudaFree is
 * not acceptable.  dq_rotate_apply allocates and frees a bf16 copy of R^T on every call; this
 * variant keeps that copy in a fixed device array inside the library (8 MiB, held by every GPU
 * that loads the library until the process exits) and calls no cudaMalloc / cudaFree or any
 * other allocating routine.
 *   - X, Y: bf16 [n][ldx] / [n][ldy]; R: fp32 [d][d]; all device, caller-owned, no aliasing.
 *   - d <= 2048 (the size of the fixed array), d % 128 == 0, n % 128 == 0, ldx % 8 == ldy % 8 == 0;
 *     anything else returns DQ_ERR_UNSUPPORTED and launches nothing.
 *   - The first call on each device also looks up the array's device address; make that call
 *     once, with that device current, before any stream capture.  It is also the call on which the
 *     CUDA runtime may load this library's kernels (and the array itself) onto the device, which
 *     takes device memory once: make it before the caller's arena takes the rest of HBM.
 *   - All calls share the one array.  Each call rewrites the part it uses before reading it, so
 *     calls on one stream are independent; calls that overlap on the GPU (different streams or
 *     threads without ordering between them) race on it and must be serialised by the caller. */
dq_status dq_rotate_apply_static(const void* d_X, int64_t n, int32_t d, int64_t ldx, const float* d_R,
                                 void* d_Y, int64_t ldy, void* cuda_stream);

/* What the paper measures a rotation by (Sec. 4.1, Eq. 1; appendix on outliers and quantisation
 * errors), for O = X R with X [n][ldx] (DQ_FP32 or DQ_BF16) and R fp32 [d][d], all device:
 *   d_out[0] = number of entries with |o| > tau                                  (Eq. 1 over all tokens)
 *   d_out[1] = mean squared error of per-token asymmetric uniform quantisation of O to `bits` bits:
 *              scale = (max - min) / (2^bits - 1), zero = round(-min / scale),
 *              q = clamp(round(o / scale) + zero, 0, 2^bits - 1), dequantised = scale (q - zero)
 * d_out is a device double[2], written on the stream.  O is computed with bf16 tensor cores for
 * DQ_BF16 (d % 128 == 0, n % 128 == 0) and fp32 FMA for DQ_FP32.  Allocates stream-ordered scratch.
 * Errors: INVALID_ARG (null, bits outside 1..16, tau < 0), UNSUPPORTED, ALLOC, CUDA. */
dq_status dq_eval_rotation(const void* d_X, int32_t x_dtype, int64_t n, int32_t d, int64_t ldx, const float* d_R,
                           float tau, int32_t bits, double* d_out, void* cuda_stream);

/* Algorithm 1, X <- token_sampling(X), and the mini-batches of the hyper-parameter appendix:
 * d_out[i] = d_X[pi(first + i)] for 0 <= i < count, where pi is a pseudo-random permutation of the
 * token rows [0, n_total) fixed by `seed` (uniform sampling without replacement: a Feistel network
 * with cycle walking over the Philox4x32-10 generator).  A sample of k tokens is first = 0,
 * count = k; mini-batches are consecutive windows; use another seed for another epoch.
 * X is [n_total][ldx], out is [count][ldo], both device, x_dtype DQ_FP32 or DQ_BF16, rows and row
 * strides multiples of 16 bytes (else DQ_ERR_UNSUPPORTED).  To calibrate on the batch, gather into
 * the buffer bound at dq_calib_init and call dq_calib_refresh_inputs. */
dq_status dq_gather_tokens(const void* d_X, int32_t x_dtype, int64_t n_total, int32_t d, int64_t ldx, uint64_t seed,
                           int64_t first, int64_t count, void* d_out, int64_t ldo, void* cuda_stream);

/* Mini-batch use (the paper feeds the loop with batches of sampled tokens): the
 * caller overwrote the borrowed activation buffer d_X in place (same shape) on
 * the handle's stream.  Every kernel reads the activations in place (no copy of them is
 * derived or kept), so today this call only orders the handle's internal stream after the
 * caller's writes; call it all the same after rewriting d_X. */
dq_status dq_calib_refresh_inputs(dq_calib_t* h);

/* Optimiser of the latent (Sec. 4.3: QR-Orth works with any standard optimiser; the paper reports
 * SGD and Adam).  Resets the optimiser state (moments, step count) and replaces the learning rate.
 *   DQ_SGD:          Z <- Z - lr g                                   (beta1, beta2, eps ignored)
 *   DQ_SGD_MOMENTUM: v <- beta1 v + g;  Z <- Z - lr v                 (beta1 = momentum)
 *   DQ_ADAM:         m <- beta1 m + (1 - beta1) g;  v <- beta2 v + (1 - beta2) g^2;
 *                    Z <- Z - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
 * Errors: INVALID_ARG (bad enum, betas outside [0, 1), eps < 0), ALLOC, CUDA. */
dq_status dq_calib_set_optimizer(dq_calib_t* h, int32_t optimizer, float lr, float beta1, float beta2, float eps);

/* How the QR-Orth forward (Sec. 4.3: Z = R U) is computed on the tensor-core path.  Both
 * give the same unique factors (diag(U) > 0).
 *   DQ_QR_ITERATIVE (default): incremental.  Blocked Householder QR (Algorithm 2 in compact-WY
 *     form) only when no factors of a nearby latent are known (first step, after
 *     dq_calib_set_latent or a change of method).  Afterwards, with the previous step's W_old = U_old^-1,
 *     Zh = Z W_old is close to orthogonal whatever Z is, its upper factor I + T is the fixed point
 *     of T <- striu(E - T^T T) + diag(E - T^T T) / 2 with E = Zh^T Zh - I, reached by sweeps of
 *     triangular tensor-core GEMMs (no dependent column steps) that start from the previous step's
 *     T^T T, and R = Zh (I + T)^-1, W = W_old (I + T)^-1 (the inverse of I + T from a few more triangular
 *     products; U itself is not formed).  The sweeps stop by themselves: each is skipped (by a
 *     device-side flag, so the launch sequence and a captured graph stay fixed) once the sweep before it
 *     moved no entry by more than 1e-5; the first two use a plain bf16 product, later ones and, after
 *     a step large enough to need them, the first-order correction products use split-bf16 operands.
 *     At most n_iters + 3 sweeps.  If the last of those still moved an entry, one optimiser step has
 *     moved the latent too far: the status word becomes DQ_ERR_NOT_CONVERGED and, as after every
 *     device-side error, the update kernels leave the latent and the optimiser state untouched from
 *     then on: the latent stays at the last good iterate.  Recover with
 *     dq_calib_set_qr_method(h, DQ_QR_HOUSEHOLDER, 0), more sweeps or a lower learning rate, and step
 *     again.  n_iters <= 0 selects the default (5 on this route: the paper's SGD steps need one
 *     sweep; an optimiser that moves every entry by its learning rate, such as Adam, may need more);
 *     at most 64.
 *   DQ_QR_HOUSEHOLDER: blocked Householder QR at every step; no assumption on the step size.
 * The call clears the status word.  For d == 128 (any path) the same two methods exist as kernels that
 * keep a whole latent in shared memory; there the sweeps stop as soon as no entry moves (one more is
 * taken) and n_iters only bounds them (4 n_iters).  On the fp32 path with d <= 1024 the incremental
 * factorisation runs on fp32 FMA products (up to n_iters + 3 sweeps, switched off the same way); larger fp32
 * latents are always factored with Householder. */
enum { DQ_QR_HOUSEHOLDER = 0, DQ_QR_ITERATIVE = 1 };
dq_status dq_calib_set_qr_method(dq_calib_t* h, int32_t method, int32_t n_iters);

/* Algorithm 1's loop around the step: token sampling and mini-batches (hyper-parameter appendix: a
 * fraction of the captured tokens per epoch, fixed batch size, several epochs).
 * d_pool: device, [n_pool][ld_pool] token rows of the handle's x_dtype, borrowed, never written.
 * Epoch e draws the seeded permutation pi of dq_gather_tokens with seed + e and uses its first
 * floor(sample_ratio * n_pool) rows (sampling without replacement), cut into optimiser steps of
 * accum micro-batches of the handle's n_tokens rows each; an incomplete last step is dropped.
 * Every micro-batch is gathered into the activation buffer given to dq_calib_init, WHICH THIS CALL
 * OVERWRITES (it must be writable device memory of n_tokens rows); dL/dR and the loss of a step are
 * the mean over all accum * n_tokens tokens of the step (gradient accumulation: the sum with
 * DQ_SUM_TOKENS), then one QR backward / optimiser update follows.  The paper does not say how tokens
 * are drawn or batched; this is the reading.  d_loss_out: nullable, device
 * [n_epochs * steps_per_epoch] with steps_per_epoch = floor(floor(sample_ratio * n_pool) /
 * (accum * n_tokens)); the product runs in double precision on the float sample_ratio.
 * h_steps_out: nullable HOST pointer, receives the number of optimiser steps enqueued.
 * Asynchronous like dq_calib_step; steps are not replayed from a graph (the gather changes).
 * Errors: INVALID_ARG (null, sizes, ratio outside (0, 1], no complete step), UNSUPPORTED (batch > 1),
 * CUDA. */
dq_status dq_calib_run_epochs(dq_calib_t* h, const void* d_pool, int64_t n_pool, int64_t ld_pool,
                              float sample_ratio, int32_t accum, int32_t n_epochs, uint64_t seed,
                              float* d_loss_out, int64_t* h_steps_out);

/* Arithmetic of the QR-Orth backward (Sec. 4.3: dL/dZ from dL/dR, Z = R U) on the tensor-core path for
 * d >= 256.  dL/dR carries the bf16 rounding of the rotation operand and of dL/dO (a few percent), so by
 * default (split = 0) its d x d products run on plain bf16 operands with fp32 accumulation (2^-9 relative);
 * split != 0 runs them on split-bf16 operands (three MMAs per product, about 2^-17).  No effect elsewhere. */
dq_status dq_calib_set_backward_precision(dq_calib_t* h, int32_t split);

/* The calibration objective.  DQ_OBJ_WHIP (default) is Eq. 4.  The other three are the objectives the
 * ablation of Sec. 5.3 compares it with; the paper names them without formulas, so they are read as
 * per-token statistics over the d channels of the rotated token o = x R (as Eq. 4 is per token),
 * averaged over tokens like the Whip loss (or summed, with DQ_SUM_TOKENS):
 *   DQ_OBJ_VARIANCE: (1/d) sum_j (o_j - mean(o))^2
 *   DQ_OBJ_KURTOSIS: m4 / m2^2 - 3 with m_p = (1/d) sum_j (o_j - mean(o))^p   (excess kurtosis)
 *   DQ_OBJ_QUANT:    (1/d) sum_j (o_j - Q(o)_j)^2, Q = per-token asymmetric uniform quantiser to `bits`
 *                    bits (the one of dq_eval_rotation); derivative with the grid held fixed and rounding
 *                    piecewise constant: (2/d) (o_j - Q(o)_j)
 * These need statistics of the whole token before any entry of dL/dO, so the rotated activations are
 * materialised chunk by chunk in fp32 instead of staying in tensor memory; everything after dL/dO
 * (contraction with X, QR backward or Cayley update, optimiser) is unchanged.  bits: 1..16, <= 0 selects
 * 4; ignored unless DQ_OBJ_QUANT.  A token whose rotated entries are all equal makes the kurtosis
 * undefined: the loss becomes non-finite and the status word DQ_ERR_NONFINITE.
 * Errors: INVALID_ARG (bad enum, bits > 16), ALLOC, CUDA. */
enum { DQ_OBJ_WHIP = 0, DQ_OBJ_VARIANCE = 1, DQ_OBJ_KURTOSIS = 2, DQ_OBJ_QUANT = 3 };
dq_status dq_calib_set_objective(dq_calib_t* h, int32_t objective, int32_t bits);

/* Which orthogonal optimiser updates the rotation.
 *   DQ_ORTH_QR (default): QR-Orth (Sec. 4.3): a free latent Z with R = the orthogonal factor of Z.
 *   DQ_ORTH_CAYLEY: Cayley SGD with momentum (Algorithm 3), the optimiser Sec. 5.3 and Table 4
 *     compare QR-Orth with.  The iterate is the rotation itself (X_1 = the orthogonal factor of the
 *     current latent, computed once); each dq_calib_step iteration computes the same loss and
 *     dL/dR as QR-Orth and then
 *       M <- beta M - dL/dR;  What = M R^T - R (R^T M R^T) / 2;  W = What - What^T;  M <- W R;
 *       a = min(lr, 2 q / (|W|_F + 1e-8));  Y^0 = R + a M;  Y^i = R + a/2 W (R + Y^(i-1)), i = 1..s;
 *       R <- Y^s
 *     with lr the handle's learning rate, six d x d tensor-core products per iteration.  The
 *     skew-symmetrisation is read as What - What^T and the norm as the Frobenius norm (Algorithm 3
 *     prints W on both sides of that step and does not name the norm).  q <= 0 selects 0.5, s <= 0 selects 2.
 *     The latent Z, the QR method and dq_calib_set_optimizer's choice are not used in this mode;
 *     dq_calib_get_rotation returns the iterate.  Selecting a method resets the momentum, and the
 *     next step starts again from the orthogonal factor of the latent.
 * Errors: INVALID_ARG (bad enum, beta outside [0, 1), q > 1, s > 16), UNSUPPORTED (fp32 path or
 * d == 128: only the tensor-core path with d >= 256 implements it), ALLOC, CUDA. */
enum { DQ_ORTH_QR = 0, DQ_ORTH_CAYLEY = 1 };
dq_status dq_calib_set_orth_method(dq_calib_t* h, int32_t method, float beta, float q, int32_t s);

/* Checkpoint / resume of the optimised parameter (Algorithm 1: Z <- Z0).  dq_calib_set_latent clears
 * the status word. */
dq_status dq_calib_get_latent(dq_calib_t* h, float* d_Z_out);
dq_status dq_calib_set_latent(dq_calib_t* h, const float* d_Z);

/* Synchronises the stream and returns the device status word
 * (DQ_OK / DQ_ERR_SINGULAR / DQ_ERR_NONFINITE / DQ_ERR_TIMEOUT / DQ_ERR_NOT_CONVERGED) or DQ_ERR_CUDA. */
dq_status dq_calib_status(dq_calib_t* h);

/* Failure detection self-test (no counterpart in the paper).  Every wait inside the tensor-core kernels (on
 * a TMA copy, an MMA, the other CTA of a pair) is bounded: when it runs out the kernel records
 * DQ_ERR_TIMEOUT in the status word and returns normally, and from then on the update kernels leave the
 * latent untouched.  This call runs that same wait, with a limit of limit_ns nanoseconds (1 .. 1e8), in a
 * one-thread kernel on a barrier that nothing ever arrives at, with no copy or MMA in flight.  Afterwards
 * dq_calib_status returns DQ_ERR_TIMEOUT and steps leave the latent unchanged until dq_calib_set_latent (or a
 * dq_calib_set_* call) clears the status.  d_waited_ns (nullable, device) receives the time waited.
 * Tensor-core path only (DQ_ERR_UNSUPPORTED otherwise). */
dq_status dq_calib_selftest_bounded_wait(dq_calib_t* h, uint64_t limit_ns, uint64_t* d_waited_ns);

/* Phase times of the most recent dq_calib_step call, averaged per step, in ms
 * (synchronises).  Order: DQ_PHASE_*.  Writes min(n, DQ_PHASE_COUNT) entries
 * of the HOST array ms_by_phase. */
enum {
  DQ_PHASE_QR_FORWARD = 0, /* factorisation, forming R, gauge, operand copies   */
  DQ_PHASE_ROTATE_WHIP = 1, /* O = X R with the fused Eq. 4 epilogue + loss reduce */
  DQ_PHASE_GRAD_ROTATION = 2, /* Gq = X^T G                                      */
  DQ_PHASE_QR_BACKWARD = 3,
  DQ_PHASE_UPDATE = 4,
  DQ_PHASE_COUNT = 5
};
dq_status dq_calib_get_timings(dq_calib_t* h, float* h_ms_by_phase, int32_t n);
/* Enable (1) / disable (0) per-phase CUDA-event timing inside dq_calib_step. */
dq_status dq_calib_set_timing(dq_calib_t* h, int32_t enabled);

/* Read-only views of the handle's device workspaces after a step, for tests and
 * diagnostics.  *d_ptr is valid until the handle is destroyed. */
enum {
  DQ_BUF_R = 0,        /* fp32 [batch][d][d]  rotation used by the last step       */
  DQ_BUF_U = 1,        /* fp32 [batch][d][d]  upper factor, positive diagonal (after incremental steps on the tensor-core
                          path only U^-1 is carried: for d >= 256 it is inverted on demand, to about 1e-5; for d == 128 the
                          view is DQ_ERR_UNSUPPORTED until the next Householder factorisation) */
  DQ_BUF_GQ = 2,       /* fp32 [batch][d][d]  dL/dR                                */
  DQ_BUF_GZ = 3,       /* fp32 [batch][d][d]  dL/dZ                                */
  DQ_BUF_G = 4,        /* dL/dO without the 1/N factor: fp32 [batch][N][d] (fp32 path)
                          or bf16 channel-major [batch][d][N] (tensor-core path)   */
  DQ_BUF_PARTIALS = 5, /* fp32 loss partial sums of the last step, a fixed number per problem: one set per
                          output tile (d = 128 on the tensor-core path: per range of token tiles that one
                          CTA covers; entries no CTA writes stay zero)             */
  DQ_BUF_Z = 6,        /* fp32 [batch][d][d]  current latent                       */
  DQ_BUF_OPT_M = 7,    /* fp32 [batch][d][d]  first moment / velocity (NULL for DQ_SGD)  */
  DQ_BUF_OPT_V = 8,    /* fp32 [batch][d][d]  second moment (DQ_ADAM only)         */
  DQ_BUF_CAYLEY_M = 9, /* fp32 [batch][d][d]  momentum of DQ_ORTH_CAYLEY            */
  DQ_BUF_CAYLEY_ALPHA = 10 /* fp32 [batch]    step size of the last Cayley iteration */
};
dq_status dq_calib_debug_buffer(dq_calib_t* h, int32_t which, void** d_ptr, int64_t* n_elems);

/* For d == 128 on the tensor-core path both contractions and the Eq. 4 epilogue run in one kernel and
 * dL/dO never leaves the chip, so DQ_BUF_G is not written.  keep != 0 makes that kernel store dL/dO to
 * DQ_BUF_G as well (for inspection and tests; the results of a step do not change).  No effect on
 * other shapes, where DQ_BUF_G is always written. */
dq_status dq_calib_set_keep_gradient(dq_calib_t* h, int32_t keep);

/* Number of kernels this library launched through the handle so far. */
int64_t dq_calib_launch_count(dq_calib_t* h);

/* bf16 tensor-core flops the handle's tcgen05 kernels were asked to issue so far (2 m n k per MMA
 * product, three products per split-bf16 term, k clipped to the non-zero blocks of triangular
 * operands exactly as the kernels clip it; counted on the host at launch).  For measurement:
 * the difference across a timed region divided by its duration is the issued MMA rate. */
double dq_calib_mma_flops(dq_calib_t* h);

/* For measurement: times (CUDA events on the handle's work stream; synchronises) `reps` launches of one
 * dense d x d x d product of the kind QR-Orth is made of, on the handle's own operand copies, result to
 * scratch: nterms = 3 on split-bf16 operands (three bf16 MMAs per product term, 6 d^3 MMA flops for the
 * 2 d^3 of the product), nterms = 1 on plain bf16 operands.  *h_ms receives the mean per launch.  Tensor-core
 * path with d >= 256 only; call it after at least one step.  Changes no state of the calibration. */
dq_status dq_calib_time_product(dq_calib_t* h, int32_t nterms, int32_t reps, float* h_ms);

/* ---------------------------------------------------------------------------------------------------------------
 * Microscaled operators (no counterpart in the paper, which quantises to integers: the forward pass of a model whose
 * activations a calibrated rotation has made quantisable, in the formats the B200's tensor cores multiply).
 *
 * Formats: OCP microscaling, blocks of 32 values along a row.  A block has one power-of-two scale, the E8M0 byte
 * max(floor(log2 max|x|) - EMAX + 127, 0), and 32 elements round-to-nearest-even(x / scale), saturated:
 *   DQ_MXFP4: E2M1 (EMAX 2, values 0, .5, 1, 1.5, 2, 3, 4, 6), two to a byte, the even one in the low half
 *   DQ_MXFP8: E4M3 (EMAX 8, largest 448), one to a byte
 * A block with a NaN or an infinity gets the NaN scale 0xFF and reads back as NaN, all 32 of it; so does every output
 * of a product that it enters.  A block of zeros has scale byte 0.  A last block that is not full is quantised as if
 * the missing values were zeros.
 * Codes: [rows][dq_mx_row_bytes]; rows are padded with zero codes to a multiple of 128 values.  32-byte aligned.
 * Scales: dq_mx_scale_bytes bytes, tiles of 128 rows x 4 blocks in the order the tensor cores read them: the scale of
 *   (row, block) is byte ((row / 128) * ceil(k / 128) + block / 4) * 512 + row % 32 * 16 + row / 32 % 4 * 4 + block % 4.
 *   Bytes of rows past the last one are not defined and not used.  16-byte aligned.
 * Matrices of values (X, Y, sums, values) are row-major with a row stride of at least their width, of DQ_FP32, DQ_BF16
 *   or DQ_FP16; 16-byte aligned rows are read and written fastest, no alignment beyond the type's is needed.
 * Calls are asynchronous on the given stream, allocate nothing, keep nothing and can be captured in a graph (make one call of
 *   each kind before, on each device: the first looks up what the device can run at once).  They use programmatic dependent
 *   launch: a kernel may be scheduled before the one in front of it has ended, but reads and writes nothing until then, with
 *   one exception: dq_mx_linear's product may read weights while the same call's quantisation still runs.  Any number of host
 *   threads may call at the same time, each with streams, outputs and workspaces of its own.
 *   A call with no rows does nothing.  Limits: k <= 2^24, rows <= 2^31 - 256.
 * Errors: INVALID_ARG (null, sizes, enums, a pointer that its type's alignment rules out), UNSUPPORTED (alignment of codes
 *   and scales, limits, a device that is not sm_100), CUDA. */
enum { DQ_FP16 = 2 };                   /* third value of the microscaled operators' *_dtype arguments */
enum { DQ_MXFP4 = 0, DQ_MXFP8 = 1 };

/* Bytes of a row of codes, of the scales of a matrix, and of dq_mx_linear's workspace; -1 for arguments out of range. */
int64_t dq_mx_row_bytes(int32_t fmt, int64_t k);
int64_t dq_mx_scale_bytes(int64_t rows, int64_t k);
int64_t dq_mx_linear_workspace(int32_t a_fmt, int64_t m, int64_t k);

/* Codes and scales of X [rows][ldx].  d_values (nullable, [rows][ldv] of X's type) receives the values that the codes
 * stand for; it may be X itself (with ldv == ldx), for evaluating a quantised model on unquantised products. */
dq_status dq_mx_quantize(const void* d_X, int32_t x_dtype, int64_t rows, int64_t k, int64_t ldx, int32_t fmt, void* d_codes,
                         void* d_scales, void* d_values, int64_t ldv, void* cuda_stream);

/* The values that codes and scales stand for, Y [rows][ldy] (rounded once where y_dtype cannot hold them). */
dq_status dq_mx_dequantize(int32_t fmt, const void* d_codes, const void* d_scales, int64_t rows, int64_t k, void* d_Y,
                           int32_t y_dtype, int64_t ldy, void* cuda_stream);

/* Root-mean-square norm with the residual's addition and a quantised output:
 *   h = x + residual (fp32),  y = h / sqrt(mean_j h_j^2 + eps) gamma,  codes and scales of y
 * X, residual, sum and values have type `dtype`.  d_residual (nullable: h = x).  d_gamma (nullable: ones, as where gamma
 * was folded into the weights before a rotation): [k] of gamma_dtype, DQ_FP32 or `dtype`.  d_sum (nullable) receives
 * h rounded once, what the next layer adds to; it may be X or residual itself (equal row strides).  y is computed from
 * the unrounded h.  The squares are summed in fp32: a row whose sum of squares passes its range (3.4e38) has
 * y = 0.  d_values (nullable) as in dq_mx_quantize.  k <= 32768. */
dq_status dq_rmsnorm_quantize(const void* d_X, const void* d_residual, int32_t dtype, int64_t rows, int64_t k, int64_t ldx,
                              int64_t ldr, const void* d_gamma, int32_t gamma_dtype, float eps, int32_t fmt, void* d_codes,
                              void* d_scales, void* d_sum, int64_t lds, void* d_values, int64_t ldv, void* cuda_stream);

/* Y[i][j] = sum_k A[i][k] W[j][k] for m rows of quantised activations (DQ_MXFP4 or DQ_MXFP8) and n rows of DQ_MXFP4
 * weights, on the block-scaled tensor-core products with fp32 accumulation, rounded once to y_dtype.  Results do not depend
 * on the run.  Y must not overlap the operands. */
dq_status dq_mx_matmul(int32_t a_fmt, const void* d_a_codes, const void* d_a_scales, int64_t m, const void* d_w_codes,
                       const void* d_w_scales, int64_t n, int64_t k, void* d_Y, int32_t y_dtype, int64_t ldy,
                       void* cuda_stream);

/* The same from activations X [m][ldx] that the call quantises to a_fmt first (exactly as dq_mx_quantize).
 * d_workspace: dq_mx_linear_workspace bytes, 32-byte aligned; calls that overlap on the GPU need one each. */
dq_status dq_mx_linear(const void* d_X, int32_t x_dtype, int64_t m, int64_t k, int64_t ldx, int32_t a_fmt,
                       const void* d_w_codes, const void* d_w_scales, int64_t n, void* d_Y, int32_t y_dtype, int64_t ldy,
                       void* d_workspace, void* cuda_stream);

/* Synchronises the stream; returns and clears the current device's status word of the microscaled operators:
 * DQ_OK, or DQ_ERR_TIMEOUT once a bounded wait inside a product gave up (its output is then not valid). */
dq_status dq_mx_status(void* cuda_stream);

/* Failure detection self-test: dq_mx_matmul's product with its waits limited to limit_ns (1 .. 1e8) each, in which the warp
 * that issues the MMAs waits at its pipeline step `step` (>= 0, of every CTA or CTA pair that has that many) for a barrier that
 * nothing arrives at.  It gives up, what it has in flight ends, and the kernel returns; dq_mx_status then says DQ_ERR_TIMEOUT,
 * and Y is not valid. */
dq_status dq_mx_selftest_bounded_wait(int32_t a_fmt, const void* d_a_codes, const void* d_a_scales, int64_t m, const void* d_w_codes,
                                      const void* d_w_scales, int64_t n, int64_t k, void* d_Y, int32_t y_dtype, int64_t ldy,
                                      int64_t step, uint64_t limit_ns, void* cuda_stream);

/* ---------------------------------------------------------------------------------------------------------------
 * Attention over a key/value cache in 4 bits (the paper evaluates its rotations with keys and values quantised so, per token
 * and head, asymmetrically, behind the online Hadamard rotation of queries and keys).
 *
 * Cache: pages of page_size tokens (a power of two, 16 .. 4096), [n_pages][heads][dq_kv_page_bytes], of head_dim 64, 128 or
 * 256, in groups of 16 tokens: key codes [16][head_dim / 2], key parameters [16] (scale, offset: two bf16), the same of the
 * values.  Two codes a byte, the even dimension in the low half.  value = offset + scale * code with
 *   offset = the largest bf16 number <= min x,  scale = the smallest bf16 number >= (max x - offset) / 15 (formed in fp32),
 *   code = round-to-nearest-even((x - offset) / scale); 0 where scale is 0.
 * A head of a token with a NaN, an infinity or a range past fp32's gets NaN parameters and reads back as NaN.  d_pages: 128-byte
 * aligned.
 * d_table [n_seqs][table_width]: the pages of a sequence, in order; an index outside [0, n_pages) is no page: what would be
 * written there is dropped, and keys there take no part.  Pages may be shared between sequences as long as no call writes
 * to one that the table names twice.  d_lengths [n_seqs]: tokens (slots) of a sequence, those of the call included; taken as 0 where negative and as
 * table_width * page_size (at most 2^30) where above.  Both are read on the device when the call runs.
 * Tokens of a call: sequence b has rows d_starts[b] .. d_starts[b + 1] - 1 of the call's tensors (d_starts [n_seqs + 1], not
 * decreasing), or tokens / n_seqs each where d_starts is NULL.  They are its last: token i of n has slot length - n + i, and
 * sees the slots up to its own.  Rows that belong to no sequence are left as they are.
 * Tensors of heads (dq_heads_t): [token][head][head_dim] with contiguous values and any strides, counted in values, so that
 * views of a fused projection can be given; heads that start on 16-byte boundaries are read and written fastest.
 * Calls behave as the microscaled operators' do: asynchronous, nothing allocated or kept, capturable, dependent launch; a wait
 * that gives up (of dq_kv_attention and dq_kv_attention_weights, 1 s) is reported by dq_mx_status.
 * Errors: INVALID_ARG (null, sizes, enums, heads that do not fit, a pointer that its type's alignment rules out), UNSUPPORTED
 * (head_dim, page_size, alignment of pages and workspace, limits, a type, a device that is not sm_100), CUDA. */
typedef struct {
  void* d_data;
  int64_t token_stride, head_stride; /* in values */
  int32_t heads;
} dq_heads_t;

typedef struct {
  void* d_pages;
  int64_t n_pages;
  const int32_t* d_table;
  const int32_t* d_lengths;
  int32_t n_seqs, table_width, heads, head_dim, page_size;
} dq_kv_cache_t;

/* Bytes of a page of one head, of dq_kv_attention's and dq_kv_evict's workspaces; -1 for arguments out of range. */
int64_t dq_kv_page_bytes(int32_t page_size, int32_t head_dim);
int64_t dq_kv_attention_workspace(int32_t head_dim);
int64_t dq_kv_evict_workspace(int32_t n_seqs, int32_t heads, int32_t keep);

/* Queries and keys of each head, in one pass:
 *   DQ_QK_NORM:     h = x / sqrt(mean x^2 + eps) * gamma (gamma: [head_dim] of gamma_dtype, DQ_FP32 or `dtype`; NULL: ones)
 *   rotation:       pairs (a, b) of the first rot_dim values, (i, i + rot_dim / 2), or (2 i, 2 i + 1) with DQ_QK_NEIGHBOURS, to
 *                   (a cos t - b sin t, b cos t + a sin t) with t = position * inv_freq[i], formed in 64 bits
 *   DQ_QK_HADAMARD: y = h H / sqrt(head_dim) with Sylvester's H (head_dim 64, 128, 256), which keeps q . k
 * computed in fp32, rounded once.  d_positions [tokens], d_inv_freq [rot_dim / 2]; rot_dim 0: no rotation.  K and K_out may be
 * NULL.  An output may be its input.  head_dim and rot_dim: multiples of 16, head_dim at most 256. */
enum { DQ_QK_NORM = 1, DQ_QK_NEIGHBOURS = 2, DQ_QK_HADAMARD = 4 };
dq_status dq_qk_norm_rope(const dq_heads_t* Q, const dq_heads_t* K, int32_t dtype, int64_t tokens, int32_t head_dim,
                          const int32_t* d_positions, const float* d_inv_freq, int32_t rot_dim, const void* d_q_gamma,
                          const void* d_k_gamma, int32_t gamma_dtype, float eps, int32_t flags, const dq_heads_t* Q_out,
                          const dq_heads_t* K_out, void* cuda_stream);

/* Quantises the call's keys and values into their slots.  k_values, v_values (nullable; may be K and V): what the codes stand
 * for, rounded once to `dtype`.  d_slot_positions (nullable, [n_seqs][heads][ld_slots], ld_slots >= table_width * page_size):
 * the slots' positions, from d_positions [tokens], or the slots' own numbers where that is NULL. */
dq_status dq_kv_append(const dq_heads_t* K, const dq_heads_t* V, int32_t dtype, int64_t tokens, const dq_kv_cache_t* cache,
                       const int32_t* d_starts, const dq_heads_t* k_values, const dq_heads_t* v_values, const int32_t* d_positions,
                       int32_t* d_slot_positions, int64_t ld_slots, void* cuda_stream);

/* The keys and values of the sequences' last tokens, as the cache holds them, rounded once to `dtype` (zeros where there is no page
 * or no slot). */
dq_status dq_kv_dequantize(const dq_kv_cache_t* cache, const int32_t* d_starts, int64_t tokens, const dq_heads_t* K,
                           const dq_heads_t* V, int32_t dtype, void* cuda_stream);

/* out = softmax(scale * q k^T) v over the slots that each query sees; query head j reads kv head j / (Q's heads / cache's heads).
 * dtype: DQ_BF16 or DQ_FP16.  A query that sees nothing gets zeros.  d_lse (nullable, [tokens][Q's heads]): the natural logarithm of the
 * sums of exp(scale * q . k), -infinity for a query that sees nothing.  d_workspace: dq_kv_attention_workspace bytes, 16-byte
 * aligned, set to zero once before its first use (every call leaves it ready for the next); calls that overlap on the GPU need one each.
 * out overlaps neither Q nor the cache.  Results do not depend on the run.  Products take 16-bit operands and fp32 sums: queries times a power of
 * two (digits below 2^-24 of a row's largest value are lost) and, with few query rows a sequence (below 64 to 256), the codes themselves and exp times a
 * value's scale (2^-11 of it, and 2^-31 of the largest scale).  With more rows keys and values are rounded: a key's element is off by up to
 * 2^-14 of the largest scale among the same 128 slots, seen by the query or not (by nothing where its own scale is within 2^-7 of that), a
 * value's by 2^-11 of its terms (offset and scale * code) and 2^-14 of the largest scale or 2^-28 of the largest value up to there.  With few
 * rows values times exponentials are added before the division, so the values' size times 2^8 times their number has to stay within fp32's
 * range.  Queries of 2^118 and more count as infinite. */
dq_status dq_kv_attention(const dq_heads_t* Q, int32_t dtype, int64_t tokens, const dq_kv_cache_t* cache, const int32_t* d_starts,
                          float scale, const dq_heads_t* out, float* d_lse, void* d_workspace, void* cuda_stream);

/* The probability that each slot received, added up: for the slots of sequence b and kv head h,
 *   weights_out[b][h][slot] = (slot < length - n ? weights[b][h][slot] : 0) + sum over the n queries and the query heads of h that see
 *   the slot of exp(scale * q . k - lse)
 * with dq_kv_attention's d_lse.  [n_seqs][heads][ld_slots], ld_slots >= table_width * page_size; d_weights NULL: zeros; d_weights_out may
 * be d_weights.  Slots from the length on are left as they are.  Results do not depend on the run. */
dq_status dq_kv_attention_weights(const dq_heads_t* Q, int32_t dtype, int64_t tokens, const float* d_lse, const dq_kv_cache_t* cache,
                                  const int32_t* d_starts, float scale, const float* d_weights, float* d_weights_out,
                                  int64_t ld_slots, void* cuda_stream);

/* Leaves the sequences min(length, keep) slots: in each head those whose position is above the head's largest less `recent`, then
 * those with the largest weights (a NaN last); of equals the lower slots.  Kept slots from `keep` on move, in order, into the
 * slots below that are given up, with their codes, weights and positions, so a head's slots are in no order of positions
 * afterwards, and the heads of a sequence keep different tokens.  Pages play no part in the choice; a kept slot that moves to where there is no page
 * takes its weight and position along and loses its codes, and one without a page, whose place would be a slot with one, is given up: there
 * the slot's token stays, with its weight and position.  d_lengths_out [n_seqs] receives the new lengths.  The outputs may be the
 * inputs (d_lengths_out the cache's lengths); entries from the new length on are left as they are.  0 <= recent <= keep, keep > 0.
 * d_workspace: dq_kv_evict_workspace bytes; calls that overlap on the GPU need one each. */
dq_status dq_kv_evict(const dq_kv_cache_t* cache, const float* d_weights, const int32_t* d_positions, int64_t ld_slots, int32_t keep,
                      int32_t recent, float* d_weights_out, int32_t* d_positions_out, int32_t* d_lengths_out, void* d_workspace,
                      void* cuda_stream);

const char* dq_status_string(dq_status s);
void dq_calib_destroy(dq_calib_t* h);

/* Compile-time facts of the loaded library: returns a static string such as
 * "dartquant-b200 sm_100a". */
const char* dq_version(void);

#ifdef __cplusplus
}
#endif
#endif /* DARTQUANT_H_ */
