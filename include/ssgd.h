/*
 * ssgd.h - C ABI of the MI355X library that simulates straggler-aware
 * distributed SGD with P virtual workers on one GPU.
 *
 * The calls follow the problem statement of "Slow and Stale Gradients Can Win
 * the Race" (arXiv 2003.10579): a parameter server with P workers (Sec. 2.1),
 * mini-batch size m, learning rate eta, K workers or mini-batches waited for
 * per update (Sec. 2.2), i.i.d. random compute delays per worker and
 * mini-batch (Sec. 3.1), the expected runtime per iteration (Sec. 2.3, Sec. 3)
 * and AdaSync (Sec. 6).
 *
 * Conventions
 *  - Pointers are tagged DEVICE (address in the memory of the current HIP
 *    device) or HOST.  The library never takes ownership of a caller buffer.
 *  - Every call returns an ssgd_status; nothing throws or aborts across the
 *    ABI.  On an error `ssgd_last_error` gives a static or context-owned text.
 *  - A context is bound to the HIP device that was current in ssgd_create and
 *    to the stream given there.  It is not thread-safe; distinct contexts are
 *    independent.
 *  - Determinism: identical arguments give identical delays, selections,
 *    staleness counts and clock values, bit for bit.
 */
#ifndef SSGD_H
#define SSGD_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ssgd_ctx ssgd_ctx; /* opaque, library-owned */

typedef enum {
    SSGD_OK = 0,
    SSGD_EINVAL = 1,  /* bad argument; nothing was changed */
    SSGD_ENOMEM = 2,  /* a device or host allocation failed */
    SSGD_EDEVICE = 3, /* a HIP call or a kernel reported an error */
    SSGD_ESTATE = 4   /* call not valid in the context's current state */
} ssgd_status;

/* Loss f(w, xi) behind the objective F(w) = (1/N) sum_n f(w, xi_n) (Eq. (1)).
 * Parameter vector layout (fp32):
 *   SSGD_LSQ      f = (x.w - y)^2 / 2                 w[d]
 *   SSGD_SOFTMAX  f = -log softmax(W x + b)_y         W[classes][d], b[classes]
 *   SSGD_MLP2     two-layer ReLU network + softmax    W1[hidden][d], b1[hidden],
 *                                                     W2[classes][hidden], b2[classes] */
typedef enum { SSGD_LSQ = 0, SSGD_SOFTMAX = 1, SSGD_MLP2 = 2 } ssgd_model_kind;

/* The four variants of Sec. 2.2. */
typedef enum {
    SSGD_K_SYNC = 0,       /* Eq. (2): first K of P workers, the rest are cancelled */
    SSGD_K_BATCH_SYNC = 1, /* first K mini-batches; a finished worker starts another at w_j */
    SSGD_K_ASYNC = 2,      /* Eq. (3): first K of P workers, nobody is cancelled, stale w */
    SSGD_K_BATCH_ASYNC = 3 /* first K mini-batches, nobody is cancelled: a worker that pushes re-reads the
                              current parameters and starts its next mini-batch at once.  Fixed K or
                              AdaSync mode 1.  Linear models: d % 4 == 0, at most 15 classes,
                              K <= 64 (any m), N d 4 < 2^32; MLP2: its usual limits, K <= 256;
                              else SSGD_EINVAL */
} ssgd_variant;

/* Delay X of one mini-batch on one worker (Sec. 3.1).
 *   SSGD_EXP          X = E / rate,          E ~ Exp(1)   (rate = mu, E[X] = 1/mu)
 *   SSGD_SHIFTED_EXP  X = shift + E / rate                (Lemma 4)
 *   SSGD_PARETO       X = scale * exp(E / alpha)          (Pareto(alpha, scale), Fig. 5)
 *   SSGD_TABLE        X = table[(((version * P) + worker) * R + ordinal) mod table_len],
 *                     R = 1 for K-sync / K-async, Kmax + 1 for the batch variants.
 *                     `table` is a HOST pointer, copied in ssgd_create. */
typedef enum { SSGD_EXP = 0, SSGD_SHIFTED_EXP = 1, SSGD_PARETO = 2, SSGD_TABLE = 3 } ssgd_delay_kind;

typedef struct {
    int32_t kind; /* ssgd_delay_kind */
    double shift, rate, alpha, scale;
    const float *table; /* HOST, SSGD_TABLE only */
    int64_t table_len;
} ssgd_delay_dist;

typedef struct {
    int32_t kind; /* ssgd_model_kind */
    int32_t d, classes, hidden;
    int32_t bf16;    /* SSGD_MLP2: 1 = bf16 operands, fp32 accumulation, in the two
                        contractions over d; must be 0 for the linear models */
    const float *X;  /* DEVICE, N x d row-major fp32; must outlive the context and stay unchanged:
                      * SSGD_MLP2 keeps its values rounded to bf16, taken when the context is made */
    const void *y;   /* DEVICE, float[N] (LSQ) or int32[N] labels in [0, classes) */
    int64_t N;       /* 1 <= N < 2^32 */
} ssgd_model;

/* AdaSync (Sec. 6): how K changes between updates.
 *   mode 0  K fixed
 *   mode 1  windows of `window` updates; if the mean training loss of a window is
 *           above (1 - rel_tol) times that of the window before, K doubles (<= Kmax)
 *   mode 2  Algorithm 1: whenever the clock crosses a multiple of interval_t and
 *           K < Kmax, K = K0 sqrt(F(w_0) / F(w_start)), rounded, never decreasing
 *   mode 3  the K-sync rule of App. D: K^2/(P-K) = K0^2/(P-K0) F(w_0)/F(w_start)
 * F is estimated by the mean mini-batch loss of the contributors. */
typedef struct {
    int32_t mode, K0, Kmax, window;
    double rel_tol, interval_t;
} ssgd_adasync;

/* Create `replicas` independent simulations (same data, same w_0, delays and
 * mini-batches keyed by the replica index) of `variant` with P workers that
 * waits for K, mini-batch size m, learning rate lr.  All P workers start at
 * time 0 with w_0 (zeros; uniform(-1/sqrt(fan_in), 1/sqrt(fan_in)) weights for
 * the MLP).  `hip_stream` is a hipStream_t (NULL = default stream); all work
 * is enqueued there.  `adasync` may be NULL (mode 0).
 * Limits: 1 <= K <= P <= 256 for K-sync / K-async, 1 <= K <= 256 for the batch
 * variants, m >= 1, d >= 1, classes <= 16 for SOFTMAX; MLP2 needs bf16 = 1, m <= 64,
 * d % 128 == 0, hidden % 128 == 0, and with several replicas a fixed K or AdaSync mode 1;
 * SSGD_K_BATCH_ASYNC has the limits given with the enumeration.  Invalid arguments give
 * SSGD_EINVAL and leave *out untouched.
 * Device memory of a linear model: for K-async and K-batch-async P gradients per replica, and up to
 * 32 times as much (about one gigabyte at most on 256 CUs) where several clusters of workgroups share a replica's
 * updates and keep gradients in flight each for itself; where that does not fit they do not share. */
ssgd_status ssgd_create(const ssgd_model *model, int32_t P, int32_t K, int32_t m, int32_t variant,
                        const ssgd_delay_dist *dist, double lr, uint64_t seed, int32_t replicas,
                        const ssgd_adasync *adasync, void *hip_stream, ssgd_ctx **out);

/* Perform J further parameter-server updates in every replica: delays,
 * K-of-P selection, mini-batch gradients at the (possibly stale) parameters each
 * contributor read, w_{j+1} = w_j - (lr/K) sum_l g_l.  Appends to the trace.
 * Returns after the work has completed on the stream.  The library may use further
 * streams of its own (default priority; they start after the work queued on
 * `hip_stream` and that stream waits for them) and, for one replica of SSGD_MLP2,
 * two short-lived host threads that launch kernels during the call. */
ssgd_status ssgd_run(ssgd_ctx *ctx, int64_t J);

/* Make room in the trace for `updates` further updates now, so that later ssgd_run
 * calls up to that total do not reallocate it. */
ssgd_status ssgd_reserve_trace(ssgd_ctx *ctx, int64_t updates);

/* One update; additionally writes the averaged gradient (1/K) sum_l g_l that the
 * update applied, for replica 0, to agg_grad_out (DEVICE, |w| floats, nullable). */
ssgd_status ssgd_step(ssgd_ctx *ctx, float *agg_grad_out);

/* Number of parameters |w| of the context's model. */
int64_t ssgd_param_count(const ssgd_ctx *ctx);
/* Updates done so far, current K, and the row width Kmax of the trace arrays. */
int64_t ssgd_updates_done(const ssgd_ctx *ctx);
int32_t ssgd_current_K(const ssgd_ctx *ctx, int32_t replica);
int32_t ssgd_trace_width(const ssgd_ctx *ctx);

/* Copy updates [from, from+n) of one replica's trace to HOST arrays (each
 * nullable): t[n] clock after the update (fp64), loss[n] mean mini-batch loss of
 * the contributors, K[n], and n x Kmax matrices (unused entries -1) of the
 * contributing workers in arrival order, their staleness j - tau, and the
 * ordinal of the contributed mini-batch. */
ssgd_status ssgd_get_trace(ssgd_ctx *ctx, int32_t replica, int64_t from, int64_t n, double *t,
                           float *loss, int32_t *K, int32_t *sel_workers, int32_t *staleness,
                           int32_t *ordinal);

/* Copy the current parameters of one replica to w_out (HOST, |w| floats). */
ssgd_status ssgd_get_params(ssgd_ctx *ctx, int32_t replica, float *w_out);
/* Overwrite the current parameters of one replica from w_in (HOST, |w| floats).
 * Gradients of mini-batches already in flight keep the parameters they read. */
ssgd_status ssgd_set_params(ssgd_ctx *ctx, int32_t replica, const float *w_in);
/* Force K for the following updates (1 <= K <= Kmax); AdaSync keeps running. */
ssgd_status ssgd_force_K(ssgd_ctx *ctx, int32_t K);

/* The objective F(w) = (1/N) sum_n f(w, xi_n) of Eq. (1) over the whole data set at the replica's
 * current parameters (what the paper's error-versus-time curves plot), one streaming pass over
 * X.  loss_out: HOST.  Linear models need d % 4 == 0 (else SSGD_EINVAL) and evaluate in fp32
 * with fp64 sums.  The two-layer network evaluates with the forward pass of its trainer (inputs,
 * W1 and W2 at their bf16 values, fp32 accumulation), through temporary device buffers that the
 * call allocates and frees (SSGD_ENOMEM if they do not fit); mini-batches in flight are untouched. */
ssgd_status ssgd_full_loss(ssgd_ctx *ctx, int32_t replica, double *loss_out);

/* The gradient of that objective, grad F(w) = (1/N) sum_n grad f(w, xi_n), at the replica's current
 * parameters: the quantity in which the staleness bound (fifth assumption of Sec. 4.1) is stated
 * (E||grad F(w_j) - grad F(w_tau)||^2 <= gamma E||grad F(w_j)||^2).  grad_out: HOST, |w| floats in the
 * layout of the parameters.  fp32 with fp64 sums over chunks of samples, through a work area that the
 * context allocates at the first call and keeps (SSGD_ENOMEM if it does not fit).  Linear models need d % 4 == 0, else
 * SSGD_EINVAL.  The two-layer network: with the arithmetic of its training gradients (bf16 operands in
 * the two large contractions, fp32 accumulation), the data set in blocks of up to 256 x 64 rows that are
 * added on the host in fp64; parameters, trace and mini-batches in flight are untouched. */
ssgd_status ssgd_full_gradient(ssgd_ctx *ctx, int32_t replica, float *grad_out);

/* ssgd_full_gradient for callers that cannot allocate device memory (code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc): the same kernels in the same launch shape,
 * hence the same values bit for bit, but the intermediate results (partial gradients) live in a static
 * device array of the library, 36 MiB that every GPU the library runs on holds until the process ends, and the gradient is written to
 * grad_out_device (DEVICE, |w| floats, layout of the parameters).  The call allocates and frees
 * nothing, copies nothing to the host and does not wait: the work is enqueued on the context's stream
 * and the result is complete when that stream reaches the end of it.  Data sets that the array is not
 * meant for (16 N + min(64, ceil(N / 256)) * classes * (d + 1) > 4 Mi) give SSGD_EINVAL,
 * as do the shapes ssgd_full_gradient refuses.  All calls on one GPU, from any context, share that
 * GPU's array: calls that overlap on one GPU (different streams or threads) race; calls on one stream
 * are ordered.  Nothing in the array has to be zero at entry: a call writes every word before it
 * reads it, so the contents left by an earlier, larger call do not matter. */
ssgd_status ssgd_full_gradient_static(ssgd_ctx *ctx, int32_t replica, float *grad_out_device);

/* The mini-batch each worker of a K-async run has in flight (Sec. 2.2: a worker that is not
 * among the K selected keeps computing on the parameters it read): version read tau_i, ordinal,
 * absolute finish time f_i.  HOST arrays of P entries, each nullable.  SSGD_EINVAL for the
 * synchronous variants, which restart every worker at every update. */
ssgd_status ssgd_get_workers(ssgd_ctx *ctx, int32_t replica, int32_t *tau, int32_t *ord, double *finish);

/* Snapshot and resume.  A snapshot holds everything later updates depend on: the trace so far,
 * update count, simulated clock, current K and the AdaSync bookkeeping, every worker's tau_i and
 * f_i, the parameters, and the gradients (linear models) or gradient factors (MLP) of the
 * mini-batches in flight, which were taken at parameters that no longer exist.  It is an opaque
 * HOST buffer of ssgd_state_bytes() bytes (the size grows with the trace); ssgd_set_state accepts
 * it only on a context created with the same model shape, P, m, variant, replicas, seed and
 * AdaSync mode and only if its size fits the number of updates its header states (else
 * SSGD_EINVAL, context unchanged), replaces that context's state and trace, and the updates that
 * follow are those the original context would have run.  A device error while the state is
 * copied leaves the context unusable (SSGD_ESTATE from then on).  The data set is not part of
 * the snapshot and has to be the one that the snapshot was taken with: the rows of mini-batches in
 * flight of SSGD_MLP2 are read from it again. */
ssgd_status ssgd_state_bytes(ssgd_ctx *ctx, int64_t *bytes);
ssgd_status ssgd_get_state(ssgd_ctx *ctx, void *host_buf, int64_t bytes);
ssgd_status ssgd_set_state(ssgd_ctx *ctx, const void *host_buf, int64_t bytes);

/* Monte-Carlo estimate of the runtime per iteration T (Sec. 2.3, Lemmas 1-3;
 * the simulation behind Fig. 6).  Trial r draws P fresh delays; for every K in
 * [Kmin, Kmax] the variant's event process is run for chain_len updates from that
 * fresh start and T_l (l = 1..chain_len) is recorded; for SSGD_K_BATCH_ASYNC (Lemma 5)
 * the pushes of all workers form one sequence for every K and update l is push l K.
 * P <= 256, chain_len <= 4096, for SSGD_K_BATCH_ASYNC chain_len * Kmax <= 7500 (else
 * SSGD_EINVAL); a rate, alpha or scale that is not above zero and a parameter that is no number give
 * SSGD_EINVAL too.  Outputs are HOST arrays of
 * (Kmax-Kmin+1) x chain_len entries: mean and unbiased variance of T_l, and
 * (nullable) the raw sums `sum` and `sumsq`; per_trial (HOST, nullable,
 * trials x (Kmax-Kmin+1) x chain_len fp64) receives every trial's T_l. */
ssgd_status ssgd_runtime_mc(int32_t variant, int32_t P, int32_t Kmin, int32_t Kmax,
                            const ssgd_delay_dist *dist, int64_t trial0, int64_t trials,
                            int32_t chain_len, uint64_t seed, void *hip_stream, double *mean,
                            double *var, double *sum, double *sumsq, double *per_trial);

/* Delays and mini-batch indices as the library draws them (DEVICE kernels, HOST
 * outputs), for bit-exact checks: n delays for raw 32-bit words, and the m sample
 * ids of the mini-batch (replica, worker, ordinal, version). */
ssgd_status ssgd_debug_delays(const ssgd_delay_dist *dist, const uint32_t *bits, int64_t n, float *out);
ssgd_status ssgd_debug_batch(uint64_t seed, uint32_t replica, uint32_t worker, uint32_t ordinal,
                             uint32_t version, int32_t m, int64_t N, uint32_t *out);

/* Measurement aid (the achievable ceiling that Sec. 6-style throughput figures of the HBM-bound paths are
 * set against): `passes` plain streaming reads of `bytes` bytes at `data` (DEVICE, 16-byte aligned), timed
 * with HIP events on hip_stream; *bytes_per_s (HOST) receives bytes read per second.  The buffer is only
 * read.  SSGD_EINVAL for a null or misaligned buffer, bytes < 16 or passes < 1. */
ssgd_status ssgd_stream_read_rate(const void *data, int64_t bytes, int32_t passes, void *hip_stream,
                                  double *bytes_per_s);

/* ------------------------------------------------------------------------------------------------
 * Operators of a low-precision training step, beside the simulated workers: the master's update as
 * an adaptive one, the norm in front of a product, and the product itself on few bits.  They take no
 * context: tensors are DEVICE pointers on the HIP device that is current, all work is enqueued on
 * `hip_stream` (a hipStream_t of that device; NULL = default stream) and nothing is awaited, allocated
 * or copied to the host unless a call says so.  Arguments are checked before anything is enqueued
 * (SSGD_EINVAL, text in ssgd_last_error(NULL)).  Rows of a matrix are contiguous and `pitch` elements
 * apart (pitch >= columns); no buffer has to be aligned beyond its element type unless that is said.  Inputs and
 * outputs must not overlap unless that is said.  A result does not depend on the stream, the pitch, the
 * alignment or on other work on the device: every sum is taken in a fixed order. */
typedef enum { SSGD_F32 = 0, SSGD_BF16 = 1 } ssgd_dtype;

/* Microscaled matrices: 32 consecutive columns of a row share the scale 2^(byte - 127), and each value is an E2M1 (4 bits: 0, 0.5,
 * 1, 1.5, 2, 3, 4, 6 and their negatives; two to a byte, the first in the low nibble) or an E4M3 (8 bits, magnitudes to 448)
 * multiple of it.  byte - 127 = floor(log2 of the block's largest magnitude) - 2 (E2M1) or - 8 (E4M3), at least -127; a value is
 * divided by the scale and rounded to the nearest of the format, ties to the even code, and to the largest where it is past it (a
 * block's largest magnitude is at most 8 / 6 or 512 / 448 of it).  A block of zeros has byte 0.  A block with an infinity or NaN
 * has byte 255 and zeros as values, and stands for NaN.
 * Layout, row-major: values rows x ssgd_mx_row_bytes(fmt, cols), scales rows x (that row's columns / 32) bytes.  Rows are padded
 * with zeros (values and scale bytes) to a multiple of 128 columns, since a product contracts 128 at a time; the padding is
 * written by ssgd_mx_quantize and ssgd_rmsnorm and relied upon by the products.  Both arrays 16-byte aligned. */
typedef enum { SSGD_MX_FP4 = 0, SSGD_MX_FP8 = 1 } ssgd_mx_format;
/* Bytes of a row of values; a row of scales has ceil(cols / 128) * 4.  -1 for an invalid argument. */
int64_t ssgd_mx_row_bytes(int32_t fmt, int64_t cols);
/* A matrix of rows x cols, quantised along its rows (values, scales in `fmt`: rows x cols), along its columns (values_t, scales_t in
 * `fmt_t`: the transposed matrix, cols x rows), or both from one read; the outputs of a direction that is not wanted are NULL. */
ssgd_status ssgd_mx_quantize(const void *x, int32_t dtype, int64_t rows, int64_t cols, int64_t pitch, int32_t fmt, void *values,
                             void *scales, int32_t fmt_t, void *values_t, void *scales_t, void *hip_stream);
/* The values read back (exact in fp32; in bf16 too, but for results outside the normal numbers). */
ssgd_status ssgd_mx_dequantize(const void *values, const void *scales, int32_t fmt, int64_t rows, int64_t cols, void *out,
                               int32_t dtype, int64_t pitch, void *hip_stream);

/* The product out[m][n] = sum over k of A[m][k] B[n][k] of microscaled matrices, A (M x K) in a_fmt, B (N x K) in SSGD_MX_FP4, both as
 * ssgd_mx_quantize lays them out; out M x N in out_dtype, rows out_pitch elements apart.  Accumulated in fp32 in a fixed order and
 * rounded once.  (The matrix unit adds 4-bit products exactly; of products of 8 by 4 bits it drops what is below about 2^-14 of the
 * largest of 128, an error of 4e-6 of a typical result.)  A block that is NaN makes the results that use it NaN.  K = 0 gives zeros; K is at most 2^24 - 128.
 * M and N are below 2^31, and refused too where a launch would need 2^32 threads: 2^23 tiles of 128 x 128 results, and for up to 16 rows of A N from
 * 2^27 (rows quantised on the way) or 2^28 on.
 * work: ssgd_mx_matmul_work_bytes bytes, 16-byte aligned (zero for most shapes: it holds the parts of a long contraction with few results). */
int64_t ssgd_mx_matmul_work_bytes(int32_t a_fmt, int64_t M, int64_t N, int64_t K);
ssgd_status ssgd_mx_matmul(const void *a_values, const void *a_scales, int32_t a_fmt, int64_t M, const void *b_values,
                           const void *b_scales, int64_t N, int64_t K, void *out, int32_t out_dtype, int64_t out_pitch,
                           void *work, void *hip_stream);
/* The same for rows x (M x K, `dtype`) that are quantised to a_fmt on the way, the results those of ssgd_mx_quantize and
 * ssgd_mx_matmul.  work: ssgd_mx_linear_work_bytes bytes, 16-byte aligned. */
int64_t ssgd_mx_linear_work_bytes(int32_t a_fmt, int64_t M, int64_t N, int64_t K);
ssgd_status ssgd_mx_linear(const void *x, int32_t dtype, int64_t pitch, int64_t M, int32_t a_fmt, const void *b_values,
                           const void *b_scales, int64_t N, int64_t K, void *out, int32_t out_dtype, int64_t out_pitch, void *work,
                           void *hip_stream);

/* The product with a dense layer's epilogue, or with that of a gated feed-forward block:
 *   p = A B^T + bias,   out[m][n] = residual + act(p[m][n])      or, gated (N even, no bias, no residual),   out[m][c] = act(p[m][2 c]) p[m][2 c + 1]
 * so a gated block's B has gate and up rows in turn.  act: none, relu, gelu (x Phi(x), Phi the normal distribution's function to 3.2e-7, below
 * zero to 16 + 1.6 x^2 units of 2^-24 of itself) or silu (x / (1 + e^-x), below zero to 7 + 1.3 |x| units);
 * infinities and NaN follow the formulas, and where Phi (x < -13.2) or the quotient (x < -87.3) is below fp32's normal numbers it may count as zero.
 * In fp32 from the product's sums on, rounded once to the output: out (M x N, gated M x N / 2) in out_dtype, or values and
 * scales (16-byte aligned), the rows quantised to SSGD_MX_FP8.  p itself goes, where the backward pass wants it, to kept (kept_dtype) or to kept_values
 * and kept_scales (SSGD_MX_FP8), all nullable.  K = 0: p = bias.
 * With A in SSGD_MX_FP8 the matrix unit drops what is below about 2^-14 of the largest of 128 products, 4e-6 of a typical p: 0.1 to 0.6 % (2-norm) of an output in 8 bits,
 * the other side of a border now and then, scales among them. */
typedef enum { SSGD_ACT_NONE = 0, SSGD_ACT_RELU = 1, SSGD_ACT_GELU = 2, SSGD_ACT_SILU = 3 } ssgd_activation;
typedef struct {
    int32_t gated, activation;
    int32_t bias_dtype, residual_dtype, out_dtype, kept_dtype;
    const void *bias;                            /* nullable, N contiguous elements */
    const void *residual; int64_t residual_pitch; /* nullable */
    void *out; int64_t out_pitch; void *values, *scales;
    void *kept; int64_t kept_pitch; void *kept_values, *kept_scales;
} ssgd_mx_epilogue;
/* A: either rows x (M x K, dtype, pitch), quantised to a_fmt on the way, or a_values and a_scales.  Limits as for ssgd_mx_matmul.  The epilogue is read during the call.
 * work: ssgd_mx_dense_work_bytes bytes, 16-byte aligned (from_rows: A is x; eight_bits: an output or what is kept is in 8 bits). */
int64_t ssgd_mx_dense_work_bytes(int32_t a_fmt, int32_t from_rows, int32_t eight_bits, int64_t M, int64_t N, int64_t K);
ssgd_status ssgd_mx_dense(const void *x, int32_t dtype, int64_t pitch, const void *a_values, const void *a_scales, int32_t a_fmt, int64_t M,
                          const void *b_values, const void *b_scales, int64_t N, int64_t K, const ssgd_mx_epilogue *epilogue, void *work,
                          void *hip_stream);
/* What lies between the products of its backward pass.  dy (rows x cols) is the gradient of act(p), or of the gated block's output, and p what the forward pass has
 * kept (rows x cols, gated rows x 2 cols): a matrix in p_dtype, or p_values and p_scales (SSGD_MX_FP8); neither is needed with SSGD_ACT_NONE, not gated.
 *   dp = dy act'(p)      gated:   dp[m][2 c] = dy u act'(g),  dp[m][2 c + 1] = dy act(g),   g = p[m][2 c], u = p[m][2 c + 1]
 * relu' is 1 where p (g) > 0 and 0 elsewhere, and selects: where it is 0, dp (dg) is zero whatever dy and u are, infinities and NaN among them.  All else are products in fp32,
 * from left to right.
 * Outputs, each nullable but one: dp quantised along its rows (values, scales in fmt) and along its columns (values_t, scales_t in fmt_t), for the products with the transposed
 * weight and with the layer's input; act(p), or the gated block's output, along its columns (values_h, scales_h in fmt_h), for the next weight's gradient; dbias
 * (fp32, not gated), the sum of dp over its rows.  rows < 2^31, columns of p up to 2^24 - 128.  work: ssgd_mx_activation_backward_work_floats floats, 16-byte aligned, used when dbias is given. */
int64_t ssgd_mx_activation_backward_work_floats(int64_t rows, int64_t cols);
ssgd_status ssgd_mx_activation_backward(const void *dy, int32_t dtype, int64_t dy_pitch, int64_t rows, int64_t cols, int32_t gated, int32_t activation,
                                        const void *p, int32_t p_dtype, int64_t p_pitch, const void *p_values, const void *p_scales, int32_t fmt,
                                        void *values, void *scales, int32_t fmt_t, void *values_t, void *scales_t, int32_t fmt_h, void *values_h,
                                        void *scales_h, float *dbias, float *work, void *hip_stream);
/* A microscaled matrix (rows x cols in fmt), quantised again along its columns: the transposed matrix in fmt_t, from the values that the first one stands for. */
ssgd_status ssgd_mx_transpose(const void *values, const void *scales, int32_t fmt, int64_t rows, int64_t cols, int32_t fmt_t, void *values_t,
                              void *scales_t, void *hip_stream);

/* Root-mean-square norm of rows of d columns with the residual's addition:
 *   s = x + residual (rounded to dtype; without a residual s = x),  rstd = (mean of s^2 + eps)^(-1/2),  y = s rstd weight
 * x, residual, sum and y have `dtype`, weight weight_dtype (d contiguous elements).  sum receives s and may be x or residual itself (same pitch); it
 * is given exactly when a residual is.  Output: either y, or values and scales (16-byte aligned), the rows quantised to SSGD_MX_FP8 (without
 * a rounding to dtype in between).  rstd (fp32, one per row) is for the backward pass.  1 <= d < 2^25; sums in fp32 and fp64, for
 * all values of the types (squares that fp32 does not hold are taken in fp64). */
ssgd_status ssgd_rmsnorm(const void *x, int64_t x_pitch, const void *residual, int64_t residual_pitch, const void *weight, int32_t dtype,
                         int32_t weight_dtype, int64_t rows, int64_t d, double eps, void *sum, int64_t sum_pitch, void *y, int64_t y_pitch,
                         void *values, void *scales, float *rstd, void *hip_stream);
/* Its gradients, from s and rstd of the forward pass: dx (the gradient of x and of the residual alike) and dweight (fp32, nullable)
 *   g = dy weight,  dx = rstd (g - s rstd mean(g s rstd)) + dsum,  dweight = sum over rows of dy s rstd
 * dsum (nullable): the gradient that reaches s past the norm.  dx may be dy, or dsum, itself (same pitch).  An output in 8 bits has the
 * gradient of the one before rounding.  work: ssgd_rmsnorm_work_floats floats, 16-byte aligned, used when dweight is given. */
int64_t ssgd_rmsnorm_work_floats(int64_t rows, int64_t d);
ssgd_status ssgd_rmsnorm_backward(const void *dy, int64_t dy_pitch, const void *s, int64_t s_pitch, const void *weight, int32_t dtype,
                                  int32_t weight_dtype, const float *rstd, const void *dsum, int64_t dsum_pitch, int64_t rows, int64_t d,
                                  void *dx, int64_t dx_pitch, float *dweight, float *work, void *hip_stream);

/* What lies between two blocks of a residual stream: the norm behind the first, its gate, the scaled residual, and the norm in front of the second.
 *   sum = scale s + gate (o rstd_o) post_weight,   rstd_o = (mean of o^2 + eps)^(-1/2)         (rounded to dtype)
 *   y = sum rstd weight,                          rstd = (mean of sum^2 + eps)^(-1/2)
 * o, s, sum and y have `dtype`; the weights are d contiguous elements of their own types.  gate (nullable: 1): `gates` rows of d elements of gate_dtype,
 * gate_pitch apart, each for rows / gates rows of the stream that lie together (one for all: a gate per column; rows % gates == 0).  Output: y, or values and
 * scales (SSGD_MX_FP8, 16-byte aligned).  The sum is taken in fp64, rounded to fp32 and from there to dtype.  rstd_o and rstd (fp32, one per row) are for the backward
 * pass.  rows < 2^31, 1 <= d < 2^24. */
ssgd_status ssgd_block_norm(const void *o, int64_t o_pitch, const void *s, int64_t s_pitch, const void *post_weight, int32_t post_dtype,
                            const void *weight, int32_t weight_dtype, const void *gate, int32_t gate_dtype, int64_t gates, int64_t gate_pitch,
                            double scale, double eps, int32_t dtype, int64_t rows, int64_t d, void *sum, int64_t sum_pitch, void *y, int64_t y_pitch,
                            void *values, void *scales, float *rstd_o, float *rstd, void *hip_stream);
/* Its gradients, from o, sum and both rstd of the forward pass; dsum (nullable): the gradient that reaches the sum past the second norm.
 *   G = rstd (dy weight - sum rstd mean(dy weight sum rstd)) + dsum,   t = G gate post_weight
 *   grad_s = scale G,   grad_o = rstd_o (t - o rstd_o mean(t o rstd_o))
 *   dweight = sum over rows of dy sum rstd,   dpost = sum over rows of G gate o rstd_o,   dgate[g] = sum over its rows of G post_weight o rstd_o
 * dpost and dweight (fp32, nullable, given together), dgate (fp32, gates x d contiguous, nullable).  work: ssgd_block_norm_work_floats floats (gates: 1 without a
 * gate), 16-byte aligned, used when dweight is given. */
int64_t ssgd_block_norm_work_floats(int64_t rows, int64_t d, int64_t gates);
ssgd_status ssgd_block_norm_backward(const void *dy, int64_t dy_pitch, const void *o, int64_t o_pitch, const void *sum, int64_t sum_pitch,
                                     const void *post_weight, int32_t post_dtype, const void *weight, int32_t weight_dtype, const void *gate,
                                     int32_t gate_dtype, int64_t gates, int64_t gate_pitch, double scale, const float *rstd_o, const float *rstd,
                                     const void *dsum, int64_t dsum_pitch, int32_t dtype, int64_t rows, int64_t d, void *grad_o, int64_t grad_o_pitch,
                                     void *grad_s, int64_t grad_s_pitch, float *dpost, float *dweight, float *dgate, float *work, void *hip_stream);

/* AdamW over many tensors at once.  For every element, with the gradient g, the update's number t and
 *   g' = g c,   c = min(1, max_norm / (norm + 1e-6)),   norm = (sum of g^2 over all tensors)^(1/2)
 *   m  = beta1 m + (1 - beta1) g',   v = beta2 v + (1 - beta2) g'^2
 *   p  = p (1 - lr weight_decay) - lr / (1 - beta1^t)  m / ((v / (1 - beta2^t))^(1/2) + eps)
 * in fp32 (the norm in fp64; max_norm = 0: no clipping, c = 1).  Infinities and NaN follow the formulas.
 * Moments lie in arrays of ssgd_adamw_state_elements elements, in which tensor k begins behind the tensors before it, each
 * rounded up to a multiple of 128 elements (the rest of the last 128 stays zero):
 *   state_bits 32: m, v fp32 (m_scale, v_scale NULL)
 *   state_bits 8:  m and the square root of v as E4M3 values times an fp32 scale per block of 128 elements, the largest
 *                  magnitude of the block / 448 (one below 2^-100 makes the block zero).  The update uses the new moments
 *                  before they are rounded.  Rounding is stochastic: a value between two neighbours goes to the upper one
 *                  with the probability of its place between them (in 1/65536), so that averages move that a nearest
 *                  rounding would stop (beta2 = 0.999 changes v by less than half a place).  The random numbers are a hash
 *                  of (seed, t, place in the state array), so equal arguments give equal results.  The root of a v above zero is never
 *                  rounded to zero.  A block with an infinity or NaN becomes NaN in the next step. */
typedef struct ssgd_adamw ssgd_adamw; /* opaque, library-owned */
typedef struct {
    double beta1, beta2; /* in [0, 1) */
    double eps;          /* > 0, an fp32 number too */
    double max_norm;     /* >= 0; 0: no clipping; one above 0 is not 0 in fp32 */
    int32_t state_bits;  /* 32 or 8 */
    uint64_t seed;       /* of the stochastic rounding */
} ssgd_adamw_options;

/* Elements of a moment's array for these tensors (sizes >= 0; -1 for an invalid argument). */
int64_t ssgd_adamw_state_elements(int32_t tensors, const int64_t *sizes);
/* A handle for these tensors: sizes[k] elements of contiguous fp32 parameters at params[k]; copies (HOST array, nullable, and
 * its entries too) receive the new parameters in bf16; weight_decay[k] (HOST).  m and v: 16-byte aligned.  The handle keeps
 * the DEVICE pointers and a work area on the current device (this call allocates and waits). */
ssgd_status ssgd_adamw_create(int32_t tensors, const int64_t *sizes, float *const *params, void *const *copies,
                              const double *weight_decay, const ssgd_adamw_options *options, void *m, void *v,
                              float *m_scale, float *v_scale, ssgd_adamw **out);
/* Update number t (>= 1) with the gradients grads[k] (HOST array of DEVICE pointers, sizes[k] contiguous elements of grad_dtype, an
 * ssgd_dtype).  norm_out (DEVICE, nullable, one float): the norm of all gradients, written when max_norm > 0.  Steps of one handle
 * share its work area and have to be ordered among themselves. */
ssgd_status ssgd_adamw_step(ssgd_adamw *handle, const void *const *grads, int32_t grad_dtype, double lr, int64_t t,
                            float *norm_out, void *hip_stream);
/* Waits for the device and frees the work area. */
void ssgd_adamw_destroy(ssgd_adamw *handle);

/* Text of the last error of a context (ctx may be NULL: last error of a call
 * that has no context).  Valid until the next call on that context. */
const char *ssgd_last_error(const ssgd_ctx *ctx);

/* Average duration in milliseconds (HIP events on the context's stream) of the
 * gradient kernel launches of the last ssgd_run, and their number. */
ssgd_status ssgd_last_kernel_ms(const ssgd_ctx *ctx, double *avg_ms, int64_t *launches);

void ssgd_destroy(ssgd_ctx *ctx);

#ifdef __cplusplus
}
#endif
#endif /* SSGD_H */
