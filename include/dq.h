/*
 * dq.h -- C ABI of the double-quantization hot path on one AMD MI355X (gfx950).
 *
 * Method: Yu, Wu, Huang, "Double Quantization for Communication-Efficient
 * Distributed Optimization" (arXiv 1805.10111): AsyLPG (Alg. 1), Sparse-AsyLPG
 * (Alg. 2), Acc-AsyLPG (Alg. 3) for  min_x P(x) = f(x) + h(x)  (eq. (1)) with
 *   f_i(x) = log(1 + exp(-y_i a_i.x)) + (l2/2)||x||^2,   h(x) = l1 ||x||_1 .
 * The M workers of the parameter-server network are a batch dimension: every
 * entry point that takes M processes M workers (rows) in one launch.
 *
 * Conventions (all entry points)
 *  - Every data pointer is a DEVICE pointer unless the comment says "host".
 *    The dq_problem struct itself lives in host memory and holds device pointers.
 *  - The caller owns every buffer.  The library allocates nothing, frees
 *    nothing, and keeps no state between calls except a thread-local record of
 *    the last HIP error (dq_last_device_error) and the fact that a kernel's
 *    launch attribute (its on-chip memory limit) has been raised, which happens
 *    once per process on first use and is safe from concurrent threads.  No
 *    environment variable is read.
 *  - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *    Calls only enqueue work and return; results, including scalars (delta,
 *    norms, counts, status), land in device memory.  The caller synchronises.
 *  - Return value: DQ_OK, or a negative DQ_ERR_* code; on error nothing has
 *    been enqueued unless the code is DQ_ERR_DEVICE.
 *  - Alignment: vectors of floats / words that are read or written with
 *    128-bit accesses must be 16-byte aligned and row strides (`ld`, `lda`,
 *    in elements) multiples of 4; the comments say where this is required.
 *  - b is the number of bits per coordinate.  Packed buffers: any b in [2,16] for
 *    dq_quantize_pack, dq_unpack_dequant_sum and the model message (b_x); gradient
 *    messages of the worker / master calls use b in {2,4,8} (or 32 = float32, not
 *    quantized); unpacked int8 codes support any b in [2,8].
 *  - `status` (nullable) is a device uint32 that is OR-ed into, never cleared:
 *    bit 0 = a scale delta was not finite (NaN/Inf in the input vector), or a row's loss, its mean square, a matrix's norm;
 *    bit 1 = a class (label, teacher's entry) was not below the number of classes;
 *    bit 31 = dq_run_rounds, where the blocks of one launch do many rounds: they waited for each other
 *    for seconds and gave up, the state is not that of the rounds asked for.  (Without a status word no launch does
 *    many rounds that way.)
 *  - Random streams are addressed, not stateful: (seed, iter, worker, tag,
 *    coordinate) names one variate; the same address gives the same variate in
 *    any call, any launch shape.  Generator: Philox4x32-10; key = halves of
 *    seed; counter = (coordinate/4, iter, worker, tag); variate = word
 *    coordinate%4; uniform = (word >> 8) * 2^-24.
 */
#ifndef DQ_H_
#define DQ_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DQ_OK                0
#define DQ_ERR_INVALID_ARG  (-1)  /* null / misaligned pointer, size <= 0, b out of range */
#define DQ_ERR_UNSUPPORTED  (-2)  /* valid request the library has no kernel for */
#define DQ_ERR_WORKSPACE    (-3)  /* workspace smaller than dq_workspace_bytes() */
#define DQ_ERR_DEVICE       (-4)  /* a HIP call failed; see dq_last_device_error() */

/* Stream tags: which random decision a variate is used for. */
#define DQ_TAG_GRAD      0u   /* rounding of a worker's gradient (Alg. 1, worker (ii))     */
#define DQ_TAG_MODEL     1u   /* rounding of the model (Alg. 1, master (i))                */
#define DQ_TAG_SPARSIFY  2u   /* Bernoulli keep decisions of eq. (3)                       */
#define DQ_TAG_SAMPLE    3u   /* mini-batch sampling (Alg. 1, worker (i))                  */
#define DQ_MASTER_ID     0xFFFFFFFFu   /* worker id used for the master's own stream       */

/* Finite-sum problem of eq. (1) with logistic loss (Section 5.1).
 * layout 0: dense row-major features, row i at dense + i*lda, lda % 4 == 0, lda >= d,
 *           dense 16-byte aligned and n*lda floats long (the padding of a row may be read, never used).
 * layout 1: CSR; indptr[n+1], indices sorted and unique within a row; indices and values must
 *           be non-null even when the matrix has no nonzeros (they are then never read).  lda: the number of
 *           nonzeros if the caller knows it, else 0; it only helps to choose between launches with the same results.
 * y[n] holds +1/-1.  l2 multiplies ||x||^2/2 inside every f_i (smooth part),
 * l1 multiplies ||x||_1 in h (handled by the prox). */
typedef struct dq_problem {
    int32_t layout;
    int64_t n, d;
    const float *dense;
    int64_t lda;
    const int64_t *indptr;
    const int32_t *indices;
    const float *values;
    const float *y;
    float l2, l1;
} dq_problem;

/* Operations that need a workspace (argument of dq_workspace_bytes). */
#define DQ_OP_FULL_GRAD    1
#define DQ_OP_VR_GRAD      2   /* dq_vr_grad, dq_worker_step and dq_run_rounds (which also keeps data there between the
                                  rounds of a call) */
#define DQ_OP_WORKER_STEP  3   /* one dq_vr_grad or dq_worker_step call alone: never more than DQ_OP_VR_GRAD */

const char *dq_version(void);
/* Last hipError_t (as int) seen by this thread inside the library, 0 if none. */
int32_t dq_last_device_error(void);
/* Bytes of device workspace `op` needs for this problem with M workers of batch B
 * (a multiple of 16, possibly 0; negative = DQ_ERR_*).  Workspaces are 16-byte aligned.
 * Limits that make a problem DQ_ERR_UNSUPPORTED: dense rows wider than 16384 floats; CSR with 2^20
 * columns or more. */
int64_t dq_workspace_bytes(int32_t op, const dq_problem *prob /*host*/, int64_t M, int64_t B);
/* Zero-fills a workspace (optional: no operation needs initialised workspace memory;
 * provided so that a caller can keep its buffers defined).  Two calls that share a
 * workspace must not run concurrently.  ws_bytes must be a multiple of 16. */
int32_t dq_workspace_init(void *ws, int64_t ws_bytes, void *stream);

/* ---- Section 3.1: the (delta, b) representation and the quantizer Q ------------- */

/* absmax_out[m] = ||v_m||_inf for M rows v_m = v + m*ld of length d
 * (numerator of delta in Alg. 1, master (i) and worker (ii)).
 * A NaN anywhere in a row gives a NaN result (max over the magnitude bit patterns). */
int32_t dq_absmax(const float *v, int64_t d, int64_t M, int64_t ld, float *absmax_out, void *stream);

/* Stochastic quantization Q_(delta,b) of Section 3.1, coordinate-wise, with
 * delta_m = ||v_m||_inf / (2^(b-1)-1).  codes_out[m*ld_codes + i] = k with
 * Q(v_mi) = k*delta_m.  Row m uses the stream (seed, iter, worker0+m, tag).
 * Per coordinate (float32): t = v*(L/amax), z = floor(t), k = z + [u < t-z],
 * clamped to [-2^(b-1), 2^(b-1)-1].  A row whose delta is zero or below the
 * smallest normal float gives delta 0 and all-zero codes; a non-finite delta
 * gives zero codes and sets status bit 0.
 * absmax: device float[M]; if absmax_given == 0 it is overwritten with
 * ||v_m||_inf first, else it is read as supplied.  delta_out: device float[M]. */
int32_t dq_quantize(const float *v, int64_t d, int64_t M, int64_t ld, int32_t b,
                    float *absmax, int32_t absmax_given,
                    uint64_t seed, uint32_t iter, uint32_t tag, uint32_t worker0,
                    int8_t *codes_out, int64_t ld_codes, float *delta_out,
                    uint32_t *status, void *stream);

/* v_out[m*ld + i] = delta[m] * codes[m*ld_codes + i]  (the value a code represents). */
int32_t dq_dequantize(const int8_t *codes, int64_t ld_codes, const float *delta, int64_t d, int64_t M,
                      float *v_out, int64_t ld, void *stream);

/* Wire format of Section 3.1 (32 + b*d bits per vector: delta plus b bits per
 * coordinate).  Field i of a row = bits [(i*b)%32, (i*b)%32+b) of word
 * floor(i*b/32), two's complement, low bits first; unused tail bits are 0.
 * For a width that does not divide 32 the row is one little-endian bit string with field i at
 * bits [i*b, i*b+b): a field may continue in the low bits of the next word (the model-precision
 * study of Section 5.2 uses b_x from 2 to 11).
 * Rows of packed words have stride ld_words >= ceil(d*b/32).  b in [2,8] here (int8 codes);
 * dq_quantize_pack, dq_unpack_dequant_sum and the model message of the worker and master
 * calls take any width in [2,16]. */
int32_t dq_pack(const int8_t *codes, int64_t ld_codes, int64_t d, int64_t M, int32_t b,
                uint32_t *packed_out, int64_t ld_words, void *stream);
int32_t dq_unpack(const uint32_t *packed, int64_t ld_words, int64_t d, int64_t M, int32_t b,
                  int8_t *codes_out, int64_t ld_codes, void *stream);

/* Sparse message of Section 4.2 (after sparsification most codes are zero): the scale plus,
 * per NONZERO coordinate in ascending order, an entry of ceil(log2 d) position bits (low) and
 * the b-bit two's-complement code (high), entries back to back, low bits first across 32-bit
 * words: 32 + nnz*(ceil(log2 d) + b) bits in all.  dq_sparse_stream_words(d, b) is the row
 * capacity (every coordinate nonzero).  dq_sparse_encode turns M rows of dense packed codes
 * into M streams (stride ld_stream >= capacity, words past the used ones zero) and writes
 * nnz_out[M]; dq_sparse_decode is the inverse (packed_out rows fully rewritten).  Either may work in place (equal strides).  b in {2,4,8};
 * streams of more than 36864 words (144 KB) are DQ_ERR_UNSUPPORTED. */
int64_t dq_sparse_stream_words(int64_t d, int32_t b);
int32_t dq_sparse_encode(const uint32_t *packed, int64_t ld_words, int64_t d, int64_t M, int32_t b,
                         uint32_t *stream_out, int64_t ld_stream, int32_t *nnz_out, void *stream);
int32_t dq_sparse_decode(const uint32_t *stream_in, int64_t ld_stream, const int32_t *nnz, int64_t d, int64_t M,
                         int32_t b, uint32_t *packed_out, int64_t ld_words, void *stream);

/* dq_quantize followed by dq_pack in one pass (same bits as the two calls), for any
 * width b in [2,16] (2, 4 and 8 take the word-aligned fast path).
 * v and packed_out 16-byte aligned; with M > 1, ld % 4 == 0 and ld_words % 4 == 0. */
int32_t dq_quantize_pack(const float *v, int64_t d, int64_t M, int64_t ld, int32_t b,
                         float *absmax, int32_t absmax_given,
                         uint64_t seed, uint32_t iter, uint32_t tag, uint32_t worker0,
                         uint32_t *packed_out, int64_t ld_words, float *delta_out,
                         uint32_t *status, void *stream);

/* Master's receive side (Alg. 1, master (ii), first half): decode M packed
 * gradients and aggregate,  out[i] = scale * sum_{m<M} delta[m]*k_mi,
 * summed in the order m = 0..M-1 with fused multiply-adds, then one multiply
 * by scale (1/M for the mean over a synchronous round of M workers).  b in [2,16]. */
int32_t dq_unpack_dequant_sum(const uint32_t *packed, int64_t ld_words, const float *delta,
                              int64_t d, int64_t M, int32_t b, float scale, float *out, void *stream);

/* ---- sampling, gradients -------------------------------------------------------- */

/* Mini-batch of Alg. 1, worker (i) (Section 5.1 uses mini-batches): for worker
 * m and slot j, idx_out[m*B + j] = floor(word * n / 2^32) with the variate at
 * (seed, iter, worker0+m, DQ_TAG_SAMPLE, j): uniform on {0..n-1}, with replacement. */
int32_t dq_sample_indices(int64_t n, int64_t M, int64_t B, uint64_t seed, uint32_t iter,
                          uint32_t worker0, int32_t *idx_out, void *stream);

/* Epoch prologue (Alg. 1, global gradient computation):
 *   g_out = (1/n) sum_i grad f_i(x) = (1/n) sum_i s_i a_i + l2*x,
 *   s_i = -y_i / (1 + exp(y_i a_i.x)).
 * z_out (nullable, float[n]) receives the margins a_i.x; obj_out (nullable,
 * double[1]) receives P(x) of eq. (1).  Deterministic for a given problem shape (dense features: float32
 * sums in a fixed order; CSR features: the sums over rows are accumulated per column in fixed point -- int32
 * multiples of a power of two chosen so that no sum can overflow, flushed to float32 every 1024 rows -- and do
 * not depend on the order of the additions; a term is rounded to within 2^-31 of the bound of its column's sum). */
int32_t dq_full_grad(const dq_problem *prob /*host*/, const float *x, float *g_out, float *z_out,
                     double *obj_out, void *ws, int64_t ws_bytes, void *stream);

/* Worker step (i) of Alg. 1 for M workers with mini-batches idx[m*B .. m*B+B):
 *   alpha_m = (1/B) sum_{i in I_m} [grad f_i(q) - grad f_i(x_snap)],
 * q = delta_x * (codes unpacked from xq_packed) is the b_x-bit model the worker
 * received (Alg. 1, master (i)), b_x in [2,16]; b_x == 32 means xq_packed holds float32
 * values of the model itself (no quantization; delta_x ignored).
 * model_is_snapshot != 0 is the flag-bit case of Section 4.1 (q = x_snap): alpha = 0.
 * z_snap (nullable) = margins a_i.x_snap cached by dq_full_grad; if NULL they
 * are recomputed.  alpha_out rows have stride ld (ld % 4 == 0, 16-byte aligned).
 * absmax_out[M] = ||alpha_m||_inf; l1norm_out (nullable) [M] = ||alpha_m||_1.
 * CSR features: the sum over the mini-batch is accumulated in fixed point as in dq_full_grad (bit-reproducible;
 * the bound, hence the unit, follows the size of the coefficients, which shrink as q approaches x_snap); a NaN
 * or Inf among the values, labels or cached margins of a mini-batch makes the whole alpha_m NaN. */
int32_t dq_vr_grad(const dq_problem *prob /*host*/, const int32_t *idx, int64_t M, int64_t B,
                   const uint32_t *xq_packed, const float *delta_x, int32_t b_x,
                   int32_t model_is_snapshot, const float *x_snap, const float *z_snap,
                   float *alpha_out, int64_t ld, float *absmax_out, float *l1norm_out,
                   void *ws, int64_t ws_bytes, void *stream);

/* Eq. (3), gradient sparsification (Alg. 2, worker (ii)):
 *   beta_i = Z_i alpha_i / p_i,  Z_i ~ Bernoulli(p_i)  (keep iff u_i < p_i),
 * phi == NULL: the budget of Section 5.1, phi = ||alpha||_1/||alpha||_inf, i.e.
 *   p_i = |alpha_i| / ||alpha||_inf;
 * else p_i = min(1, |alpha_i| * phi[m] / ||alpha_m||_1)  (Lemma 2).
 * Outputs: beta_out (stride ld_out), absmax_out[M] = ||beta_m||_inf,
 * nnz_out[M] = kept coordinates.  Stream tag DQ_TAG_SPARSIFY. */
int32_t dq_sparsify(const float *alpha, int64_t d, int64_t M, int64_t ld, const float *phi,
                    uint64_t seed, uint32_t iter, uint32_t worker0,
                    float *beta_out, int64_t ld_out, float *absmax_out, int32_t *nnz_out, void *stream);

/* The whole worker side of one round, fused (Alg. 1, worker (i)-(ii); with
 * sparsify != 0: Alg. 2, worker (i)-(iii)):  dq_vr_grad -> [dq_sparsify] ->
 * dq_quantize_pack with tag DQ_TAG_GRAD, bit-identical to those calls, without
 * writing alpha to memory (dense features with B > 32: partial sums of alpha pass through
 * `ws`; CSR with a model too wide for the on-chip buffer: alpha passes through `ws`, in one launch
 * or between two or three; CSR with sparsify != 0 and few workers: the sparsified gradient passes
 * through `ws` between two launches).
 * ws, ws_bytes: at least dq_workspace_bytes(DQ_OP_WORKER_STEP, prob, M, B) bytes (a DQ_OP_VR_GRAD workspace is never
 * smaller).  CSR features whose model fits the on-chip buffer also run without (NULL, 0), in a single launch.  packed_out: M rows of ld_words words; delta_out[M];
 * nnz_out (nullable) [M] = nonzero codes.  alpha_out (nullable): also store alpha.
 * idx == NULL: the mini-batches are sampled inside the kernel, exactly as
 * dq_sample_indices(n, M, B, seed, iter, worker0, .) would produce them.
 * b == 32: no gradient quantization, packed_out rows receive alpha (or beta) as
 * float32 (ld_words >= d) and delta_out = 1.  Gradient widths: b in {2,4,8,32}
 * (others in [2,8]: DQ_ERR_UNSUPPORTED). */
int32_t dq_worker_step(const dq_problem *prob /*host*/, const int32_t *idx, int64_t M, int64_t B,
                       const uint32_t *xq_packed, const float *delta_x, int32_t b_x,
                       int32_t model_is_snapshot, const float *x_snap, const float *z_snap,
                       int32_t sparsify, int32_t b, uint64_t seed, uint32_t iter, uint32_t worker0,
                       uint32_t *packed_out, int64_t ld_words, float *delta_out, int32_t *nnz_out,
                       float *alpha_out, int64_t ld, uint32_t *status,
                       void *ws, int64_t ws_bytes, void *stream);

/* dq_worker_step for callers that cannot allocate device memory or hand over a workspace (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): same arguments without ws / ws_bytes, same
 * results bit for bit.  The partial sums and per-worker rows that dq_worker_step passes through `ws` live in a
 * workspace of DQ_STATIC_WS_BYTES bytes built into the library, one copy per GPU, held until the process ends;
 * nothing is allocated or freed by the call.  A problem whose dq_workspace_bytes(DQ_OP_WORKER_STEP, prob, M, B) exceeds
 * DQ_STATIC_WS_BYTES returns DQ_ERR_WORKSPACE and enqueues nothing.  All calls on one GPU share that workspace:
 * calls that may overlap on the GPU (different streams without an ordering between them) race; calls on one
 * stream, or otherwise ordered, are safe, and no call depends on what an earlier one left there. */
#define DQ_STATIC_WS_BYTES  (8ll << 20)
int32_t dq_worker_step_static(const dq_problem *prob /*host*/, const int32_t *idx, int64_t M, int64_t B,
                              const uint32_t *xq_packed, const float *delta_x, int32_t b_x,
                              int32_t model_is_snapshot, const float *x_snap, const float *z_snap,
                              int32_t sparsify, int32_t b, uint64_t seed, uint32_t iter, uint32_t worker0,
                              uint32_t *packed_out, int64_t ld_words, float *delta_out, int32_t *nnz_out,
                              float *alpha_out, int64_t ld, uint32_t *status, void *stream);

/* ---- master --------------------------------------------------------------------- */

/* Master step for one synchronous round of M workers (Alg. 1, master (ii) and (i);
 * Alg. 3 with y != NULL):
 *   u     = scale * sum_m delta[m]*k_m + g_snap                    (as dq_unpack_dequant_sum)
 *   Alg.1: x <- prox_{eta h}(x - eta*u)         prox = soft-threshold at eta*l1
 *   Alg.3: y <- prox_{eta h}(y - eta*u);  x <- x_snap + theta*(y - x_snap);  xsum += x
 * then the new model is quantized to b_x bits with the master's stream
 * (seed, iter, DQ_MASTER_ID, DQ_TAG_MODEL) and packed into xq_packed_out, with
 * delta_x_out[0] its scale and absmax_x_out[0] = ||x||_inf (scratch + output).
 * b == 32: `packed` holds M rows of float32 gradients (stride ld_words, delta
 * ignored).  b_x == 32: no model quantization, xq_packed_out receives x as float32.
 * b in {2,4,8,32}; b_x in [2,16] or 32.  One launch for d <= 8192 (for b_x other than 2, 4, 8, 32
 * only up to M*d = 250,000, dq_master_step_each 100,000), else three (update with ||x||_inf, quantize + pack, and a
 * one-word fill before them).
 * All float32, in the order written; x, y, xsum are updated in place. */
int32_t dq_master_step(const uint32_t *packed, int64_t ld_words, const float *delta, int64_t M, int32_t b,
                       float scale, const float *g_snap, float *x, float *y, const float *x_snap,
                       float *xsum, float eta, float theta, float l1, int64_t d,
                       int32_t b_x, uint64_t seed, uint32_t iter,
                       uint32_t *xq_packed_out, float *delta_x_out, float *absmax_x_out,
                       uint32_t *status, void *stream);

/* The master's rule of Alg. 1 (Alg. 3 with y != NULL) taken one received gradient at a time: the M
 * messages are applied in worker order, each as its own update with the full step,
 *   for m:  u = delta[m]*k_m + g_snap;  x <- prox_{eta h}(x - eta*u)
 *           (Alg. 3: y <- prox_{eta h}(y - eta*u);  x <- x_snap + theta*(y - x_snap);  xsum += x, i.e. M terms per call),
 * then the model is quantized and packed once, exactly as in dq_master_step.  Same arguments
 * without `scale`, same limits. */
int32_t dq_master_step_each(const uint32_t *packed, int64_t ld_words, const float *delta, int64_t M, int32_t b,
                            const float *g_snap, float *x, float *y, const float *x_snap,
                            float *xsum, float eta, float theta, float l1, int64_t d,
                            int32_t b_x, uint64_t seed, uint32_t iter,
                            uint32_t *xq_packed_out, float *delta_x_out, float *absmax_x_out,
                            uint32_t *status, void *stream);

/* The two sides of the precision-loss condition on the model quantization (eq. (2); eq. (4) for
 * Alg. 3):  out[0] = E_Q ||Q_(delta_x,b)(x) - x||^2 over the rounding decisions, which is
 * delta_x^2 * sum_i p_i (1 - p_i) (proof of Lemma 5; nothing is sampled), and
 * out[1] = ||x - x_snap||^2.  The condition holds for a given mu iff out[0] <= mu * out[1]
 * (theta_s * mu for Alg. 3).  out: device double[2].  b in [2,16].  Diagnostic, one block. */
int32_t dq_mu_terms(const float *x, const float *x_snap, int64_t d, int32_t b, double *out, void *stream);

/* Parameters of epoch s = 1, 2, ... of Alg. 3 as Section 5.1 sets them: theta_s = 2/(s+2), eta_s = lr/theta_s,
 * both in float32.  theta_out, eta_out: HOST pointers.  s < 1: DQ_ERR_INVALID_ARG. */
int32_t dq_acc_params(float lr, int64_t s, float *theta_out /*host*/, float *eta_out /*host*/);

/* Start of an epoch of Alg. 3:  x_out = x_snap + theta*(y - x_snap)  (= theta*y + (1-theta)*x_snap). */
int32_t dq_acc_mix(const float *y, const float *x_snap, float theta, int64_t d, float *x_out, void *stream);
/* End of an epoch of Alg. 3:  x_snap_out = xsum / m. */
int32_t dq_acc_snapshot(const float *xsum, int64_t m, int64_t d, float *x_snap_out, void *stream);

/* ---- models of many classes ------------------------------------------------------- */

/* The binary model of eq. (1) taken to c classes: a row a_t of features has the scores z_t = W a_t, W [c][d].
 * Types of the features and of the model (one for both, and for their gradients): float32, float16, bfloat16.  Sums, scores, their
 * maxima and sums of exponentials, and losses are float32 (what 16-bit gradients are made from: at dq_class_grad); products of
 * float32 are carried out to float32's own precision on the matrix cores, in three bfloat16 parts (magnitudes of 2^127 * 1.99 and
 * more count as infinite; of those below 2^-110 what is left are multiples of 2^-133; anything not finite gives losses that are not
 * finite). */
#define DQ_F32   0
#define DQ_F16   1
#define DQ_BF16  2

/* Host struct: n rows of features and a model of c classes, both d wide; lda, ldw: elements from one row to the next (>= d; any,
 * as any alignment to the element, but 16-bit rows that are 16-byte aligned with d % 8 == 0 are read in place). */
typedef struct dq_classes {
    int32_t type;                    /* DQ_F32, DQ_F16, DQ_BF16 */
    int64_t n, c, d;
    const void *a; int64_t lda;
    const void *w; int64_t ldw;
} dq_classes;

/* Host struct: a teacher's largest logits.  Row t's entries are cls[t*ld + j], logit[t*ld + j], j < k, in any order; a class below 0
 * is an entry that is not there.  A class that comes twice counts twice.  tau > 0: the temperature (finite, and so is 1 / tau). */
typedef struct dq_teacher {
    int64_t k;
    const int32_t *cls;
    const float *logit;
    int64_t ld;
    float tau;
} dq_teacher;
#define DQ_MAX_TEACHER 1024          /* largest k */

#define DQ_OP_CLASS_LOSS  4   /* dq_class_loss, dq_distill_loss */
#define DQ_OP_CLASS_GRAD  5   /* dq_class_grad, dq_distill_grad */
/* Bytes of workspace of `op`, as dq_workspace_bytes; k: the teacher's, 0 for labels.  The scores of all classes are never kept:
 * the gradients take the classes in pieces whose n columns of gradients fit 1 GB.  DQ_ERR_UNSUPPORTED, here and in the calls: more than 2^30
 * classes, 2^20 columns, strides of 2^22 or DQ_MAX_TEACHER entries, and what no launch takes: 2^28 rows (2^26 with a teacher), 2^23 tiles of
 * 256 x 256 scores (float32: 256 x 128; up to 64 rows: 2^24 tiles of 64 classes). */
int64_t dq_class_workspace_bytes(int32_t op, const dq_classes *prob /*host*/, int64_t k);

/* Softmax cross entropy: loss_out[t] = lse_t - z_t,label[t],  lse_t = log sum_j exp z_tj  (lse_out nullable).
 * A row with a label below 0 is left out: its loss is 0 (its lse is still written).  A label of c or more leaves the row out too and
 * sets status bit 1.  Status bit 0: the lse or the loss of a row that is not left out is not finite. */
int32_t dq_class_loss(const dq_classes *prob /*host*/, const int32_t *label, float *loss_out, float *lse_out,
                      uint32_t *status, void *ws, int64_t ws_bytes, void *stream);

/* The same losses, and the gradients of  scale * sum_t weight[t] loss_t  (weight nullable: all 1):
 *   g_tj = scale weight_t (softmax(z_t)_j - [j = label_t]),   da_out = g W  [n][ldda],   dw_out = g^T a  [c][lddw],
 * either nullable, of the problem's type, whole (rows left out: zeros in da_out, nothing to dw_out, whatever the row holds).
 * loss_out, lse_out nullable.  Deterministic: sums in a fixed order.  The outputs must not overlap the inputs.
 * g is rounded to the problem's type for the two products (float32: kept whole), by up to 2^-8 of each term in bfloat16 and 2^-11 in
 * float16, there as a multiple of the largest finite |weight| that keeps terms down to 2^-28 of it normal.  Before that, in 16-bit calls of more
 * than 64 rows, softmax(z_t)_j of classes without a target is off by a factor of up to 1 -+ 0.00071 in bfloat16 and 0.00018 in float16 (kept as a
 * 16-bit logarithm; classes behind the first piece: not), and zero below 2^-128 (float16 2^-32) of the largest among its tile's, 128 or 256
 * neighbouring classes. */
int32_t dq_class_grad(const dq_classes *prob /*host*/, const int32_t *label, const float *weight, float scale,
                      float *loss_out, float *lse_out, void *da_out, int64_t ldda, void *dw_out, int64_t lddw,
                      uint32_t *status, void *ws, int64_t ws_bytes, void *stream);

/* Distillation: with q_t = softmax(logit_t / tau) over the entries of row t and p_t = softmax(z_t / tau) over all classes,
 *   loss_out[t] = tau^2 sum_j q_tj (log q_tj - log p_tj),   lse_out[t] = log sum_j exp(z_tj / tau).
 * A row without an entry (or whose logits are all -inf) is left out, as above.  Entries with a class of c or more are not there, and
 * set status bit 1.  An entry whose logit is a NaN or +inf makes its row's loss and da, and dW of its classes, NaN (status bit 0). */
int32_t dq_distill_loss(const dq_classes *prob /*host*/, const dq_teacher *teacher /*host*/, float *loss_out, float *lse_out,
                        uint32_t *status, void *ws, int64_t ws_bytes, void *stream);
/* The same with gradients:  g_tj = scale weight_t tau (p_tj - q_tj). */
int32_t dq_distill_grad(const dq_classes *prob /*host*/, const dq_teacher *teacher /*host*/, const float *weight, float scale,
                        float *loss_out, float *lse_out, void *da_out, int64_t ldda, void *dw_out, int64_t lddw,
                        uint32_t *status, void *ws, int64_t ws_bytes, void *stream);

/* ---- models in 4 bits --------------------------------------------------------------- */

/* A matrix in microscaled 4-bit numbers (the (delta, b) idea with one power-of-two scale per 32 neighbours, and levels that the
 * matrix cores multiply): value = level * 2^(scale - 127), level one of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} (code: sign bit 8, the
 * level's number below it).  A row of d numbers is stored in whole groups of 128: dq_mx4_row_bytes(d) bytes of codes (number 2i in
 * the low half of byte i) and dq_mx4_row_scales(d) bytes of scales, codes behind the row's end zero, their scales finite (not 255;
 * dq_mx4_quantize writes 0).  codes 16-byte aligned with ld_codes % 16 == 0, scales 4-byte aligned with ld_scales % 4 == 0. */
typedef struct dq_mx4 {
    int64_t n, d;
    uint8_t *codes; int64_t ld_codes;
    uint8_t *scales; int64_t ld_scales;
} dq_mx4;
int64_t dq_mx4_row_bytes(int64_t d);
int64_t dq_mx4_row_scales(int64_t d);

/* q = v rounded, v [q.n][ld] of `type`, q.d wide: scale exponent floor(log2 of the block's largest magnitude) - 2, at least -127; each
 * number to the nearest level, ties to the even code, beyond 6 to 6.  A block with an infinity or a NaN gets scale 255 (all its
 * values are NaN) and sets status bit 0.  Its gradient in training is taken straight through (the identity). */
int32_t dq_mx4_quantize(const void *v, int32_t type, int64_t ld, const dq_mx4 *q /*host*/, uint32_t *status, void *stream);
/* out = the values of q (exact in every type for scales that the type can hold, else rounded once). */
int32_t dq_mx4_dequantize(const dq_mx4 *q /*host*/, void *out, int32_t type, int64_t ld, void *stream);

/* out[t][j] = sum_i a_ti w_ji over a.d = w.d, products exact, sums float32: [a.n][ld] of `type`. */
int32_t dq_mx4_product(const dq_mx4 *a /*host*/, const dq_mx4 *w /*host*/, void *out, int32_t type, int64_t ld, void *stream);

/* Scores of n rows against a model in 4 bits: dq_mx4_quantize of the rows, then dq_mx4_product, `type` and `out_type` their types.
 * ws: at least dq_mx4_scores_bytes(n, w.d) bytes. */
int64_t dq_mx4_scores_bytes(int64_t n, int64_t d);
int32_t dq_mx4_scores(const void *a, int32_t type, int64_t n, int64_t lda, const dq_mx4 *w /*host*/, void *out, int32_t out_type,
                      int64_t ld, uint32_t *status, void *ws, int64_t ws_bytes, void *stream);

/* ---- models in 8 bits --------------------------------------------------------------- */

/* A matrix in 8-bit blocks: value = number * 2^(scale - 127), one scale per 128 neighbours of a row, numbers of e4m3 (sign, four bits of
 * exponent with bias 7, three behind the leading one, no infinities; largest 448).  A row of d numbers is stored in whole blocks:
 * dq_fp8_row_bytes(d) bytes of codes, dq_fp8_row_scales(d) bytes of scales (a multiple of four), zeros behind the row's end (dq_fp8_quantize
 * writes them).  codes 16-byte aligned with ld_codes % 16 == 0, scales 4-byte aligned with ld_scales % 4 == 0. */
typedef struct dq_fp8 {
    int64_t n, d;
    uint8_t *codes; int64_t ld_codes;
    uint8_t *scales; int64_t ld_scales;
} dq_fp8;
int64_t dq_fp8_row_bytes(int64_t d);
int64_t dq_fp8_row_scales(int64_t d);

/* v [n][ld] of `type`, d wide, to 8 bits along its rows (q: n x d) and along its columns (qt: the transpose, d x n); either nullable.  A block's scale
 * exponent is the least e >= -127 with (largest magnitude) <= 448 * 2^e; each number goes to the nearest, ties to the even code.  A block
 * with an infinity or a NaN gets scale 255 (all its values are NaN) and sets status bit 0.  Its gradient in training is taken straight through.
 * DQ_ERR_UNSUPPORTED, here and below: more than 2^30 rows, 2^21 columns or strides of 2^22, and more blocks than a launch has. */
int32_t dq_fp8_quantize(const void *v, int32_t type, int64_t n, int64_t d, int64_t ld, const dq_fp8 *q /*host*/, const dq_fp8 *qt /*host*/,
                        uint32_t *status, void *stream);
/* out = the values of q (exact in every type for scales that the type can hold, else rounded once). */
int32_t dq_fp8_dequantize(const dq_fp8 *q /*host*/, void *out, int32_t type, int64_t ld, void *stream);

/* out[t][j] = sum_i a_ti w_ji over a.d = w.d, products exact, sums float32 in a fixed order: [a.n][ld] of `type`.  (With 16-bit results of more than 64
 * rows, or of more than 16 and 4096 columns, the matrix cores leave out, of the eight neighbouring products that they take together, what is less than 2^-13 of
 * the power of two of the largest: 1.5 10^-5 of a sum of normally distributed numbers.  Otherwise numbers below 2^-126 may count as zero.)  All three products of a layer
 * z = a w^T are of this form: z from a and w along their rows, da = g w from g along its rows and w along its columns, dw = g^T a from
 * g and a along their columns.  ws: at least dq_fp8_product_bytes(type, a.n, w.n, a.d) bytes (where that is 0: may be null). */
int64_t dq_fp8_product_bytes(int32_t type, int64_t n, int64_t c, int64_t d);
int32_t dq_fp8_product(const dq_fp8 *a /*host*/, const dq_fp8 *w /*host*/, void *out, int32_t type, int64_t ld, void *ws, int64_t ws_bytes,
                       void *stream);

/* Scores of n rows against a model in 8 bits: dq_fp8_quantize of the rows, then dq_fp8_product, `type` and `out_type` their types.
 * ws: at least dq_fp8_scores_bytes(out_type, n, w.n, w.d) bytes. */
int64_t dq_fp8_scores_bytes(int32_t out_type, int64_t n, int64_t c, int64_t d);
int32_t dq_fp8_scores(const void *a, int32_t type, int64_t n, int64_t lda, const dq_fp8 *w /*host*/, void *out, int32_t out_type,
                      int64_t ld, uint32_t *status, void *ws, int64_t ws_bytes, void *stream);

/* ---- the rows' norm ------------------------------------------------------------------ */

/* Host struct: n rows of `type`, d wide; h_t = x_t + residual_t, rounded to the type (residual nullable: h = x), and
 *   y_t = h_t s_t gain,   s_t = 1 / sqrt(mean_j h_tj^2 + eps),   gain [d] float32 (nullable: ones), eps > 0.
 * ldx, ldr: elements from one row to the next (>= d; any, as any alignment to the element).  DQ_ERR_UNSUPPORTED: more than 2^30 rows, 2^22
 * columns, or more rows than a launch of dq_rms_norm has (2^22 of more than 8192 columns, 2^24 of more than 1024). */
typedef struct dq_norm {
    int32_t type;
    int64_t n, d;
    const void *x; int64_t ldx;
    const void *residual; int64_t ldr;
    const float *gain;
    float eps;
} dq_norm;

/* h_out (only with a residual) = h, out = y, both of p.type; q = y in 8-bit blocks (of float32 rows as if y were rounded once, of 16-bit rows from its float32 value): each nullable, not all.
 * h_out may be x or the residual itself (their very rows), and so may out; otherwise outputs overlap neither inputs nor each other.  Status bit 0: a row's
 * mean square, or a block of q, is not finite. */
int32_t dq_rms_norm(const dq_norm *p /*host*/, void *h_out, int64_t ldh, void *out, int64_t ldo, const dq_fp8 *q /*host*/, uint32_t *status,
                    void *stream);
/* Gradients, dy that of y:  dx_out = s (u - h s^2 mean_j(u_j h_j)) + dh,  u = dy gain  (of x and of the residual alike; dh, nullable, is what arrives
 * at h from elsewhere), and dgain_out = sum_t dy_t h_t s_t, float32 (its sums in a fixed order); either nullable.  dx_out may be x, the residual, dy or
 * dh itself.  A caller that kept h passes it as x.  ws: for dgain_out, at least dq_rms_norm_grad_bytes(n, d) bytes. */
int64_t dq_rms_norm_grad_bytes(int64_t n, int64_t d);
int32_t dq_rms_norm_grad(const dq_norm *p /*host*/, const void *dy, int64_t lddy, const void *dh, int64_t lddh, void *dx_out, int64_t lddx,
                         float *dgain_out, void *ws, int64_t ws_bytes, void *stream);

/* ---- a matrix update, orthogonalized ------------------------------------------------- */

/* out = v [n][ld] of `type`, d wide, with its singular values brought near 1:  X = v / |v|_F, then `steps` (1..64) times, on the shorter side,
 *   A = X X^T,   X = 3.4445 X + (-4.7750 A + 2.0315 A^2) X
 * (five steps take singular values from 0.002 of the norm on into 0.68 .. 1.21).  A matrix of zeros stays one; anything not finite makes every
 * result a NaN and sets status bit 0.  A, B = -4.7750 A + 2.0315 A^2 and X are rounded to 22 bits in every step, and to 2^-39 of X's norm (float32: together
 * at most four times as far off as sums in float32 are, mostly less; 16-bit types 10^-5 to 1.4 10^-3 of the result's norm), the result to its type.
 * A direction that v has nothing of, or no more than those roundings, is filled by them, and every step makes that 3.4445 times as large: up to 2^-22 3.4445^steps
 * of the result's norm, 10^-4 at five steps, 0.005 at eight, 0.06 at ten.  At twelve and more such a direction is as large as the others, whatever the
 * type, and no status bit tells: more than eight steps are for matrices whose every singular value is well above 2^-22 of the norm.
 * out may be v itself.  At most 2^20 by 2^15 numbers, either way round.  ws: at least dq_orthogonalize_bytes(type, n, d) bytes. */
int64_t dq_orthogonalize_bytes(int32_t type, int64_t n, int64_t d);
int32_t dq_orthogonalize(const void *v, int32_t type, int64_t n, int64_t d, int64_t ld, int32_t steps, void *out, int64_t ldo,
                         uint32_t *status, void *ws, int64_t ws_bytes, void *stream);

/* ---- message sizes ---------------------------------------------------------------- */

/* Bits on the wire of one message (host arithmetic, nothing is enqueued); negative = DQ_ERR_INVALID_ARG.
 * DQ_MSG_DENSE : Section 3.1, a vector of d coordinates at b bits each plus its 32-bit scale, 32 + b*d;
 *                b == 32 (not quantized): 32*d.  nnz is ignored.
 * DQ_MSG_FLAG  : Section 4.1, the model equals the snapshot and the master sends one flag bit: 1.
 * DQ_MSG_SPARSE: Section 4.2, the scale plus ceil(log2 d) position bits and b value bits per nonzero code,
 *                32 + nnz*(ceil(log2 d) + b); b == 32: nnz*(ceil(log2 d) + 32) (no scale).  0 <= nnz <= d.
 * b in [2,16] or 32. */
#define DQ_MSG_DENSE   0
#define DQ_MSG_FLAG    1
#define DQ_MSG_SPARSE  2
int64_t dq_message_bits(int32_t kind, int64_t d, int32_t b, int64_t nnz);

/* ---- inner loop ------------------------------------------------------------------ */

#define DQ_ALGO_ASYLPG  0   /* Alg. 1 */
#define DQ_ALGO_SPARSE  1   /* Alg. 2: sparsify before quantizing */
#define DQ_ALGO_ACC     2   /* Alg. 3: momentum */

/* Settings of a run (host struct). */
typedef struct dq_run_config {
    int32_t algo;        /* DQ_ALGO_* */
    int64_t M, B;        /* workers per round, mini-batch per worker */
    int32_t b_x, b;      /* bits of the model message and of the gradient message (32 = not quantized) */
    int64_t m;           /* rounds per epoch */
    uint64_t seed;
    int32_t tau;         /* emulated bounded delay (Assumption 3): 0 = every worker reads the current model;
                            tau > 0: the workers form tau+1 contiguous groups, worker w belongs to group
                            g = floor(w*(tau+1)/M) and reads the model message of round max(0, t-g) */
    int32_t each;        /* 0: one master update per round with the mean of the M gradients (dq_master_step,
                            scale 1/M); 1: one update per received gradient (dq_master_step_each); Alg. 3 then
                            averages m*M iterates for its snapshot */
} dq_run_config;

/* Device buffers of a run (host struct holding device pointers; all caller-owned).
 * x, x_snap, g_snap: float[d].  y, xsum: float[d], Alg. 3 only.  z_snap: float[n] margins at the
 * snapshot from dq_full_grad, nullable.  xq: ring of tau+1 model messages, slot s at
 * xq + s*xq_stride_words (each ceil(d*b_x/32) words, or d floats; 16-byte aligned slots);
 * delta_x: float[tau+1], one scale per slot; absmax_x: float[2] (scratch: the largest magnitude of the model after
 * the last two rounds, in alternating entries).  The message of round t lives in
 * slot t mod (tau+1).  packed: M rows of ld_words words; delta: float[M];
 * nnz: int32[m*M] nonzero codes per round and worker (written by Alg. 2 only), nullable.  ws: DQ_OP_VR_GRAD workspace
 * (scratch of the call: between the rounds of one call it also carries what one round leaves for the next, e.g. the
 * sparsified gradients that the master quantizes and, on CSR features, the decoded model minus the snapshot and the
 * next round's mini-batches -- row numbers drawn, extents, labels and entries read -- laid out by the round before).
 * wire (nullable, Alg. 2 with b in {2,4,8} only): M rows of ld_wire >= dq_sparse_stream_words(d, b) words.  When
 * given, every round really sends the sparse message of Section 4.2: the workers' packed codes are encoded into
 * `wire` (dq_sparse_encode), then the master's input is rebuilt from `wire` alone (dq_sparse_decode); wire_nnz:
 * int32[M], required with wire. */
typedef struct dq_run_state {
    float *x, *x_snap, *y, *xsum, *g_snap;
    const float *z_snap;
    uint32_t *xq;
    float *delta_x, *absmax_x;
    uint32_t *packed;
    int64_t ld_words;
    float *delta;
    int32_t *nnz;
    uint32_t *status;
    void *ws;
    int64_t ws_bytes;
    int64_t xq_stride_words;
    uint32_t *wire;
    int64_t ld_wire;
    int32_t *wire_nnz;
} dq_run_state;

/* Enqueues rounds t0 .. t0+rounds-1 of epoch `epoch` (0-based) of Alg. 1, 2 or 3: per round the
 * worker side (dq_worker_step with in-kernel sampling; the flag-bit case of Section 4.1 at the
 * first round of an epoch whose start equals the snapshot) and the master side (dq_master_step with
 * the mean over the M workers, or dq_master_step_each; model re-quantized for the next round).  Random streams use
 * iter = epoch*m + t.  eta, theta: step size and momentum weight of this epoch (theta unused by
 * Alg. 1/2; for Alg. 3 they are dq_acc_params(lr, epoch + 1, ...)).  The epoch prologue (dq_full_grad,
 * dq_acc_mix / copy) and epilogue stay with the caller.  Everything is validated before the first launch
 * (null or misaligned state pointers, a workspace smaller than dq_workspace_bytes(DQ_OP_VR_GRAD, prob, M, B),
 * which covers every worker group of a delayed run).  worker_events (host array, nullable): 2*rounds hipEvent_t handles created by the caller; for
 * round k the pair [2k], [2k+1] receives the start and the end time of the kernel of the worker step
 * that reads the feature rows (its first kernel; for CSR sparsifier and quantization may be launches of their own
 * after it; with tau > 0 the one of the first worker group): they are the start and stop events of that launch (hipExtLaunchKernel), so
 * hipEventElapsedTime over the pair is the kernel's own duration.  A flag-bit round leaves its pair
 * untouched; a pair of null handles makes that round's launch a plain one.  Pass null while `stream` is being
 * captured into a graph.
 * Rounds in few launches: on small dense problems, and on CSR features with mini-batches and a model that LDS has room for
 * (Alg. 1 and 3, eight rounds or more, with cached margins and a status word), a launch does many rounds, up to 512 on CSR
 * features, without worker_events.  On CSR features its blocks are one die's compute units, which have room for little else
 * meanwhile: a kernel of another stream that has blocks for that die ends only after them, up to 5 ms at 10 us a round.  Where
 * other streams' work leaves no die free for about as long as the rounds take, at most 2 to 4 ms, they are done with the
 * compute units that there are, 20 us each with 16 to 31 of a die's 32, 35 with 8.  Callers for whom either is too long make
 * calls of fewer than eight rounds.  Streams with a mask of compute units (hipExtStreamCreateWithCUMask) have launches for
 * each round; a graph takes what the stream of its capture does. */
int32_t dq_run_rounds(const dq_problem *prob /*host*/, const dq_run_config *cfg /*host*/, const dq_run_state *st /*host*/,
                      int64_t epoch, int64_t t0, int64_t rounds, float eta, float theta,
                      void **worker_events /*host*/, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* DQ_H_ */
