/* C ABI of the MI355X (gfx950) ELMO classifier-head library.
 *
 * The library implements the hot path of ELMO (arxiv 2510.11168): the label-chunked training
 * step of a linear extreme-classification head whose weights live only in BF16 or FP8-E4M3,
 * with the weight gradient fused into the SGD update (Algorithm 1 "Float8 XMC classifier",
 * Sections 4.1-4.3), stochastic rounding (Section 3, Eq. 1), optional Kahan compensation in
 * BF16 (Section 3; Appendix "Precision Recovery"), and the top-k scoring needed by P@k
 * (Appendix, definition of P@k).
 *
 * General rules
 *  - Every pointer named W, comp, workspace, X, indptr, indices, dX_out, loss_out, idx_out,
 *    score_out, src, dst is a DEVICE pointer owned by the caller; the library never allocates or
 *    frees device memory and never synchronises the device (exception: ELMO_VALIDATE, below).
 *  - Work is enqueued on `hip_stream` (a hipStream_t passed as void*; NULL = the null stream);
 *    results are valid once the stream has reached that point.  Calls on one head must not
 *    overlap in time: they share its workspace.
 *  - Return value: 0 success; -1 invalid argument; -2 unsupported format/flag; -3 HIP runtime
 *    error; -4 invalid label data found by a previous validated step.  elmo_last_error() gives
 *    the text for the calling thread.
 *  - All matrices are row-major and densely packed.
 */
#ifndef ELMO_HEAD_H
#define ELMO_HEAD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct elmo_head elmo_head_t; /* opaque, host-side */

/* Storage format of the classifier weights (Section 4.1 pure 16-bit; Section 4.3 8-bit).
 * ELMO_FP8_E4M3 is the OCP "FN" flavour: bias 7, largest finite value 448, no infinities. */
enum { ELMO_BF16 = 0, ELMO_FP8_E4M3 = 1, ELMO_FP32 = 2 /* optimiser moments of elmo_kahan_adamw, values of the row-wise operators */,
       ELMO_INT8 = 3 /* 8-bit rows of elmo_rms_norm */ };

/* ELMO_SR: the update rounds with stochastic rounding (Eq. 1), otherwise to nearest even.
 * ELMO_KAHAN: a BF16 compensation buffer carries the rounding error of every update into the
 *             next one (the recurrence of Section 3 with s = w, v = -lr*grad), for all labels or,
 *             with elmo_head_opts.kahan_rows, for the head labels only.
 * ELMO_VALIDATE: each step checks the label data on the device (ids inside [0, L), ascending
 *             within a row) and the NEXT call on the head reads that flag back (one blocking
 *             4-byte copy) and fails with -4 if it was raised. */
enum { ELMO_SR = 1u, ELMO_KAHAN = 2u, ELMO_VALIDATE = 4u };

typedef struct {
  uint32_t flags;         /* ELMO_SR | ELMO_KAHAN | ELMO_VALIDATE */
  int32_t max_B;          /* largest batch any step / top-k call will use (>= 1) */
  int64_t max_nnz;        /* largest number of positives in one batch (>= 1) */
  void* W;                /* [L, d] weights in weight_dtype, updated in place by every step */
  size_t W_bytes;
  void* comp;             /* [kahan_rows, d] BF16 compensation, required iff ELMO_KAHAN, start at zero */
  size_t comp_bytes;
  int64_t kahan_rows;     /* with ELMO_KAHAN: only the labels [0, kahan_rows) carry compensation, the rest
                             are updated as without the flag ("Kahan summation for head labels", appendix
                             "Precision Recovery for Sensitive Applications": number the labels by falling
                             frequency and the top-p% head is this prefix; memory 2 bytes x kahan_rows x d).
                             0 = every label.  Otherwise L or a multiple of 128.  Must be 0 without the flag. */
  float weight_decay;     /* L2 weight decay of the classifier (the "WD ... XMC" column of the paper's
                             hyper-parameter table; Algorithm 1 itself has none): the update uses
                             g + weight_decay * w in place of the gradient g, two more FP32 operations, each
                             rounded.  0 = none (the two operations are skipped).  In [0, 1]. */
  float dropout_p;        /* dropout on the classifier weights inside the products (appendix "Low-Memory
                             Dropout for Classifier": the weights are masked after they are loaded, before
                             the matrix product, so no masked copy of W exists).  Per step every weight
                             element is dropped with probability T/256, T = round(256 * dropout_p), the
                             same mask for all samples of the batch; the logits and the input gradient use
                             the masked weights scaled by 256/(256-T), and the weight gradient is that of
                             the masked model (zero at dropped elements, scaled elsewhere).  The mask is
                             byte e % 16 >= T of Philox4x32-10 with key = seed of the step and counter =
                             (e / 16, step | 2^63), e = label * d + column; steps must stay below 2^63.
                             elmo_head_topk never drops.  0 = none.  In [0, 255/256]. */
  void* workspace;        /* scratch; contents need not survive between calls */
  size_t workspace_bytes;
} elmo_head_opts;

/* Bytes of the three buffers a head needs.  workspace = one chunk's logit-gradient buffer
 * (chunk x round_up(max_B, 64) BF16 values, the paper's per-chunk logits buffer of Section 4.4)
 * plus O(max_B * d) staging for the inputs and the input-gradient partial sums, plus the
 * per-batch label index.  Any of the three output pointers may be NULL. */
int elmo_head_sizes(int64_t L, int32_t d, int weight_dtype, int64_t chunk, int32_t max_B,
                    int64_t max_nnz, uint32_t flags, int64_t kahan_rows, size_t* W_bytes,
                    size_t* comp_bytes, size_t* workspace_bytes);

/* Bytes of the logit / logit-gradient buffer for `batch` samples and `labels` labels held in
 * 16 bits, batch * labels * 2 -- the quantity Section 4.4 divides by the number of chunks. */
size_t elmo_logit_buffer_bytes(int64_t batch, int64_t labels);

/* Create a head over caller-owned buffers.  Requirements: L >= 1; d a positive multiple of 128, at most 2^20;
 * chunk >= 1 (the labels processed per pass, Section 4.2 "chunking"; it need not divide L, the last
 * chunk is short.  The kernels work on whole 128-label tiles, so a pass takes round_up(chunk, 128)
 * labels, or more where the workspace holds their gradients anyway; the updated weights do not
 * depend on the chunk size at all and the input gradient only through the order of its FP32 sums, so
 * the rounding shows in the workspace size only); buffers at
 * least as large as elmo_head_sizes says and 256-byte aligned.  Launches nothing.  *out receives the
 * handle.  Heads may be created and stepped from several host threads (one head per thread at a
 * time); the library's one-time set-up is guarded. */
int elmo_head_create(int64_t L, int32_t d, int weight_dtype, int64_t chunk,
                     const elmo_head_opts* opts, elmo_head_t** out);

/* One training step of the head (Algorithm 1, XMC_update):
 *   for each chunk c of labels:  Z = Xq W_c^T ; G = sigmoid(Z) - Y_c ; dX += G W_c (old W_c);
 *                                W_c <- Q(W_c - lr * G^T X)   (fused, FP32 arithmetic)
 * X      [B, d] BF16 inputs (the encoder's output).  With FP8 weights the logits use X rounded
 *        to E4M3 (nearest even); the weight gradient always uses the BF16 X.  With BF16 weights X
 *        is 16-byte aligned (the logits product reads it as it is, 16 bytes at a time); with FP8
 *        weights it may begin at any BF16 element.
 * indptr [B+1], indices [nnz] int32: CSR of the positive label ids of each sample; within a row
 *        ids are distinct, ascending, in [0, L); nnz == indptr[B] <= max_nnz.
 * lr     learning rate; the gradient is summed over the batch (no 1/B).
 * seed, step: select the stochastic-rounding stream (Philox4x32-10, key = seed, counter =
 *        (flat element index / 8, step); element l*d+j uses 16-bit field (l*d+j) % 8).  The
 *        updated weights depend on (seed, step) only -- not on chunk or launch geometry.
 * dX_out [B, d] BF16 input gradient, or NULL.  loss_out: one float, the summed BCE loss
 *        sum(softplus(z) - y z) over the batch and all labels, or NULL.
 * The call only enqueues kernels on hip_stream (no allocation, no memset node, no host
 * synchronisation unless ELMO_VALIDATE is set), so after one ordinary call it can be captured
 * into a HIP graph; lr, seed and step are then part of the captured launches. */
int elmo_head_step(elmo_head_t* h, const void* X, int32_t B, const int32_t* indptr,
                   const int32_t* indices, int64_t nnz, float lr, uint64_t seed, uint64_t step,
                   void* dX_out, float* loss_out, void* hip_stream);

/* Top-k scoring (the top_k of the P@k definition): for each of the B rows of X the k labels with
 * the largest logit over all L labels, ordered by (logit descending, label id ascending).
 * X is aligned as for elmo_head_step.
 * idx_out [B, k] int32, score_out [B, k] float (either may be NULL).  1 <= k <= L.
 * Up to k = 128 the labels are swept once; larger k is produced in pages of 128 entries, one more
 * sweep per page (each page admits only what ranks strictly after the last entry of the page
 * before it), exact for any k. */
int elmo_head_topk(elmo_head_t* h, const void* X, int32_t B, int32_t k, int32_t* idx_out,
                   float* score_out, void* hip_stream);

/* Top-k scoring for callers that cannot allocate device memory or keep a head: code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same result as
 * elmo_head_topk on a head over the same weights (same kernels), but the call takes the weights
 * directly and needs no workspace: its scratch (staged E4M3 copy of X, thresholds, candidate lists)
 * is a device array of 18 MiB inside the library, one copy per GPU the library runs on, held until
 * the process ends.  The call allocates and frees nothing and launches only kernels (no memset
 * node).  Limits, rejected with -1: B <= 128 queries, d a multiple of 128 up to 4096, 1 <= k <= L.
 * W [L, d] in weight_dtype (ELMO_BF16 or ELMO_FP8_E4M3), X [B, d] BF16, both device pointers,
 * 16-byte aligned; idx_out [B, k] int32, score_out [B, k] float (either may be NULL).
 * All calls on one GPU share that GPU's array and nothing of it survives a call: calls that overlap
 * in time on one GPU (two streams, two host threads) race.  The first call on a device looks the
 * array's address up (hipGetSymbolAddress); make that call outside any stream capture. */
int elmo_topk_static(const void* W, int64_t L, int32_t d, int weight_dtype, const void* X, int32_t B,
                     int32_t k, int32_t* idx_out, float* score_out, void* hip_stream);

/* Precision at k (evaluation section, P@k(y, y^) = (1/k) sum over l in top_k(y^) of y_l), as exact
 * integer numerators: hits_out[j-1] = number of (row, label) pairs with the label among the row's
 * first j entries of idx and among the row's positives, summed over the B rows, j = 1..k; then
 * P@j = hits_out[j-1] / (j * B).  idx [B, k] int32 as written by elmo_head_topk (best first);
 * indptr / indices: the CSR positives of the same B rows (ids ascending within a row); hits_out
 * [k] int64.  All device pointers; 1 <= k <= 2^20 and B * k < 2^31.  Needs no head. */
int elmo_precision_hits(const int32_t* idx, int32_t B, int32_t k, const int32_t* indptr,
                        const int32_t* indices, int64_t* hits_out, void* hip_stream);

int elmo_head_destroy(elmo_head_t* h);

/* Measurement hooks.  elmo_head_profile(h, 1) makes every later step / top-k call record a HIP
 * event on its stream at each boundary between kernel classes; elmo_head_profile(h, 0) stops.
 * elmo_head_profile_read waits for the last recorded event, then returns per class the summed
 * event-to-event time in milliseconds and the number of spans, and clears the record.  Classes:
 * 0 step set-up, 1 logits + epilogue, 2 input gradient, 3 fused update, 4 finalise, 5 top-k.
 * ms and launches are HOST arrays of 6 entries. */
int elmo_head_profile(elmo_head_t* h, int enable);
int elmo_head_profile_read(elmo_head_t* h, double ms[6], int64_t launches[6]);

/* Text of the last error on the calling thread; never NULL. */
const char* elmo_last_error(void);

/* Test hooks for the bit-exactness clause of the parity contract.
 * elmo_quantize: dst[i] = Q(src[i]) for i in [0, n): dtype ELMO_BF16 writes uint16, ELMO_FP8_E4M3
 * writes uint8; mode 0 = round to nearest even, mode 1 = stochastic rounding with the field of
 * flat element index first_elem + i (same stream as elmo_head_step).  src: device FP32. */
int elmo_quantize(const float* src, int64_t n, int dtype, int mode, uint64_t seed, uint64_t step,
                  uint64_t first_elem, void* dst, void* hip_stream);

/* Simulated low-precision formats (the bit-width study of Section 4.3, "simulating floating-point
 * numbers with a specific number of mantissa and exponent bits"): dst[i] = the FP32 value of src[i]
 * rounded to a format with exp_bits exponent and man_bits mantissa bits, mode and rounding fields as
 * in elmo_quantize.  The format follows the IEEE pattern (bias 2^(E-1)-1, top exponent code reserved,
 * gradual underflow): (8,7) is BF16, (5,10) FP16, (5,2) E5M2; finite overflow and infinities clip to
 * the largest finite value, NaN passes through.  2 <= exp_bits <= 8, 1 <= man_bits <= 22 (else -2).
 * src, dst: device FP32, n entries each (may be the same buffer). */
int elmo_quantize_em(const float* src, int64_t n, int exp_bits, int man_bits, int mode, uint64_t seed,
                     uint64_t step, uint64_t first_elem, float* dst, void* hip_stream);

/* AdamW with Kahan-compensated BF16 parameters, in place (Section 4.1: the encoder's parameters
 * are kept in BF16 and their optimiser step uses Kahan summation so that updates below half a
 * grid spacing are not cancelled).  Textbook AdamW (decoupled weight decay, bias-corrected
 * moments) in FP32 arithmetic, every operation rounded once:
 *   m' = b1 m + o1 g;   v' = b2 v + (o2 g) g;   r = (m'/bc1) / (sqrt(v'/bc2) + eps);
 *   r += weight_decay * p (skipped when 0);   u = lr r;
 *   y = -u - c;   s = p + y;   p' = RNE_BF16(s);   c' = RNE_BF16((p' - p) - y)
 * with b_i = (float)beta_i, o_i = (float)(1 - beta_i), bc_i = (float)(1 - beta_i^t) formed in double.
 * param, comp, grad: device BF16 [n] (comp starts at zero); m, v: device moments [n] in
 * state_dtype = ELMO_BF16 (stored round-to-nearest-even) or ELMO_FP32, starting at zero.
 * t >= 1 counts the steps.  All buffers 16-byte aligned, caller-owned, updated in place (grad is
 * only read).  n = 0 is a no-op.  Errors: -1 bad argument, -2 unsupported state_dtype, -3 HIP. */
int elmo_kahan_adamw(void* param, void* comp, void* m, void* v, const void* grad, int64_t n, int state_dtype,
                     float lr, double beta1, double beta2, float eps, float weight_decay, int64_t t,
                     void* hip_stream);

/* Host-side view of the dropout mask of elmo_head_opts.dropout_p: bit i of the result is 1 iff
 * weight element 16 * block + i is kept at (seed, step) for the threshold T = threshold (0..255). */
uint32_t elmo_dropout_keep16(uint64_t seed, uint64_t step, uint64_t block, uint32_t threshold);

/* Host-side Philox4x32-10 (Salmon et al., SC'11) as used for the rounding fields. */
void elmo_philox4x32_10(const uint32_t ctr[4], const uint32_t key[2], uint32_t out[4]);

/* ---------------------------------------------------------------------------------------------
 * The output end of a language model: norm, 8-bit integer product, sampling, distillation.
 *
 * Rules of these calls, beside the general ones:
 *  - Matrices are row-major with elements of a row next to each other; *_stride is the number of
 *    elements from one row to the next, at least the row's length (any value for a single row).
 *    Rows need no alignment beyond their elements'.  Nothing between rows is written.
 *  - Values are ELMO_BF16 or ELMO_FP32 as the dtype argument says; sums are FP32 or wider, every
 *    output is rounded once, to nearest even (overflow to infinity, NaN kept); E4M3 rows by way of FP32.
 *  - All pointers are device pointers owned by the caller.  A call with no rows is a no-op.  Workspaces are scratch of the call: two calls that may
 *    overlap in time (streams, captured graphs) need one each.
 *  - Only kernels are enqueued, so after one ordinary call of its kind a call can be captured into
 *    a HIP graph.  The same call gives the same bits every time.
 *  - A launch takes fewer than 2^32 work-items: fewer than 2^22 rows of elmo_sample and 2^23 of elmo_distill; of
 *    elmo_rms_norm fewer than 2^24, of more than 8192 columns 2^22, of at most 1024 columns at most 2^26 - 4.  More are refused.
 * --------------------------------------------------------------------------------------------- */

/* Root-mean-square norm of rows of d elements (1 <= d <= 16384), behind a residual's addition:
 *   h = x + residual (x alone if residual is NULL),  y = weight * h / sqrt(mean(h^2) + eps)
 * weight [d] (NULL = ones) has a dtype of its own.  sum_out (NULL = not wanted; needs a residual)
 * receives h rounded to dtype, y is formed from the unrounded h.  y_dtype: ELMO_BF16 or ELMO_FP32, or 8 bits
 * with a scale per row in scale_out [rows]: with p = weight * h and m = max |p| of the row
 *   ELMO_INT8:      y = round(127 p / m),       scale = m / (127 sqrt(mean(h^2) + eps))
 *   ELMO_FP8_E4M3:  y = round_E4M3(round_FP32(448 p / m)),  scale = m / (448 sqrt(mean(h^2) + eps))
 * so that y * scale is the norm; the quotient is p * (127 * (1 / m)), p exact and three FP64 roundings.  The conversion to E4M3 takes FP32 values: an
 * element is off by at most half a step and 2^-24 of its value (one in some million has its other neighbour by that).  A row of zeros gives zeros and scale 0; a row that holds an infinity or NaN, or whose squares
 * add up to more than FP32 holds, gives zeros and scale NaN (BF16 and FP32 rows of such squares are normalised as any others).  sum_out may be x or residual, and y the other of the two, where address, stride and dtype are the same. */
int elmo_rms_norm(const void* x, int64_t x_stride, int dtype, int64_t rows, int64_t d, const void* residual,
                  int64_t residual_stride, const void* weight, int weight_dtype, float eps, void* sum_out,
                  int64_t sum_stride, void* y, int64_t y_stride, int y_dtype, float* scale_out, void* hip_stream);

/* Its backward pass.  h: what was normalised (sum_out, or x without a residual).  With R = 1 / sqrt(mean(h^2) + eps), g = weight * dy:
 *   dh = R (g - h R^2 mean(g h)) + dsum      (the gradient of x and of the residual alike)
 *   dweight[j] = sum over rows of R dy h     (FP32 [d], overwritten; NULL = not wanted; zeros for no rows)
 * h is taken as it is stored: behind a BF16 sum_out the gradient is that at the rounded sum.  R itself has to lie within FP32.  dsum (NULL = none) is the gradient that reaches sum_out from elsewhere.  dh may be dy, h or dsum where address and stride are
 * the same.  dweight needs a workspace of elmo_rms_norm_backward_bytes(rows, d) bytes, 4-byte aligned. */
size_t elmo_rms_norm_backward_bytes(int64_t rows, int64_t d);
int elmo_rms_norm_backward(const void* dy, int64_t dy_stride, const void* h, int64_t h_stride, int dtype, int64_t rows,
                           int64_t d, const void* weight, int weight_dtype, float eps, const void* dsum,
                           int64_t dsum_stride, void* dh, int64_t dh_stride, float* dweight, void* workspace,
                           size_t workspace_bytes, void* hip_stream);

/* 8-bit integer product with a scale for each row of either operand (token and output channel):
 *   out[m, n] = (sum_k a[m, k] b[n, k]) a_scale[m] b_scale[n] + bias[n]
 * a [M, K] and b [N, K] int8 (all 256 values), scales and bias FP32 (bias NULL = none), out [M, N] in out_dtype.  The sum is exact
 * (0 <= K <= 131071; of no products it is 0) and rounded to FP32, as are the two products and the bias's addition.  M and N up to 2^30, fewer than 2^23 tiles of 256 x 256 outputs.
 * elmo_int8_matmul_tile: how these sizes are worked on, in tiles of 64, 128 or 256, or 0 for the kernel of few tokens that streams the weights (-1: refused). */
int elmo_int8_matmul(const int8_t* a, int64_t a_stride, const float* a_scale, const int8_t* b, int64_t b_stride,
                     const float* b_scale, const float* bias, int64_t M, int64_t N, int64_t K, void* out,
                     int64_t out_stride, int out_dtype, void* hip_stream);
int elmo_int8_matmul_tile(int64_t M, int64_t N, int64_t K);

/* One token for each row of V logits (1 <= V < 2^31), from a given random number u[row] in [0, 1).  Tokens are ordered by (logit
 * falling, index rising) and weigh exp((z - max z) / temperature).  Kept are the first top_k of them, of those the shortest beginning
 * that has at least top_p of their weight, and of those the ones of weight >= min_p (relative to the largest).  The token is the
 * first one in order of index at which the kept weight so far exceeds u times the kept weight.
 * temperature, top_k, top_p, min_p: one value a row, or NULL (1, off, off, off).  temperature <= 0 or NaN: the largest logit, lowest
 * index.  top_k < 1, top_p >= 1 or NaN, min_p <= 0 or NaN: off; top_p <= 0 keeps one token, min_p >= 1 those equal to the largest.  u is
 * clamped to [0, 1), NaN counts as 0.  Logits of -infinity and NaN are never drawn; beside logits of +infinity nothing else is.
 * Weights are whole multiples of 2^-F of the largest, F = min(50, 62 - ceil(log2 V)), rounded to nearest from FP64 values that are right to 2^-51 (a
 * token below half a multiple is never drawn), and their sums are exact: the token does not depend on how a row is split.
 * idx_out [rows]: the token, -1 where a row has none; prob_out [rows] (NULL = not wanted): its share of the kept weight, from
 * its FP64 weight, 0 where there is none.  workspace: elmo_sample_bytes(rows, V) bytes, 256-byte aligned (NULL if that is 0, and with top_k). */
size_t elmo_sample_bytes(int64_t rows, int64_t V);
int elmo_sample(const void* logits, int64_t logits_stride, int dtype, int64_t rows, int64_t V, const float* u,
                const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p, int32_t* idx_out,
                float* prob_out, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Distillation from a teacher's top logits, loss and gradient in one call.  teacher_idx, teacher_logits [rows, K], dense: the
 * teacher's tokens and their logits, 1 <= K <= 1024; entries whose index is outside [0, V) do not count, an index that appears
 * twice counts twice.  With q = softmax(teacher / T) over the row's entries, p = softmax(logits / T) over all V (1 <= V < 2^31),
 * T = temperature in [1e-6, 1e6], v = row_weight[row] (NULL = 1):
 *   loss_out[row] = v T^2 sum_j q_j log(q_j / p_j)       grad_out = d loss / d logits = v T (p - q)
 * grad_out (NULL = not wanted) has the logits' dtype and may be the logits themselves where the strides are the same.  Rows of weight
 * 0 and rows without a teacher entry above -infinity give loss 0 and a gradient of zeros whatever the logits hold.  A logit of -infinity has p = 0 (loss
 * +infinity if q > 0 there; so for a row of nothing else); NaN and +infinity make the row's loss and gradient NaN.
 * workspace: elmo_distill_bytes(rows, V) bytes, 256-byte aligned (NULL if that is 0). */
size_t elmo_distill_bytes(int64_t rows, int64_t V);
int elmo_distill(const void* logits, int64_t logits_stride, int dtype, int64_t rows, int64_t V,
                 const int32_t* teacher_idx, const void* teacher_logits, int teacher_dtype, int64_t K, float temperature,
                 const float* row_weight, float* loss_out, void* grad_out, int64_t grad_stride, void* workspace,
                 size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ELMO_HEAD_H */
