/*
 * zo_ops.h -- operators that stand next to the optimizer step of zo_adam.h, on
 * one MI355X (gfx950): matrices in microscaled 4-bit floating point and in 8-bit
 * integers (quantised from the binary32 shard or from activations, read back,
 * multiplied), the root-mean-square norm before such products, a teacher's top
 * logits, the distillation loss with the gradient of the student's logits, and
 * the log probabilities of tokens with theirs.
 *
 * Conventions
 *   - No handle and no state: every call takes its buffers.  Device pointers
 *     are caller-owned; the calls allocate nothing and keep nothing.
 *   - Every call validates its arguments on the host before enqueueing
 *     anything and returns a negative status of zo_adam.h if it refuses;
 *     zo_ops_last_hip_error() is the text behind the calling thread's last
 *     ZO_EHIP.
 *   - Calls are asynchronous on `stream`, may run from any host thread, and
 *     may be recorded into a HIP graph (kernels only: no memset, no copy).
 *   - Element types are ZO_DTYPE_F32, ZO_DTYPE_F16 and ZO_DTYPE_BF16.  Matrices
 *     of these types are row-major with a row stride `ld` in elements
 *     (ld >= columns) and need no alignment beyond their element's.
 *   - A launch holds fewer than 2^32 threads.  A call on matrices that needs more
 *     (none below 2^23 tiles of 64 x 128 elements or results does) is ZO_EINVAL;
 *     logits go into as many launches as their rows take, up to 2^31 - 1 of them.
 *   - Buffers that a call writes may not overlap any other of its buffers,
 *     except where the call says so.
 *   - Sums, softmax statistics and products accumulate in binary32; a result
 *     is rounded once, to nearest even, to the type of its buffer.
 *   - Results depend on the inputs alone: no atomics decide an order of sums.
 *   - Calls that may run at once need workspaces of their own.
 */
#ifndef ZO_OPS_H
#define ZO_OPS_H

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#include "zo_adam.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * A matrix in microscaled 4-bit floating point ("mx4"): elements E2M1 (0, 0.5,
 * 1, 1.5, 2, 3, 4, 6 and their negatives), 32 consecutive elements of a row
 * sharing a scale 2^(b - 127) (E8M0: the byte b; b = 255: all 32 read as NaN).
 * The row is the axis that products reduce over.
 *
 * Layout: the order in which the matrix instruction takes its operands.  With
 * KT = ceil(cols / 128), element (r, c), k = c % 128:
 *   codes   nibble c % 2 (low first) of byte
 *           ((r / 16 * KT + c / 128) * 64 + k / 32 * 16 + r % 16) * 16 + k % 32 / 2
 *   scales  byte ((r / 64 * KT + c / 128) * 64 + k / 32 * 16 + r % 16) * 4 + r % 64 / 16
 * for ceil(rows / 64) * 64 rows of KT * 128 columns.  Columns beyond `cols`
 * hold codes 0 and scale bytes 0; rows beyond `rows` hold anything and reach
 * no result.
 *   codes   device, zo_mx4_code_bytes(rows, cols) bytes, 16-byte aligned
 *   scales  device, zo_mx4_scale_bytes(rows, cols) bytes, 4-byte aligned
 * rows, cols in [0, 2^30].
 */
typedef struct zo_mx4 {
    void *codes, *scales;
    int64_t rows, cols;
} zo_mx4;

/* Buffer sizes of a rows x cols mx4 matrix, or a negative status (host only). */
int64_t zo_mx4_code_bytes(int64_t rows, int64_t cols);
int64_t zo_mx4_scale_bytes(int64_t rows, int64_t cols);

/*
 * zo_mx4_quantize -- x [rows, cols] of element type dtype into
 *   q   (NULL or rows x cols) along x's rows, and / or
 *   qt  (NULL or cols x rows) along x's columns (the transpose),
 * reading x once.  A block of 32 with largest magnitude a > 0 gets
 *   b = max(0, floor(log2 a) - 2 + 127), codes = RNE_E2M1(x / 2^(b-127)),
 * magnitudes above 6 becoming 6 (a is below 8 scales); a block of zeros b = 0.
 * A block with a NaN or an infinity gets b = 255 and codes 0.
 * Both NULL is ZO_EINVAL.
 */
int zo_mx4_quantize(const void *x, int32_t dtype, int64_t rows, int64_t cols, int64_t ld,
                    const zo_mx4 *q, const zo_mx4 *qt, hipStream_t stream);

/* zo_mx4_dequantize -- the values of q into out [q->rows, q->cols]: exact for
 * binary32 and bfloat16, rounded to nearest even for binary16. */
int zo_mx4_dequantize(const zo_mx4 *q, void *out, int32_t dtype, int64_t ld,
                      hipStream_t stream);

/*
 * zo_mx4_product -- out[m, n] = sum over k of a(m, k) b(n, k): both operands'
 * rows are the reduced axis, a->cols = b->cols.  out is [a->rows, b->rows].
 * With x, w, dy the activations [t, k], weights [n, k] and output gradients
 * [t, n] of a layer y = x w^T, quantised along the reduced axes:
 *   y = product(q(x), q(w)), dx = product(q(dy), qt(w)), dw = product(qt(dy), qt(x)).
 */
int zo_mx4_product(const zo_mx4 *a, const zo_mx4 *b, void *out, int32_t dtype, int64_t ld,
                   hipStream_t stream);

/*
 * zo_mx4_linear -- zo_mx4_quantize(x) along its rows and
 * zo_mx4_product(x, w) in one call (the form of a decode step: with few rows,
 * one kernel).  x is [xq->rows, xq->cols], out [xq->rows, w->rows], xq
 * workspace whose contents afterwards are unspecified.
 */
int zo_mx4_linear(const void *x, int32_t dtype, int64_t ldx, const zo_mx4 *w,
                  const zo_mx4 *xq, void *out, int32_t out_dtype, int64_t ldo,
                  hipStream_t stream);

/*
 * zo_top_logits -- of every row of z [rows, vocab], its `top` largest logits
 * in descending order, the columns they stand in, and the row's log-sum-exp:
 *   values   float [rows, top], columns  int32 [rows, top],
 *   lse      NULL or float [rows]: log sum over columns of exp(z / tau).
 * Equal values are ordered by column, the lowest first; -0 equals +0; NaN
 * orders above +infinity.  A row of only -infinity has lse = -infinity, one
 * with a NaN has lse = NaN.  top in [1, min(vocab, 1024)], vocab < 2^31,
 * tau > 0 and finite.
 */
int zo_top_logits(const void *z, int32_t dtype, int64_t rows, int64_t vocab, int64_t ld,
                  int32_t top, float tau, float *values, int32_t *columns, float *lse,
                  hipStream_t stream);

/*
 * Arguments of zo_distill_loss (host struct, read during the call).
 *   z            student logits [rows, vocab], row stride ldz.
 *   values,      the teacher's top logits and their columns, [rows, top];
 *   columns      a column outside [0, vocab) marks an unused slot, and of
 *                slots with the same column the first counts.
 *   teacher_lse  NULL, or float [rows]: log-sum-exp of the teacher's
 *                logits / tau over the whole vocabulary.
 *   labels       NULL, or int32 [rows]; outside [0, vocab): no label.
 *   row_weight   NULL (all 1), or float [rows]: w_t, the gradient that comes
 *                from above.  A row of weight 0 is not read: loss 0, dz 0.
 *   tau, kd_weight, ce_weight   finite, tau > 0.
 *   loss         NULL, or float [rows].
 *   dz           NULL, or [rows, vocab] of z's type, row stride lddz; may be z
 *                itself (with lddz = ldz).
 * top in [1, 1024], vocab in [1, 2^18].
 */
typedef struct zo_distill {
    const void *z;
    int32_t dtype;
    int64_t rows, vocab, ldz;
    int32_t top;
    const float *values;
    const int32_t *columns;
    const float *teacher_lse;
    const int32_t *labels;
    const float *row_weight;
    float tau, kd_weight, ce_weight;
    float *loss;
    void *dz;
    int64_t lddz;
} zo_distill;

/*
 * zo_distill_loss -- per row, with q = softmax(z / tau), S the columns of the
 * used slots, u the teacher's logits there:
 *   without teacher_lse  p = softmax of u / tau over S,
 *     KL = sum over S of p log(p / q);
 *   with teacher_lse L   p = exp(u / tau - L), and what p leaves of 1 is one
 *     more outcome: p_r = max(0, 1 - sum p), q_r = sum of q outside S,
 *     KL = sum over S of p log(p / q) + p_r log(p_r / q_r);
 *   loss = w (kd_weight tau^2 KL + ce_weight (lse(z) - z[label])),
 *   dz = w (kd_weight tau d + ce_weight (softmax(z) - onehot(label))),
 *     d = q - p on S; outside S d = q, with L q - p_r (q / q_r).
 * A part whose weight is 0 is left out.  Outcomes with p = 0 add 0 to KL; one
 * with p > 0 that the student excludes (logits of -infinity, and those whose
 * distance from the row's largest, over tau, passes binary32) makes the loss
 * +infinity and leaves the gradient finite, and so does an excluded label.
 * p_r below 2^-16 counts as 0 where the student excludes everything outside S or
 * its largest logit there has less than 2^-32768 of the row's largest one's
 * probability (masks of -1e9 or of a type's lowest value): it is no more than
 * the rounding of L.  A student row of only -infinity has q = 0.  Without L, a
 * row whose used slots hold no teacher's logit above -infinity has no KL part.
 */
int zo_distill_loss(const zo_distill *args, hipStream_t stream);

/*
 * A matrix in 8-bit integers ("i8"): element (r, c) is scale(r) times its code,
 * an integer in [-127, 127].  The row is the axis that products reduce over: a
 * token's activations, a channel's weights.
 *
 * Layout: row r's codes are bytes r * W .. r * W + cols - 1 with
 * W = ceil(cols / 128) * 128; the row's other bytes are 0.
 *   codes   device, zo_i8_code_bytes(rows, cols) bytes, 16-byte aligned
 *   scales  device, float [rows]; NaN: the row reads as NaN
 * rows, cols in [0, 2^30].  Without columns the scales are neither written nor read.
 */
typedef struct zo_i8 {
    void *codes;
    float *scales;
    int64_t rows, cols;
} zo_i8;

/* Bytes of a rows x cols i8 matrix's codes, and of the workspace of zo_i8_quantize
 * along the columns of a rows x cols matrix; or a negative status (host only). */
int64_t zo_i8_code_bytes(int64_t rows, int64_t cols);
int64_t zo_i8_work_bytes(int64_t rows, int64_t cols);

/*
 * zo_i8_quantize -- x [rows, cols] of element type dtype into
 *   q   (NULL or rows x cols) along x's rows, and / or
 *   qt  (NULL or cols x rows) along x's columns (the transpose).
 * A row (of qt: a column) with largest magnitude a gets the scale s = a / 127,
 * rounded to binary32, and the codes x / s, the exact quotients rounded to
 * nearest even and clamped to +-127 (an s of 0: zeros).  One with a NaN or an
 * infinity gets the scale NaN and codes 0.
 *   work    with qt: device, zo_i8_work_bytes(rows, cols) bytes, 4-byte aligned,
 *           whose contents afterwards are unspecified; otherwise not touched.
 * Both NULL is ZO_EINVAL.
 */
int zo_i8_quantize(const void *x, int32_t dtype, int64_t rows, int64_t cols, int64_t ld,
                   const zo_i8 *q, const zo_i8 *qt, void *work, hipStream_t stream);

/* zo_i8_dequantize -- the values of q (scale times code in binary32) into out
 * [q->rows, q->cols].  127 times the scale of a row with binary32's largest number, which
 * is rounded up, passes binary32: it is read back as infinity. */
int zo_i8_dequantize(const zo_i8 *q, void *out, int32_t dtype, int64_t ld, hipStream_t stream);

/*
 * zo_i8_product -- out[m, n] = (sum over k of a's code(m, k) b's code(n, k)) times
 * a's scale(m), times b's scale(n): the sum exact, the products in binary32, in this
 * order.  a->cols = b->cols <= 131072 (so that 32 bits hold the sum); out is
 * [a->rows, b->rows].  The products of a layer's forward and backward are those of
 * zo_mx4_product.
 */
int zo_i8_product(const zo_i8 *a, const zo_i8 *b, void *out, int32_t dtype, int64_t ld,
                  hipStream_t stream);

/*
 * zo_i8_linear -- zo_i8_quantize(x) along its rows and zo_i8_product(x, w) in one call
 * (the form of a decode step: with few rows, one kernel).  x is [xq->rows, xq->cols],
 * out [xq->rows, w->rows], xq workspace whose contents afterwards are unspecified.
 */
int zo_i8_linear(const void *x, int32_t dtype, int64_t ldx, const zo_i8 *w, const zo_i8 *xq,
                 void *out, int32_t out_dtype, int64_t ldo, hipStream_t stream);

/*
 * Arguments of zo_rms_norm (host struct, read during the call).
 *   x          [rows, cols] of element type dtype, row stride ldx.
 *   residual   NULL, or of x's shape and type, row stride ldr.
 *   weight     [cols], of element type weight_dtype: dtype or ZO_DTYPE_F32.
 *   h          NULL, or of x's shape and type, row stride ldh: x + residual.  May be
 *              x or residual itself (with its stride).
 *   out        NULL, or of x's shape and type, row stride ldo; may be x or residual
 *              itself too, where h is not the same.
 *   q          NULL, or rows x cols.
 *   rstd       NULL, or float [rows].
 *   eps        at least 2^-126, finite.
 * rows < 2^31, cols in [1, 32768].  Nothing to write is ZO_EINVAL.
 */
typedef struct zo_norm {
    const void *x;
    int32_t dtype;
    int64_t rows, cols, ldx;
    const void *residual;
    int64_t ldr;
    const void *weight;
    int32_t weight_dtype;
    float eps;
    void *h;
    int64_t ldh;
    void *out;
    int64_t ldo;
    const zo_i8 *q;
    float *rstd;
} zo_norm;

/*
 * zo_rms_norm -- the residual's addition and the root-mean-square norm.  Per row:
 *   h = x + residual (in binary32, rounded to the type of x; without a residual x),
 *   rstd = 1 / sqrt(mean of h^2 + eps), out = h rstd weight,
 *   q = the 8-bit row of h weight (each product rounded to binary32, codes and s as
 *       zo_i8_quantize makes them) with the scale s rstd: the codes do not depend on
 *       rstd, which cancels.
 * Sums of squares that binary32 does not hold are formed from scaled values.  A row of
 * zeros gives zeros; one with a NaN has rstd NaN, one with an infinity rstd 0.
 */
int zo_rms_norm(const zo_norm *args, hipStream_t stream);

/*
 * Arguments of zo_rms_norm_grad (host struct, read during the call).
 *   dy         [rows, cols] of element type dtype, row stride lddy: the gradient of out.
 *   h, weight, rstd   as zo_rms_norm took and left them; h of dtype.
 *   dh         NULL, or of dy's shape and type, row stride lddh: what reaches h past
 *              the norm (the residual stream's gradient).
 *   dx         NULL, or of dy's shape and type, row stride lddx: the gradient of x and
 *              of the residual.  May be dy, dh or h itself (with its stride).
 *   dw         NULL, or float [cols]: the gradient of the weight.
 *   work       with dw: device, zo_rms_norm_work_bytes(rows, cols) bytes, 4-byte
 *              aligned, whose contents afterwards are unspecified.
 * rows < 2^31, cols in [1, 32768].  Nothing to write is ZO_EINVAL.
 */
typedef struct zo_norm_back {
    const void *dy;
    int32_t dtype;
    int64_t rows, cols, lddy;
    const void *h;
    int64_t ldh;
    const void *weight;
    int32_t weight_dtype;
    const float *rstd;
    const void *dh;
    int64_t lddh;
    void *dx;
    int64_t lddx;
    float *dw;
    void *work;
} zo_norm_back;

/* Bytes of that workspace, or a negative status (host only). */
int64_t zo_rms_norm_work_bytes(int64_t rows, int64_t cols);

/*
 * zo_rms_norm_grad -- with n = h rstd and g = dy weight, per row
 *   dx = dh + rstd (g - n mean(g n)), and dw = sum over rows of dy n
 * (of no rows: zeros).
 */
int zo_rms_norm_grad(const zo_norm_back *args, hipStream_t stream);

/*
 * Arguments of zo_token_logprobs (host struct, read during the call).
 *   z          logits [rows, vocab] of element type dtype, row stride ldz.
 *   tokens     NULL, or int32 [rows]; outside [0, vocab): no token.
 *   tau        finite, at least 2^-126: probabilities are softmax(z / tau).
 *   logp       float [rows], with tokens: the log probability of the row's token, 0
 *              where there is none.
 *   stats      NULL, or float [rows, 3]: the largest logit m, the logarithm of
 *              S = sum of exp((z - m) / tau), and the entropy.
 *   top        0, or how many of the most likely alternatives:
 *   values     float [rows, top], their log probabilities in descending order,
 *   columns    int32 [rows, top], the columns they stand in (order of
 *              zo_top_logits).
 * rows < 2^31, vocab in [1, 2^31), top <= min(vocab, 1024).  Nothing to write is
 * ZO_EINVAL.
 */
typedef struct zo_score {
    const void *z;
    int32_t dtype;
    int64_t rows, vocab, ldz;
    const int32_t *tokens;
    float tau;
    float *logp, *stats;
    int32_t top;
    float *values;
    int32_t *columns;
} zo_score;

/*
 * zo_token_logprobs -- per row, with d = (z - m) / tau:
 *   log p = d - log S, entropy = log S - sum of exp(d) d / S,
 * in one read of the logits.  Where S < 2, S - 1 is formed apart from its 1: log S, the
 * largest log probability and the entropy are then right in relation to themselves, down
 * to terms of 2^-126.  log S and the entropy are not below 0, log p not above.  A d that
 * passes binary32 is -infinity; a difference z - m may pass it.  A row's results are the
 * same bits in any batch and whatever else is wanted.  A logit of -infinity has log p =
 * -infinity and adds 0 to the entropy.  A row of only -infinity has the statistics
 * -infinity, -infinity, 0 and log probabilities of -infinity; in one with a NaN or
 * +infinity all of them are NaN.
 */
int zo_token_logprobs(const zo_score *args, hipStream_t stream);

/*
 * Arguments of zo_token_logprobs_grad (host struct, read during the call).
 *   z, tokens, tau, stats   as zo_token_logprobs took and left them.
 *   dlogp      NULL (0), or float [rows]: the gradient of logp; needs tokens.
 *   dentropy   NULL (0), or float [rows]: the gradient of the entropy.
 *   dz         [rows, vocab] of z's type, row stride lddz; may be z itself (with
 *              lddz = ldz).
 * rows < 2^31, vocab in [1, 2^31).  Both NULL is ZO_EINVAL.
 */
typedef struct zo_score_back {
    const void *z;
    int32_t dtype;
    int64_t rows, vocab, ldz;
    const int32_t *tokens;
    const float *stats;
    float tau;
    const float *dlogp, *dentropy;
    void *dz;
    int64_t lddz;
} zo_score_back;

/*
 * zo_token_logprobs_grad -- per row, with p and log p of z,
 *   dz = (dlogp (onehot(token) - p) - dentropy p (log p + entropy)) / tau.
 * A row without a token has no first part.  Rows in which both gradients are 0 are not
 * read: dz = 0.  A logit of -infinity has p = 0; a row of only -infinity has no
 * gradient; one with NaN statistics has dz = NaN.
 */
int zo_token_logprobs_grad(const zo_score_back *args, hipStream_t stream);

/* HIP error behind the calling thread's last ZO_EHIP from this header. */
const char *zo_ops_last_hip_error(void);

#ifdef __cplusplus
}
#endif

#endif /* ZO_OPS_H */
