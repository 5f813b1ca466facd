/*
 * zo_ops.h -- operators that stand next to the optimizer step of zo_adam.h, on
 * one MI355X (gfx950): matrices in microscaled 4-bit floating point (quantised
 * from the binary32 shard or from activations, read back, multiplied), a
 * teacher's top logits, and the distillation loss with the gradient of the
 * student's logits.
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

/* HIP error behind the calling thread's last ZO_EHIP from this header. */
const char *zo_ops_last_hip_error(void);

#ifdef __cplusplus
}
#endif

#endif /* ZO_OPS_H */
