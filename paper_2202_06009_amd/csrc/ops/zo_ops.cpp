// zo_ops.cpp -- host side of the operators of include/zo_ops.h: every argument
// is checked here, then one launcher is called.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>

#include "zo_internal.h"
#include "zo_ops.h"
#include "zo_ops_internal.h"

namespace {

constexpr int64_t kMaxDim = (int64_t)1 << 30;
constexpr int64_t kMaxLd = (int64_t)1 << 40;

thread_local char hip_err[192];

int from_hip(hipError_t e)
{
    if (e == hipSuccess) return ZO_OK;
    std::snprintf(hip_err, sizeof hip_err, "%s: %s", hipGetErrorName(e), hipGetErrorString(e));
    return ZO_EHIP;
}

// The kernels' element type, or -1.
int elem(int32_t dtype)
{
    switch (dtype) {
    case ZO_DTYPE_F32: return zo::GT_F32;
    case ZO_DTYPE_F16: return zo::GT_F16;
    case ZO_DTYPE_BF16: return zo::GT_BF16;
    default: return -1;
    }
}

bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// A matrix [rows, cols] of element type `gt` with row stride ld.
int check_matrix(const void *p, int gt, int64_t rows, int64_t cols, int64_t ld)
{
    if (gt < 0 || rows < 0 || cols < 0 || rows > kMaxDim || cols > kMaxDim) return ZO_EINVAL;
    if (rows == 0 || cols == 0) return ZO_OK;
    if (!p || ld < cols || ld > kMaxLd) return ZO_EINVAL;
    return aligned(p, gt == zo::GT_F32 ? 4 : 2) ? ZO_OK : ZO_EALIGN;
}

int check_mx4(const zo_mx4 *q)
{
    if (!q || q->rows < 0 || q->cols < 0 || q->rows > kMaxDim || q->cols > kMaxDim)
        return ZO_EINVAL;
    if (q->rows == 0 || q->cols == 0) return ZO_OK;
    if (!q->codes || !q->scales) return ZO_EINVAL;
    return aligned(q->codes, 16) && aligned(q->scales, 4) ? ZO_OK : ZO_EALIGN;
}

zo::Mx4View view(const zo_mx4 *q)
{
    return {(uint8_t *)q->codes, (uint8_t *)q->scales, q->rows, q->cols, (q->cols + 127) / 128};
}

int check_i8(const zo_i8 *q)
{
    if (!q || q->rows < 0 || q->cols < 0 || q->rows > kMaxDim || q->cols > kMaxDim)
        return ZO_EINVAL;
    if (q->rows == 0 || q->cols == 0) return ZO_OK;
    if (!q->codes || !q->scales) return ZO_EINVAL;
    return aligned(q->codes, 16) && aligned(q->scales, 4) ? ZO_OK : ZO_EALIGN;
}

zo::I8View view(const zo_i8 *q)
{
    return {(int8_t *)q->codes, q->scales, q->rows, q->cols, (q->cols + 127) / 128 * 128};
}

constexpr int64_t kMaxI8Depth = 131072;      // 127 * 127 * 131072 < 2^31
constexpr int64_t kMaxNormCols = 32768;
constexpr float kLeastNormal = 0x1p-126f;

uintptr_t size_of(int gt) { return gt == zo::GT_F32 ? 4 : 2; }

// A matrix of checked sizes and type: there, its rows apart, its elements aligned.
int check_rows(const void *p, int gt, int64_t cols, int64_t ld)
{
    if (!p || ld < cols || ld > kMaxLd) return ZO_EINVAL;
    return aligned(p, size_of(gt)) ? ZO_OK : ZO_EALIGN;
}

// The same of a buffer that need not be there.
int check_optional(const void *p, int gt, int64_t cols, int64_t ld)
{
    return p ? check_rows(p, gt, cols, ld) : ZO_OK;
}

// Whether p, where it is another argument's buffer, has its stride.
bool in_place(const void *p, int64_t ld, const void *from, int64_t ld_from)
{
    return !p || p != from || ld == ld_from;
}

}  // namespace

extern "C" {

const char *zo_ops_last_hip_error(void) { return hip_err; }

int64_t zo_mx4_code_bytes(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 0 || rows > kMaxDim || cols > kMaxDim) return ZO_EINVAL;
    return (rows + 63) / 64 * 64 * ((cols + 127) / 128) * 64;
}

int64_t zo_mx4_scale_bytes(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 0 || rows > kMaxDim || cols > kMaxDim) return ZO_EINVAL;
    return (rows + 63) / 64 * 64 * ((cols + 127) / 128) * 4;
}

int zo_mx4_quantize(const void *x, int32_t dtype, int64_t rows, int64_t cols, int64_t ld,
                    const zo_mx4 *q, const zo_mx4 *qt, hipStream_t stream)
{
    const int gt = elem(dtype);
    int rc = check_matrix(x, gt, rows, cols, ld);
    if (rc) return rc;
    if (!q && !qt) return ZO_EINVAL;
    if (q && (q->rows != rows || q->cols != cols)) return ZO_EINVAL;
    if (qt && (qt->rows != cols || qt->cols != rows)) return ZO_EINVAL;
    if (q && (rc = check_mx4(q))) return rc;
    if (qt && (rc = check_mx4(qt))) return rc;
    if (!zo::mx4_quantize_fits(gt, rows, cols, qt != nullptr)) return ZO_EINVAL;
    zo::Mx4View v{}, vt{};
    if (q) v = view(q);
    if (qt) vt = view(qt);
    return from_hip(zo::launch_mx4_quantize(x, gt, rows, cols, ld, q ? &v : nullptr,
                                            qt ? &vt : nullptr, stream));
}

int zo_mx4_dequantize(const zo_mx4 *q, void *out, int32_t dtype, int64_t ld, hipStream_t stream)
{
    int rc = check_mx4(q);
    if (rc) return rc;
    const int gt = elem(dtype);
    if ((rc = check_matrix(out, gt, q->rows, q->cols, ld))) return rc;
    if (!zo::mx4_dequantize_fits(q->rows, q->cols)) return ZO_EINVAL;
    return from_hip(zo::launch_mx4_dequantize(view(q), out, gt, ld, stream));
}

int zo_mx4_product(const zo_mx4 *a, const zo_mx4 *b, void *out, int32_t dtype, int64_t ld,
                   hipStream_t stream)
{
    int rc = check_mx4(a);
    if (rc) return rc;
    if ((rc = check_mx4(b))) return rc;
    if (a->cols != b->cols) return ZO_EINVAL;
    const int gt = elem(dtype);
    if ((rc = check_matrix(out, gt, a->rows, b->rows, ld))) return rc;
    if (!zo::mx4_product_fits(a->rows, b->rows, a->cols, gt, out, ld)) return ZO_EINVAL;
    return from_hip(zo::launch_mx4_product(view(a), view(b), out, gt, ld, stream));
}

int zo_mx4_linear(const void *x, int32_t dtype, int64_t ldx, const zo_mx4 *w, const zo_mx4 *xq,
                  void *out, int32_t out_dtype, int64_t ldo, hipStream_t stream)
{
    int rc = check_mx4(xq);
    if (rc) return rc;
    if ((rc = check_mx4(w))) return rc;
    if (xq->cols != w->cols) return ZO_EINVAL;
    const int gx = elem(dtype), go = elem(out_dtype);
    if ((rc = check_matrix(x, gx, xq->rows, xq->cols, ldx))) return rc;
    if ((rc = check_matrix(out, go, xq->rows, w->rows, ldo))) return rc;
    const bool fused = zo::few_fused(xq->rows, w->rows, xq->cols);
    if (!zo::mx4_product_fits(xq->rows, w->rows, w->cols, go, out, ldo) ||
        (!fused && !zo::mx4_quantize_fits(gx, xq->rows, xq->cols, false)))
        return ZO_EINVAL;
    const zo::Mx4View v = view(xq);
    if (v.rows && w->rows && fused)
        return from_hip(zo::launch_mx4_few_fused(x, gx, v.rows, v.cols, ldx, view(w), out, go, ldo,
                                                 stream));
    rc = from_hip(zo::launch_mx4_quantize(x, gx, xq->rows, xq->cols, ldx, &v, nullptr, stream));
    if (rc) return rc;
    return from_hip(zo::launch_mx4_product(v, view(w), out, go, ldo, stream));
}

int zo_top_logits(const void *z, int32_t dtype, int64_t rows, int64_t vocab, int64_t ld,
                  int32_t top, float tau, float *values, int32_t *columns, float *lse,
                  hipStream_t stream)
{
    const int gt = elem(dtype);
    if (rows < 0 || rows > INT32_MAX || vocab < 1 || vocab > INT32_MAX) return ZO_EINVAL;
    if (top < 1 || top > 1024 || top > vocab) return ZO_EINVAL;
    if (gt < 0 || !(tau > 0.0f) || !std::isfinite(tau)) return ZO_EINVAL;
    if (rows == 0) return ZO_OK;
    if (!z || ld < vocab || ld > kMaxLd || !values || !columns) return ZO_EINVAL;
    if (!aligned(z, gt == zo::GT_F32 ? 4 : 2) || !aligned(values, 4) || !aligned(columns, 4) ||
        !aligned(lse, 4))
        return ZO_EALIGN;
    const zo::TopArgs a = {z, rows, vocab, ld, top, tau, values, columns, lse};
    return from_hip(zo::launch_top_logits(a, gt, stream));
}

int zo_distill_loss(const zo_distill *args, hipStream_t stream)
{
    if (!args) return ZO_EINVAL;
    const zo_distill &a = *args;
    const int gt = elem(a.dtype);
    if (a.rows < 0 || a.rows > INT32_MAX || a.vocab < 1 || a.vocab > (1 << 18)) return ZO_EINVAL;
    if (gt < 0 || a.top < 1 || a.top > 1024) return ZO_EINVAL;
    if (!(a.tau > 0.0f) || !std::isfinite(a.tau) || !std::isfinite(a.kd_weight) ||
        !std::isfinite(a.ce_weight))
        return ZO_EINVAL;
    if (a.rows == 0) return ZO_OK;
    if (!a.z || a.ldz < a.vocab || a.ldz > kMaxLd || !a.values || !a.columns) return ZO_EINVAL;
    if (!a.loss && !a.dz) return ZO_EINVAL;
    if (a.dz && (a.lddz < a.vocab || a.lddz > kMaxLd || (a.dz == a.z && a.lddz != a.ldz)))
        return ZO_EINVAL;
    const uintptr_t ea = gt == zo::GT_F32 ? 4 : 2;
    if (!aligned(a.z, ea) || !aligned(a.dz, ea) || !aligned(a.values, 4) ||
        !aligned(a.columns, 4) || !aligned(a.teacher_lse, 4) || !aligned(a.labels, 4) ||
        !aligned(a.row_weight, 4) || !aligned(a.loss, 4))
        return ZO_EALIGN;
    return from_hip(zo::launch_distill(a, stream));
}

int64_t zo_i8_code_bytes(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 0 || rows > kMaxDim || cols > kMaxDim) return ZO_EINVAL;
    return rows * ((cols + 127) / 128 * 128);
}

int64_t zo_i8_work_bytes(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 0 || rows > kMaxDim || cols > kMaxDim) return ZO_EINVAL;
    return zo::i8_blocks(rows) * cols * 4;
}

int zo_i8_quantize(const void *x, int32_t dtype, int64_t rows, int64_t cols, int64_t ld,
                   const zo_i8 *q, const zo_i8 *qt, void *work, hipStream_t stream)
{
    const int gt = elem(dtype);
    int rc = check_matrix(x, gt, rows, cols, ld);
    if (rc) return rc;
    if (!q && !qt) return ZO_EINVAL;
    if (q && (q->rows != rows || q->cols != cols)) return ZO_EINVAL;
    if (qt && (qt->rows != cols || qt->cols != rows)) return ZO_EINVAL;
    if (q && (rc = check_i8(q))) return rc;
    if (qt && (rc = check_i8(qt))) return rc;
    if (rows == 0 || cols == 0) return ZO_OK;
    if (qt && !work) return ZO_EINVAL;
    if (qt && !aligned(work, 4)) return ZO_EALIGN;
    if (!zo::i8_quantize_fits(rows, cols, qt != nullptr)) return ZO_EINVAL;
    zo::I8View v{}, vt{};
    if (q) v = view(q);
    if (qt) vt = view(qt);
    return from_hip(zo::launch_i8_quantize(x, gt, rows, cols, ld, q ? &v : nullptr,
                                           qt ? &vt : nullptr, (uint32_t *)work, stream));
}

int zo_i8_dequantize(const zo_i8 *q, void *out, int32_t dtype, int64_t ld, hipStream_t stream)
{
    int rc = check_i8(q);
    if (rc) return rc;
    const int gt = elem(dtype);
    if ((rc = check_matrix(out, gt, q->rows, q->cols, ld))) return rc;
    return from_hip(zo::launch_i8_dequantize(view(q), out, gt, ld, stream));
}

int zo_i8_product(const zo_i8 *a, const zo_i8 *b, void *out, int32_t dtype, int64_t ld,
                  hipStream_t stream)
{
    int rc = check_i8(a);
    if (rc) return rc;
    if ((rc = check_i8(b))) return rc;
    if (a->cols != b->cols || a->cols > kMaxI8Depth) return ZO_EINVAL;
    const int gt = elem(dtype);
    if ((rc = check_matrix(out, gt, a->rows, b->rows, ld))) return rc;
    if (!zo::i8_product_fits(a->rows, b->rows, a->cols)) return ZO_EINVAL;
    return from_hip(zo::launch_i8_product(view(a), view(b), out, gt, ld, stream));
}

int zo_i8_linear(const void *x, int32_t dtype, int64_t ldx, const zo_i8 *w, const zo_i8 *xq,
                 void *out, int32_t out_dtype, int64_t ldo, hipStream_t stream)
{
    int rc = check_i8(xq);
    if (rc) return rc;
    if ((rc = check_i8(w))) return rc;
    if (xq->cols != w->cols || w->cols > kMaxI8Depth) return ZO_EINVAL;
    const int gx = elem(dtype), go = elem(out_dtype);
    if ((rc = check_matrix(x, gx, xq->rows, xq->cols, ldx))) return rc;
    if ((rc = check_matrix(out, go, xq->rows, w->rows, ldo))) return rc;
    if (!zo::i8_product_fits(xq->rows, w->rows, w->cols)) return ZO_EINVAL;
    if (xq->rows == 0 || w->rows == 0) return ZO_OK;
    const zo::I8View v = view(xq);
    if (zo::i8_few_fused(v.rows, v.cols))
        return from_hip(zo::launch_i8_few_fused(x, gx, v.rows, v.cols, ldx, view(w), out, go, ldo,
                                                stream));
    rc = from_hip(zo::launch_i8_quantize(x, gx, v.rows, v.cols, ldx, &v, nullptr, nullptr, stream));
    if (rc) return rc;
    return from_hip(zo::launch_i8_product(v, view(w), out, go, ldo, stream));
}

int zo_rms_norm(const zo_norm *args, hipStream_t stream)
{
    if (!args) return ZO_EINVAL;
    const zo_norm &a = *args;
    const int gt = elem(a.dtype), wt = elem(a.weight_dtype);
    if (gt < 0 || wt < 0 || (wt != gt && wt != zo::GT_F32)) return ZO_EINVAL;
    if (a.rows < 0 || a.rows > INT32_MAX || a.cols < 1 || a.cols > kMaxNormCols) return ZO_EINVAL;
    if (!(a.eps >= kLeastNormal) || !std::isfinite(a.eps)) return ZO_EINVAL;
    if (a.q && (a.q->rows != a.rows || a.q->cols != a.cols)) return ZO_EINVAL;
    if (a.rows == 0) return ZO_OK;
    if (!a.h && !a.out && !a.q && !a.rstd) return ZO_EINVAL;
    int rc;
    if ((rc = check_rows(a.x, gt, a.cols, a.ldx))) return rc;
    if ((rc = check_optional(a.residual, gt, a.cols, a.ldr))) return rc;
    if ((rc = check_optional(a.h, gt, a.cols, a.ldh))) return rc;
    if ((rc = check_optional(a.out, gt, a.cols, a.ldo))) return rc;
    if (a.q && (rc = check_i8(a.q))) return rc;
    if (!a.weight || (a.out && a.out == a.h)) return ZO_EINVAL;
    if (!in_place(a.h, a.ldh, a.x, a.ldx) || !in_place(a.h, a.ldh, a.residual, a.ldr) ||
        !in_place(a.out, a.ldo, a.x, a.ldx) || !in_place(a.out, a.ldo, a.residual, a.ldr))
        return ZO_EINVAL;
    if (!aligned(a.weight, size_of(wt)) || !aligned(a.rstd, 4)) return ZO_EALIGN;
    return from_hip(zo::launch_norm(a, a.q ? view(a.q) : zo::I8View{}, stream));
}

int64_t zo_rms_norm_work_bytes(int64_t rows, int64_t cols)
{
    if (rows < 0 || rows > INT32_MAX || cols < 1 || cols > kMaxNormCols) return ZO_EINVAL;
    return zo::norm_grad_blocks(rows) * cols * 4;
}

int zo_rms_norm_grad(const zo_norm_back *args, hipStream_t stream)
{
    if (!args) return ZO_EINVAL;
    const zo_norm_back &a = *args;
    const int gt = elem(a.dtype), wt = elem(a.weight_dtype);
    if (gt < 0 || wt < 0 || (wt != gt && wt != zo::GT_F32)) return ZO_EINVAL;
    if (a.rows < 0 || a.rows > INT32_MAX || a.cols < 1 || a.cols > kMaxNormCols) return ZO_EINVAL;
    if (!aligned(a.dw, 4) || !aligned(a.work, 4)) return ZO_EALIGN;
    if (a.rows > 0) {
        if (!a.dx && !a.dw) return ZO_EINVAL;
        int rc;
        if ((rc = check_rows(a.dy, gt, a.cols, a.lddy))) return rc;
        if ((rc = check_rows(a.h, gt, a.cols, a.ldh))) return rc;
        if ((rc = check_optional(a.dh, gt, a.cols, a.lddh))) return rc;
        if ((rc = check_optional(a.dx, gt, a.cols, a.lddx))) return rc;
        if (!a.weight || !a.rstd || (a.dw && !a.work)) return ZO_EINVAL;
        if (!in_place(a.dx, a.lddx, a.dy, a.lddy) || !in_place(a.dx, a.lddx, a.h, a.ldh) ||
            !in_place(a.dx, a.lddx, a.dh, a.lddh))
            return ZO_EINVAL;
        if (!aligned(a.weight, size_of(wt)) || !aligned(a.rstd, 4)) return ZO_EALIGN;
    }
    return from_hip(zo::launch_norm_grad(a, stream));
}

int zo_token_logprobs(const zo_score *args, hipStream_t stream)
{
    if (!args) return ZO_EINVAL;
    const zo_score &a = *args;
    const int gt = elem(a.dtype);
    if (a.rows < 0 || a.rows > INT32_MAX || a.vocab < 1 || a.vocab > INT32_MAX) return ZO_EINVAL;
    if (a.top < 0 || a.top > 1024 || a.top > a.vocab) return ZO_EINVAL;
    if (gt < 0 || !(a.tau >= kLeastNormal) || !std::isfinite(a.tau)) return ZO_EINVAL;
    if (a.rows == 0) return ZO_OK;
    if (!a.tokens && !a.stats && a.top == 0) return ZO_EINVAL;
    const int rc = check_rows(a.z, gt, a.vocab, a.ldz);
    if (rc) return rc;
    if ((a.tokens && !a.logp) || (a.top > 0 && (!a.values || !a.columns))) return ZO_EINVAL;
    if (!aligned(a.tokens, 4) || !aligned(a.logp, 4) || !aligned(a.stats, 4) ||
        !aligned(a.values, 4) || !aligned(a.columns, 4))
        return ZO_EALIGN;
    return from_hip(zo::launch_score(a, stream));
}

int zo_token_logprobs_grad(const zo_score_back *args, hipStream_t stream)
{
    if (!args) return ZO_EINVAL;
    const zo_score_back &a = *args;
    const int gt = elem(a.dtype);
    if (a.rows < 0 || a.rows > INT32_MAX || a.vocab < 1 || a.vocab > INT32_MAX) return ZO_EINVAL;
    if (gt < 0 || !(a.tau >= kLeastNormal) || !std::isfinite(a.tau)) return ZO_EINVAL;
    if (a.rows == 0) return ZO_OK;
    if ((!a.dlogp && !a.dentropy) || (a.dlogp && !a.tokens)) return ZO_EINVAL;
    int rc;
    if ((rc = check_rows(a.z, gt, a.vocab, a.ldz))) return rc;
    if ((rc = check_rows(a.dz, gt, a.vocab, a.lddz))) return rc;
    if (!a.stats || !in_place(a.dz, a.lddz, a.z, a.ldz)) return ZO_EINVAL;
    if (!aligned(a.tokens, 4) || !aligned(a.stats, 4) || !aligned(a.dlogp, 4) ||
        !aligned(a.dentropy, 4))
        return ZO_EALIGN;
    return from_hip(zo::launch_score_grad(a, stream));
}

}  // extern "C"
