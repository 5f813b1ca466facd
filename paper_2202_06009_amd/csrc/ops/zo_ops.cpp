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

}  // extern "C"
