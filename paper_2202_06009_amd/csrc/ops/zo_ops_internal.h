// zo_ops_internal.h -- launchers of the operators of zo_ops.h, called by its
// host side after every argument has been checked.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "zo_ops.h"

namespace zo {

// An mx4 matrix as the kernels take it: KT = ceil(cols / 128) tiles of 128
// columns.
struct Mx4View {
    uint8_t *codes, *scales;
    int64_t rows, cols, kt;
};

// A launch holds fewer than 2^32 threads.  The launchers of matrices count on their
// callers' having asked; rows of logits go into as many launches as they need.
inline bool fits_a_launch(int64_t groups, int threads)
{
    return groups <= (int64_t)UINT32_MAX / threads;
}
constexpr int64_t kLaunchRows = 1 << 21;     // of up to 1024 threads each

bool mx4_quantize_fits(int gt, int64_t rows, int64_t cols, bool transposed);
bool mx4_dequantize_fits(int64_t rows, int64_t cols);
bool mx4_product_fits(int64_t m, int64_t n, int64_t k, int gt, const void *out, int64_t ld);

hipError_t launch_mx4_quantize(const void *x, int gt, int64_t rows, int64_t cols, int64_t ld,
                               const Mx4View *q, const Mx4View *qt, hipStream_t st);
hipError_t launch_mx4_dequantize(const Mx4View &q, void *out, int gt, int64_t ld,
                                 hipStream_t st);
hipError_t launch_mx4_product(const Mx4View &a, const Mx4View &b, void *out, int gt, int64_t ld,
                              hipStream_t st);
// The products of few rows of a (at most kFewRows) by b; from activations x of
// element type gx that the kernel quantises itself, where few_fused says so of
// [rows, k] by [n, k].
constexpr int kFewRows = 64;
bool mx4_few_fits(int64_t n, int64_t k);
hipError_t launch_mx4_few(const Mx4View &a, const Mx4View &b, void *out, int gt, int64_t ld,
                          hipStream_t st);
bool few_fused(int64_t rows, int64_t n, int64_t k);
hipError_t launch_mx4_few_fused(const void *x, int gx, int64_t rows, int64_t cols, int64_t ldx,
                                const Mx4View &b, void *out, int gt, int64_t ld, hipStream_t st);

struct TopArgs {
    const void *z;
    int64_t rows, vocab, ld;
    int top;
    float tau;
    float *values;
    int32_t *columns;
    float *lse;
};
hipError_t launch_top_logits(const TopArgs &a, int gt, hipStream_t st);
hipError_t launch_distill(const zo_distill &a, hipStream_t st);

}  // namespace zo
