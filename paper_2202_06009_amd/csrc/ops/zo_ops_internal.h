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

// An i8 matrix as the kernels take it: rows of `wide` bytes.
struct I8View {
    int8_t *codes;
    float *scales;
    int64_t rows, cols, wide;
};

bool i8_quantize_fits(int64_t rows, int64_t cols, bool transposed);
bool i8_product_fits(int64_t m, int64_t n, int64_t k);
// Sets of partial column maxima that a quantisation along the columns leaves in its
// workspace.
int64_t i8_blocks(int64_t rows);

hipError_t launch_i8_quantize(const void *x, int gt, int64_t rows, int64_t cols, int64_t ld,
                              const I8View *q, const I8View *qt, uint32_t *work, hipStream_t st);
hipError_t launch_i8_dequantize(const I8View &q, void *out, int gt, int64_t ld, hipStream_t st);
hipError_t launch_i8_product(const I8View &a, const I8View &b, void *out, int gt, int64_t ld,
                             hipStream_t st);
// As for the 4-bit products.  Few rows / tiles, us (rows x matrix): 32 x 6400 x 1600 6.6 / 7.0,
// 40 8.0 / 7.1; 32 x 50257 x 1600 19.9 / 18.8, 40 21.4 / 18.9; 32 x 1600 x 6400 10.8 / 16.3, 40
// 14.1 / 16.3, 64 17.0 / 16.6; 16 x 4096 x 1024 3.6 / 5.0, 40 5.2 / 5.0.  Where they cross goes by
// the matrix, from below 32 rows (50257 x 1600) to above 40 (1600 x 6400); this one bound for all
// gives away 6% there and 16% here.
constexpr int kI8FewRows = 32;
bool i8_few_fits(int64_t n, int64_t k);
hipError_t launch_i8_few(const I8View &a, const I8View &b, void *out, int gt, int64_t ld,
                         hipStream_t st);
bool i8_few_fused(int64_t rows, int64_t k);
hipError_t launch_i8_few_fused(const void *x, int gx, int64_t rows, int64_t cols, int64_t ldx,
                               const I8View &b, void *out, int gt, int64_t ld, hipStream_t st);

// Blocks of rows whose parts of dw a norm's backward pass leaves in its workspace.
int64_t norm_grad_blocks(int64_t rows);
hipError_t launch_norm(const zo_norm &a, const I8View &q, hipStream_t st);
hipError_t launch_norm_grad(const zo_norm_back &a, hipStream_t st);
hipError_t launch_score(const zo_score &a, hipStream_t st);
hipError_t launch_score_grad(const zo_score_back &a, hipStream_t st);

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
