// zo_mx4_device.h -- what the kernels of 4-bit matrices share: the scale and the
// codes of a block, and the scaled matrix instruction.
#pragma once

#include "zo_ops_device.h"

namespace zo {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// Largest magnitude bits of the 8 elements of a lane (dwords of one element in
// binary32, of two otherwise, then the larger of the two).
template <int GT>
__device__ __forceinline__ uint32_t mag(uint32_t a, uint32_t w)
{
    if constexpr (GT == GT_F32) {
        return max(a, w & 0x7FFFFFFFu);
    } else {
        return __builtin_bit_cast(
            uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a),
                                                __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu)));
    }
}

// Scale byte of a block from its largest magnitude's bits.
template <int GT>
__device__ __forceinline__ uint32_t scale_byte(uint32_t a)
{
    const uint32_t e = __float_as_uint(widen<GT>((typename Elem<GT>::T)a)) >> 23;
    return e == 255 ? 255u : (uint32_t)max((int)e - 2, 0);
}

// Two elements (dwords w0 and w1 in binary32, the halves of w0 otherwise) into
// byte B of `old`.
template <int GT, int B>
__device__ __forceinline__ uint32_t convert2(uint32_t old, uint32_t w0, uint32_t w1, float scale)
{
    if constexpr (GT == GT_F32)
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, __uint_as_float(w0),
                                                        __uint_as_float(w1), scale, B);
    else if constexpr (GT == GT_BF16)
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(bf16x2, w0),
                                                         scale, B);
    else
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(old, __builtin_bit_cast(f16x2, w0),
                                                        scale, B);
}

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// acc += a-tile x b-tile; SA / SB: which byte of the scale dwords.
template <int SA, int SB>
__device__ __forceinline__ f32x4 mfma(const u32x4 &a, const u32x4 &b, f32x4 acc, uint32_t sa,
                                      uint32_t sb)
{
    const i32x8 x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    const i32x8 y = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, acc, 4, 4, SA, (int)sa, SB,
                                                            (int)sb);
}

typedef float f32x16 __attribute__((ext_vector_type(16)));

// The 32 x 32 x 64 form: lane l holds row l % 32, elements 32 (l / 32) .. + 31; of its
// sixteen results lane l holds, for b's columns l % 32, a's rows
// 8 q + 4 (l / 32) + 0..3 at 4 q.
template <int SA, int SB>
__device__ __forceinline__ f32x16 mfma32(const u32x4 &a, const u32x4 &b, f32x16 acc, uint32_t sa,
                                         uint32_t sb)
{
    const i32x8 x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    const i32x8 y = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, acc, 4, 4, SA, (int)sa, SB,
                                                           (int)sb);
}

}  // namespace zo
