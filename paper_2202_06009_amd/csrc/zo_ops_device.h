// zo_ops_device.h -- device code shared by the kernels of zo_ops.h: element
// types and loads on any element boundary, reductions over a workgroup.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "zo_internal.h"
#include "zo_ops_internal.h"

namespace zo {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// The same on any element boundary: one access each, the hardware splits it.
typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32_a2 __attribute__((aligned(2)));

template <int GT>
struct Elem {
    using T = uint16_t;              // the bits of an element
    static constexpr int kVec = 8;   // elements of a 16-byte access
};
template <>
struct Elem<GT_F32> {
    using T = uint32_t;
    static constexpr int kVec = 4;
};

// Calls f(integral_constant<GT>) for a run-time element type.
template <class F>
static hipError_t with_elem_type(int gt, F &&f)
{
    switch (gt) {
    case GT_F32: return f(std::integral_constant<int, GT_F32>{});
    case GT_F16: return f(std::integral_constant<int, GT_F16>{});
    case GT_BF16: return f(std::integral_constant<int, GT_BF16>{});
    default: return hipErrorInvalidValue;
    }
}

template <int GT>
__device__ __forceinline__ float widen(typename Elem<GT>::T bits)
{
    if constexpr (GT == GT_F32)
        return __uint_as_float(bits);
    else if constexpr (GT == GT_BF16)
        return __uint_as_float((uint32_t)bits << 16);
    else
        return (float)__builtin_bit_cast(_Float16, bits);
}

// v rounded to nearest even.
template <int GT>
__device__ __forceinline__ typename Elem<GT>::T narrow(float v)
{
    if constexpr (GT == GT_F32)
        return __float_as_uint(v);
    else if constexpr (GT == GT_BF16)
        return __builtin_bit_cast(uint16_t, (__bf16)v);
    else
        return __builtin_bit_cast(uint16_t, (_Float16)v);
}

// Element q of the 16 bytes w.
template <int GT>
__device__ __forceinline__ float elem_of(const u32x4 &w, int q)
{
    if constexpr (GT == GT_F32)
        return __uint_as_float(w[q]);
    else if constexpr (GT == GT_BF16)
        return __uint_as_float(q & 1 ? w[q >> 1] & 0xFFFF0000u : w[q >> 1] << 16);
    else
        return (float)__builtin_bit_cast(_Float16, (uint16_t)(w[q >> 1] >> (16 * (q & 1))));
}

// 16 bytes from an element boundary; of the nv < kVec elements that are there
// only those, `fill` (an element's bits) in the place of the others.
template <int GT>
__device__ __forceinline__ u32x4 load16(const typename Elem<GT>::T *p, int64_t nv,
                                        uint32_t fill = 0)
{
    constexpr int V = Elem<GT>::kVec;
    if (nv >= V) return *reinterpret_cast<const u32x4_a2 *>(p);
    u32x4 w;
    if constexpr (GT == GT_F32) {
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = q < nv ? p[q] : fill;
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            w[q] = (2 * q < nv ? (uint32_t)p[2 * q] : fill) |
                   (2 * q + 1 < nv ? (uint32_t)p[2 * q + 1] : fill) << 16;
    }
    return w;
}

// Stores the first nv of kVec elements.
template <int GT>
__device__ __forceinline__ void store16(typename Elem<GT>::T *p, const u32x4 &w, int64_t nv)
{
    constexpr int V = Elem<GT>::kVec;
    if (nv >= V) {
        *reinterpret_cast<u32x4_a2 *>(p) = w;
        return;
    }
    if constexpr (GT == GT_F32) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (q < nv) p[q] = w[q];
    } else {
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (q < nv) p[q] = (uint16_t)(w[q >> 1] >> (16 * (q & 1)));
    }
}

// kVec floats rounded into 16 bytes.
template <int GT>
__device__ __forceinline__ u32x4 pack16(const float (&v)[Elem<GT>::kVec])
{
    u32x4 w;
    if constexpr (GT == GT_F32) {
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = __float_as_uint(v[q]);
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            w[q] = (uint32_t)narrow<GT>(v[2 * q]) | (uint32_t)narrow<GT>(v[2 * q + 1]) << 16;
    }
    return w;
}

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// 2^x to about one unit in the last place; results below 2^-126 become 0,
// which no sum of a softmax notices.
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xF, 0xF, true);
}

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// Over a workgroup of NW waves; `s` is NW floats of shared memory that the
// call may overwrite (it synchronises before and after).
template <int NW>
__device__ __forceinline__ float group_max(float v, float *s)
{
    v = wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    float r = s[0];
#pragma unroll
    for (int i = 1; i < NW; ++i) r = fmaxf(r, s[i]);
    return r;
}

template <int NW>
__device__ __forceinline__ float group_sum(float v, float *s)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    float r = s[0];
#pragma unroll
    for (int i = 1; i < NW; ++i) r += s[i];
    return r;
}

}  // namespace zo
