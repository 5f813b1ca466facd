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
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
// The same on any element boundary: one access each, the hardware splits it.
typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));

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

template <class T>
struct AsIs {
    using type = T;
};

// Launches a kernel; the launch's own error, which an error that an earlier call of the
// program left in the runtime is not.
template <class... P>
static hipError_t start(void (*kernel)(P...), int64_t groups, int threads, uint32_t lds,
                        hipStream_t st, typename AsIs<P>::type... args)
{
    void *at[] = {&args...};
    return hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3((uint32_t)groups),
                           dim3((uint32_t)threads), at, lds, st);
}

// Shared memory beyond 64 KiB has to be asked for.
[[maybe_unused]] static hipError_t allow_lds(const void *kernel, uint32_t lds)
{
    if (lds <= 65536) return hipSuccess;
    return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
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

// Stores the first nv of four floats, rounded.
template <int GT>
__device__ __forceinline__ void store_few(typename Elem<GT>::T *p, const f32x4 &v, int64_t nv)
{
    if (nv >= 4) {
        if constexpr (GT == GT_F32) {
            *reinterpret_cast<u32x4_a2 *>(p) = __builtin_bit_cast(u32x4, v);
        } else {
            const u32x2 w = {(uint32_t)narrow<GT>(v[0]) | (uint32_t)narrow<GT>(v[1]) << 16,
                             (uint32_t)narrow<GT>(v[2]) | (uint32_t)narrow<GT>(v[3]) << 16};
            *reinterpret_cast<u32x2_a2 *>(p) = w;
        }
    } else {
        for (int q = 0; q < 4; ++q)
            if (q < nv) p[q] = narrow<GT>(v[q]);
    }
}

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// log2(e) / tau, finite for a tau below the normal numbers too: 0 times it is then 0.
__device__ __forceinline__ float log2_factor(float tau)
{
    return fminf(kLog2e / tau, 0x1.fffffep127f);
}

// 2^x to about one unit in the last place; results below 2^-126 become 0,
// which no sum of a softmax notices.
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xF, 0xF, true);
}

// Over the 64 lanes of a wave, in a fixed order, the result in every lane: four
// steps within rows of 16 lanes, the rows' results handed on, lane 63 read.
struct OpMax {
    static constexpr float kNone = -INFINITY;
    __device__ static float of(float a, float b) { return fmaxf(a, b); }
};
struct OpMin {
    static constexpr float kNone = INFINITY;
    __device__ static float of(float a, float b) { return fminf(a, b); }
};
struct OpSum {
    static constexpr float kNone = 0.0f;
    __device__ static float of(float a, float b) { return a + b; }
};

template <class OP, int CTRL, int ROWS>
__device__ __forceinline__ float dpp_step(float v)
{
    const int o = __builtin_amdgcn_update_dpp((int)__float_as_uint(OP::kNone),
                                              (int)__float_as_uint(v), CTRL, ROWS, 0xF, false);
    return OP::of(v, __uint_as_float((uint32_t)o));
}

template <class OP>
__device__ __forceinline__ float wave_reduce(float v)
{
    v = dpp_step<OP, 0x111, 0xF>(v);   // row_shr:1, 2, 4, 8
    v = dpp_step<OP, 0x112, 0xF>(v);
    v = dpp_step<OP, 0x114, 0xF>(v);
    v = dpp_step<OP, 0x118, 0xF>(v);
    v = dpp_step<OP, 0x142, 0xA>(v);   // row_bcast:15 into rows 1 and 3
    v = dpp_step<OP, 0x143, 0xC>(v);   // row_bcast:31 into rows 2 and 3
    return __uint_as_float(
        (uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}

// The first step of a reduction over a workgroup of NW waves: the wave's result
// into s[wave].  After a barrier, group_get reads the whole.
template <class OP>
__device__ __forceinline__ void group_put(float v, float *s)
{
    v = wave_reduce<OP>(v);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
}

// A value that is the same in every lane, in a scalar register.
__device__ __forceinline__ float uniform(float v)
{
    return __uint_as_float(
        (uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(v)));
}

template <class OP, int NW>
__device__ __forceinline__ float group_get(const float *s)
{
    float r = s[0];
#pragma unroll
    for (int i = 1; i < NW; ++i) r = OP::of(r, s[i]);
    return uniform(r);
}

// A row of V < TH * NV * kVec + kVec logits in the registers of a workgroup of TH
// threads: thread tid holds the whole 16-byte vectors tid, tid + TH, ... of the
// row (-infinity where there are no more) and the first threads one each of the
// V % kVec logits that are left.  One pass over memory.
template <int GT>
constexpr uint32_t kNegInf = GT == GT_F32 ? 0xFF800000u : GT == GT_BF16 ? 0xFF80FF80u : 0xFC00FC00u;

template <int GT>
constexpr uint32_t kElemMask = GT == GT_F32 ? 0xFFFFFFFFu : 0xFFFFu;

template <int GT, int TH, int NV>
struct Resident {
    static constexpr int K = Elem<GT>::kVec;
    using T = typename Elem<GT>::T;
    u32x4 w[NV];
    float last;              // this thread's logit of the rest, or -infinity
    int vecs;                // whole vectors of the row

    __device__ __forceinline__ void load(const T *z, int64_t V)
    {
        vecs = (int)(V / K);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int i = at(v);
            w[v] = u32x4{kNegInf<GT>, kNegInf<GT>, kNegInf<GT>, kNegInf<GT>};
            if (i < vecs) w[v] = *reinterpret_cast<const u32x4_a2 *>(z + (int64_t)i * K);
        }
        last = -INFINITY;
        if ((int)threadIdx.x < (int)(V % K)) last = widen<GT>(z[last_column()]);
    }
    // Index of this thread's vector v, and column of its last logit.
    __device__ __forceinline__ int at(int v) const { return v * TH + (int)threadIdx.x; }
    __device__ __forceinline__ int last_column() const { return vecs * K + (int)threadIdx.x; }
    __device__ __forceinline__ bool has_last(int64_t V) const { return last_column() < V; }
};

template <int GT>
__device__ __forceinline__ float max_of(const u32x4 &w)
{
    float m = elem_of<GT>(w, 0);
#pragma unroll
    for (int q = 1; q < Elem<GT>::kVec; ++q) m = fmaxf(m, elem_of<GT>(w, q));
    return m;
}

// The compiler takes w for changed here: what is unpacked from it before is not
// kept for later (a resident row unpacked would not fit the registers).
template <int GT>
__device__ __forceinline__ void repack(u32x4 &w)
{
    if constexpr (GT != GT_F32)
        asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]));
}

// Where a sum of exponentials has its reference: 2^(z c - r) with r the largest
// z c rounded.  z c - r is one fused operation, rounded relative to itself, and
// r's own rounding is common to every term, so it cancels, while it is small for an
// exponent (|r| < 2^31: at most 64).  A largest logit of -infinity gives 0: every term
// is then 0.
__device__ __forceinline__ float reference(float m, float c)
{
    return m == -INFINITY ? 0.0f : m * c;
}

__device__ __forceinline__ float term(float z, float c, float r)
{
    return exp2_hw(__builtin_fmaf(z, c, -r));
}

}  // namespace zo
