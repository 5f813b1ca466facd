// zo_i8_device.h -- what the kernels of 8-bit matrices share: the step of a row, its
// codes, reductions of magnitudes, rows of a few vectors a thread.
#pragma once

#include "zo_ops_device.h"

namespace zo {

// Magnitudes are compared as the integers of their bits: their order, infinity and then
// NaN last.
constexpr uint32_t kMagMask = 0x7FFFFFFFu, kInfBits = 0x7F800000u;

__device__ __forceinline__ uint32_t mag_bits(float v) { return __float_as_uint(v) & kMagMask; }

// The largest of a wave's values, in every lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    auto step = [](uint32_t a, int o) { return max(a, (uint32_t)o); };
    v = step(v, __builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, false));  // as wave_reduce
    v = step(v, __builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, false));
    v = step(v, __builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, false));
    v = step(v, __builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, false));
    v = step(v, __builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xA, 0xF, false));
    v = step(v, __builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xC, 0xF, false));
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// v in binary32: the compiler would else form a product and its rounding to binary16 in
// one instruction, rounded once, in some kernels and not in others.
template <int GT>
__device__ __forceinline__ float as_binary32(float v)
{
    if constexpr (GT == GT_F16) asm volatile("" : "+v"(v));
    return v;
}

// Over the TH threads of a row (a wave, or the whole workgroup; then s holds a value of
// each wave and there is one barrier).  The result in every lane.
template <int TH>
__device__ __forceinline__ float row_sum(float v, float *s)
{
    v = wave_reduce<OpSum>(v);
    if constexpr (TH == 64) {
        return v;
    } else {
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
        __syncthreads();
        return group_get<OpSum, TH / 64>(s);
    }
}

template <int TH>
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t *s)
{
    v = wave_max(v);
    if constexpr (TH == 64) {
        return v;
    } else {
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
        __syncthreads();
        uint32_t r = s[0];
#pragma unroll
        for (int i = 1; i < TH / 64; ++i) r = max(r, s[i]);
        return (uint32_t)__builtin_amdgcn_readfirstlane((int)r);
    }
}

// A row's step s = a / 127 (a: its largest magnitude, as bits), and how codes x / s are
// formed: as x times the rounded inverse, which is within 2^-16 of the quotient, or,
// where that is next to the border of two codes, by a division in 64 bits.  A quotient of
// two 24-bit numbers that is not such a border itself is at least 2^-33 of it away, so the
// rounded 64-bit quotient stands on the same side.  Steps below 2^-100, whose inverse may
// pass binary32, take the division throughout.  inv = 0 makes every code 0, those of NaN
// and infinity too.
struct Step {
    float s, inv;
    bool far;
};

__device__ __forceinline__ Step step_of(uint32_t a)
{
    Step t;
    t.s = a >= kInfBits ? NAN : __uint_as_float(a) / 127.0f;
    t.far = t.s < 0x1p-100f && t.s > 0.0f;
    t.inv = t.s >= 0x1p-100f ? 1.0f / t.s : 0.0f;
    return t;
}

__device__ __forceinline__ Step step_from(float s)
{
    return {s, s >= 0x1p-100f ? 1.0f / s : 0.0f, s < 0x1p-100f && s > 0.0f};
}

__device__ __forceinline__ int exact_code(float x, float s)
{
    const double q = __builtin_rint((double)x / (double)s);
    return (int)fmin(fmax(q, -127.0), 127.0);
}

// Whether a quotient is within 2^-13 of a border.
__device__ __forceinline__ bool near_border(float r, float rounded)
{
    return fabsf(r - rounded) > 0.5f - 0x1p-13f;
}

// The codes of four values in a dword, the first lowest.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, const Step &t)
{
    const float x[4] = {a, b, c, d};
    uint32_t w = 0;
    bool hard = t.far;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float r = x[q] * t.inv, f = __builtin_rintf(r);
        hard |= near_border(r, f);
        w |= ((uint32_t)(int)f & 255u) << (8 * q);
    }
    if (hard) {
        w = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) w |= ((uint32_t)exact_code(x[q], t.s) & 255u) << (8 * q);
    }
    return w;
}

// The codes of a vector's elements, at p (kVec bytes, aligned to them).
template <int K>
__device__ __forceinline__ void store_codes(int8_t *p, const float (&x)[K], const Step &t)
{
    const uint32_t lo = codes4(x[0], x[1], x[2], x[3], t);
    if constexpr (K == 8)
        *reinterpret_cast<u32x2 *>(p) = u32x2{lo, codes4(x[4], x[5], x[6], x[7], t)};
    else
        *reinterpret_cast<uint32_t *>(p) = lo;
}

// Largest magnitudes of packed elements, element by element, in their own type.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

template <int GT>
__device__ __forceinline__ uint32_t packed_max(uint32_t a, uint32_t w)
{
    if constexpr (GT == GT_F32)
        return max(a, w & kMagMask);
    else
        return __builtin_bit_cast(
            uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a),
                                                __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu)));
}

// Bits, in binary32, of the largest magnitude within the packed maxima w.
template <int GT>
__device__ __forceinline__ uint32_t max_in(const u32x4 &w)
{
    uint32_t a = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) a = packed_max<GT>(a, w[q]);
    if constexpr (GT != GT_F32) a = max(a & 0xFFFFu, a >> 16);
    return mag_bits(widen<GT>((typename Elem<GT>::T)a));
}

}  // namespace zo
