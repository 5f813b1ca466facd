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
// formed: from x times an inverse a little above that of s and one a little below it.  Where
// both round to the same whole number the quotient, which lies between, does too; where not,
// it is near the border of two codes, and a division in 64 bits decides: a quotient of two
// 24-bit numbers that is not such a border itself is at least 2^-33 of it away, so the rounded
// 64-bit quotient stands on the same side.  That is one element in 2^16 of normal values in
// binary32, 2^11 in binary16 and 2^9 in bfloat16, whose numbers often are half multiples of s (then
// in 29% of a wave's groups of four: 8192 x 1600 by rows 11.4 us, with a few large columns that
// make the other codes small 9.1).  Steps below 2^-100, whose inverse may pass
// binary32, take the division throughout.  Where both inverses are 0 all codes are 0.
struct Step {
    float s, above, below;
    bool far;
};

__device__ __forceinline__ Step step_from(float s)
{
    // the instruction is within 2^-23
    const float inv = s >= 0x1p-100f ? __builtin_amdgcn_rcpf(s) : 0.0f;
    return {s, inv * (1.0f + 0x1p-22f), inv * (1.0f - 0x1p-22f), s < 0x1p-100f && s > 0.0f};
}

__device__ __forceinline__ Step step_of(uint32_t a)
{
    // a / 127 rounded to nearest: the quotient by the rounded inverse of 127, then its
    // remainder, which is exact, by it again; a division where the quotient is near the
    // numbers below the normal ones
    constexpr float kInverse = 1.0f / 127.0f;
    const float x = __uint_as_float(a), q = x * kInverse;
    float s = __builtin_fmaf(__builtin_fmaf(-127.0f, q, x), kInverse, q);
    if (a < 0x0E000000u) s = x / 127.0f;        // 2^-99
    return step_from(a >= kInfBits ? NAN : s);
}

__device__ __forceinline__ int exact_code(float x, float s)
{
    const double q = __builtin_rint((double)x / (double)s);
    return (int)fmin(fmax(q, -127.0), 127.0);
}

// The last bytes of x inv + 1.5 * 2^23, which rounds x inv to a whole number, to nearest even.
__device__ __forceinline__ uint32_t rounded4(const float (&x)[4], float inv)
{
    uint32_t n[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) n[q] = __float_as_uint(__builtin_fmaf(x[q], inv, 0x1.8p23f));
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(n[3], n[2], 0x0C0C0400u),
                                 __builtin_amdgcn_perm(n[1], n[0], 0x0C0C0400u), 0x05040100u);
}

// The codes of four values in a dword, the first lowest.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, const Step &t)
{
    const float x[4] = {a, b, c, d};
    uint32_t w = rounded4(x, t.above);
    if (w != rounded4(x, t.below) || t.far) {
        w = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) w |= ((uint32_t)exact_code(x[q], t.s) & 255u) << (8 * q);
    }
    return t.above == 0.0f && !t.far ? 0u : w;
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

// Thread t's vectors t, t + TH, ... of a row of `cols` elements; what is not there is 0, or
// not stored.  Whole vectors first, so that all their loads are under way together.
template <int GT, int TH, int NV>
__device__ __forceinline__ void load_row(u32x4 (&w)[NV], const typename Elem<GT>::T *p, int cols,
                                         int t)
{
    constexpr int K = Elem<GT>::kVec;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * TH + t) * K;
        w[v] = u32x4{0, 0, 0, 0};
        if (c + K <= cols) w[v] = *reinterpret_cast<const u32x4_a2 *>(p + c);
    }
    if (cols % K)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * TH + t) * K;
            if (c < cols && c + K > cols) w[v] = load16<GT>(p + c, cols - c);
        }
}

// Stores vector v of the row.
template <int GT>
__device__ __forceinline__ void store_vector(typename Elem<GT>::T *p, const u32x4 &w, int c,
                                             int cols)
{
    constexpr int K = Elem<GT>::kVec;
    if (c + K <= cols)
        *reinterpret_cast<u32x4_a2 *>(p + c) = w;
    else if (c < cols)
        store16<GT>(p + c, w, cols - c);
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
