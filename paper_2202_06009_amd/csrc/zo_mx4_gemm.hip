// zo_mx4_gemm.hip -- products of microscaled 4-bit matrices on the scaled
// matrix instruction (16 x 16 x 128, E2M1 operands, binary32 accumulators).
//
// Operand layout of the instruction: lane l holds row l % 16, elements
// 32 (l / 16) .. + 31 of the 128 (16 bytes) and their scale byte, one of the
// four bytes of a register.  The storage order of an mx4 matrix (zo_ops.h) is
// that: a tile of 16 rows x 128 columns is the 1 KiB that a wave loads with
// one 16-byte access per lane, and the scale dword of a lane serves four such
// tiles, rows 0..63 of a group.
//
// With b's rows as the first operand, lane l's four results are columns
// n = 4 (l / 16) .. + 3 of row m = l % 16 of the output.
#include "zo_ops_device.h"

namespace zo {

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

// Calls f(integral_constant<0>) .. f(integral_constant<N - 1>).
template <int N, class F>
__device__ __forceinline__ void unroll(F &&f)
{
    if constexpr (N > 0) {
        unroll<N - 1>(f);
        f(std::integral_constant<int, N - 1>{});
    }
}

// Four consecutive results of a row, of which nv are inside it.
template <int GT>
__device__ __forceinline__ void store4(typename Elem<GT>::T *p, f32x4 v, int64_t nv)
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
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (q < nv) p[q] = narrow<GT>(v[q]);
    }
}

// 128 x 128 outputs per workgroup, 64 x 64 per wave, operands straight from
// memory.
template <int GT>
__global__ __launch_bounds__(256) void k_mx4_product(Mx4View a, Mx4View b,
                                                     typename Elem<GT>::T *__restrict__ out,
                                                     int64_t ld, uint32_t n_tiles)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t m0 = (int64_t)(blockIdx.x / n_tiles) * 128 + (wave >> 1) * 64;
    const int64_t n0 = (int64_t)(blockIdx.x % n_tiles) * 128 + (wave & 1) * 64;
    // a wave may lie wholly beyond the edge: the storage ends with its group of 64
    if (m0 >= a.rows || n0 >= b.rows) return;
    const uint8_t *pa = a.codes + m0 / 16 * a.kt * 1024 + lane * 16;
    const uint8_t *pb = b.codes + n0 / 16 * b.kt * 1024 + lane * 16;
    const uint8_t *sa = a.scales + m0 / 64 * a.kt * 256 + lane * 4;
    const uint8_t *sb = b.scales + n0 / 64 * b.kt * 256 + lane * 4;
    f32x4 acc[4][4] = {};
    for (int64_t t = 0; t < a.kt; ++t) {
        u32x4 x[4], w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = *reinterpret_cast<const u32x4 *>(pa + (i * a.kt + t) * 1024);
            w[i] = *reinterpret_cast<const u32x4 *>(pb + (i * b.kt + t) * 1024);
        }
        const uint32_t ea = *reinterpret_cast<const uint32_t *>(sa + t * 256);
        const uint32_t eb = *reinterpret_cast<const uint32_t *>(sb + t * 256);
        unroll<4>([&](auto i) {
            unroll<4>([&](auto j) {
                acc[i][j] = mfma<decltype(j)::value, decltype(i)::value>(w[j], x[i], acc[i][j],
                                                                         eb, ea);
            });
        });
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t m = m0 + i * 16 + (lane & 15);
        if (m >= a.rows) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t n = n0 + j * 16 + (lane >> 4) * 4;
            store4<GT>(out + m * ld + n, acc[i][j], b.rows - n);
        }
    }
}

hipError_t launch_mx4_product(const Mx4View &a, const Mx4View &b, void *out, int gt, int64_t ld,
                              hipStream_t st)
{
    if (a.rows == 0 || b.rows == 0) return hipSuccess;
    const int64_t nt = (b.rows + 127) / 128, tiles = (a.rows + 127) / 128 * nt;
    if (tiles > INT32_MAX) return hipErrorInvalidValue;
    return with_elem_type(gt, [&](auto g) {
        constexpr int GT = decltype(g)::value;
        k_mx4_product<GT><<<dim3((uint32_t)tiles), 256, 0, st>>>(
            a, b, static_cast<typename Elem<GT>::T *>(out), ld, (uint32_t)nt);
        return hipGetLastError();
    });
}

}  // namespace zo
