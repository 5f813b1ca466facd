// zo_i8_gemm.hip -- products of 8-bit matrices on the integer matrix instruction
// (32 x 32 x 32, 32-bit accumulators).
//
// Operand layout of the instruction: lane l holds row l % 32, elements 16 (l / 32) .. + 15
// of the 32 (16 bytes).  With b's rows as the first operand, a lane's sixteen results are
// runs of four columns of one row of the output: columns 8 q + 4 (l / 32) + 0..3 at 4 q.
#include "zo_i8_device.h"
#include "zo_tile_device.h"

namespace zo {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ i32x16 mfma_i8(const u32x4 &a, const u32x4 &b, i32x16 acc)
{
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a),
                                                 __builtin_bit_cast(i32x4, b), acc, 0, 0, 0);
}

// 16 bytes a lane from memory into shared memory, lane after lane from `to` on.
__device__ __forceinline__ void load_lds(const int8_t *from, u32x4 *to)
{
    __builtin_amdgcn_global_load_lds(
        reinterpret_cast<const __attribute__((address_space(1))) uint32_t *>(
            reinterpret_cast<uintptr_t>(from)),
        (__attribute__((address_space(3))) uint32_t *)to, 16, 0, 0);
}

// 32 MF WR x 32 NF WC outputs per workgroup of WR x WC waves, 32 MF x 32 NF a wave.  A step
// multiplies 128 columns of both operands out of shared memory while the next step's are
// loaded straight into a second buffer.  A row's eight chunks of 16 bytes stand at
// c ^ (row % 8), so that the 32 rows of a fragment read all banks alike: the loads place
// chunk after chunk, so a lane fetches the chunk that belongs in its place.
template <int GT, int MF, int NF, int WR, int WC, bool STREAM>
__global__ __launch_bounds__(64 * WR * WC) void k_i8_product(
    I8View a, I8View b, typename Elem<GT>::T *__restrict__ out, int64_t ld, uint32_t m_tiles,
    uint32_t n_tiles)
{
    constexpr int WAVES = WR * WC, BM = 32 * MF * WR, BN = 32 * NF * WC, ROWS = BM + BN;
    constexpr int MINE = ROWS / 8 / WAVES;           // loads of 8 rows a wave and step
    static_assert(ROWS % (8 * WAVES) == 0, "whole loads for every wave");
    __shared__ u32x4 buf0[ROWS * 8], buf1[ROWS * 8];
    const TileIndex tile = tile_index(run_index(blockIdx.x, m_tiles * n_tiles), m_tiles, n_tiles);
    const int64_t m0 = (int64_t)tile.m * BM, n0 = (int64_t)tile.n * BN;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WC, wn = wave % WC;
    const int steps = (int)(a.wide / 128);

    const int8_t *src[MINE];
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
        const int r = (i * WAVES + wave) * 8 + lane / 8;
        const int chunk = (lane & 7) ^ (r & 7);
        src[i] = r < BM ? a.codes + min(m0 + r, a.rows - 1) * a.wide + chunk * 16
                        : b.codes + min(n0 + (r - BM), b.rows - 1) * b.wide + chunk * 16;
    }
    auto fetch = [&](u32x4 *to) {
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            load_lds(src[i], to + (i * WAVES + wave) * 64);
            src[i] += 128;
        }
    };
    const int row_a = (wm * 32 * MF + (lane & 31)) * 8, row_b = (BM + wn * 32 * NF + (lane & 31)) * 8;
    i32x16 acc[MF][NF] = {};
    auto multiply = [&](const u32x4 *from) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int c = (2 * k + (lane >> 5)) ^ (lane & 7);
            u32x4 fa[MF], fb[NF];
#pragma unroll
            for (int i = 0; i < MF; ++i) fa[i] = from[row_a + i * 256 + c];
#pragma unroll
            for (int j = 0; j < NF; ++j) fb[j] = from[row_b + j * 256 + c];
#pragma unroll
            for (int i = 0; i < MF; ++i)
#pragma unroll
                for (int j = 0; j < NF; ++j) acc[i][j] = mfma_i8(fb[j], fa[i], acc[i][j]);
        }
    };
    if (steps > 0) {
        fetch(buf0);
        __syncthreads();
        int t = 0;
        for (; t + 2 <= steps; t += 2) {
            fetch(buf1);
            multiply(buf0);
            __syncthreads();
            if (t + 2 < steps) fetch(buf0);
            multiply(buf1);
            __syncthreads();
        }
        if (t < steps) {
            multiply(buf0);
            __syncthreads();
        }
    }

    static_assert(ROWS * 8 >= WAVES * NF * 256, "room for 32 binary32 rows of every wave");
    u32x4 *mine = buf0 + wave * (NF * 256);
    const int64_t mw = m0 + wm * 32 * MF, nw = n0 + wn * 32 * NF;
    f32x4 sb[NF][4];
#pragma unroll
    for (int j = 0; j < NF; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t n = nw + j * 32 + q * 8 + (lane >> 5) * 4 + e;
                sb[j][q][e] = steps > 0 ? b.scales[min(n, b.rows - 1)] : 0.0f;
            }
#pragma unroll
    for (int i = 0; i < MF; ++i) {
        const int64_t m = mw + i * 32 + (lane & 31);
        const float sa = steps > 0 ? a.scales[min(m, a.rows - 1)] : 0.0f;
        f32x16 v[NF];
#pragma unroll
        for (int j = 0; j < NF; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                v[j][e] = as_binary32<GT>((float)acc[i][j][e] * sa * sb[j][e / 4][e % 4]);
        store_rows<GT, STREAM>(out + (mw + i * 32) * ld + nw, ld, a.rows - mw - i * 32,
                               b.rows - nw, v, mine);
        __builtin_amdgcn_sched_barrier(0);
    }
}

template <int GT, int MF, int NF, int WR, int WC>
static hipError_t launch_tiles(const I8View &a, const I8View &b, void *out, int64_t ld,
                               hipStream_t st)
{
    constexpr int BM = 32 * MF * WR, BN = 32 * NF * WC;
    const int64_t mt = (a.rows + BM - 1) / BM, nt = (b.rows + BN - 1) / BN;
    const auto kernel = streamed<GT>(out, ld) ? k_i8_product<GT, MF, NF, WR, WC, true>
                                              : k_i8_product<GT, MF, NF, WR, WC, false>;
    return start(kernel, mt * nt, 64 * WR * WC, 0, st, a, b,
                 static_cast<typename Elem<GT>::T *>(out), ld, (uint32_t)mt, (uint32_t)nt);
}

enum class Form { kFew, kLarge, kMiddle, kSmall };

static int64_t tiles_of(int64_t m, int64_t n, int64_t tile_m, int64_t tile_n)
{
    return (m + tile_m - 1) / tile_m * ((n + tile_n - 1) / tile_n);
}

static Form form_of(int64_t m, int64_t n)
{
    if (m <= kI8FewRows) return Form::kFew;
    if (tiles_of(m, n, 256, 256) >= 192) return Form::kLarge;
    return tiles_of(m, n, 128, 128) >= 192 ? Form::kMiddle : Form::kSmall;
}

bool i8_product_fits(int64_t m, int64_t n, int64_t k)
{
    if (m == 0 || n == 0) return true;
    switch (form_of(m, n)) {
    case Form::kFew: return i8_few_fits(n, k);
    case Form::kLarge: return fits_a_launch(tiles_of(m, n, 256, 256), 512);
    case Form::kMiddle: return fits_a_launch(tiles_of(m, n, 128, 128), 256);
    default: return fits_a_launch(tiles_of(m, n, 64, 64), 256);
    }
}

hipError_t launch_i8_product(const I8View &a, const I8View &b, void *out, int gt, int64_t ld,
                             hipStream_t st)
{
    if (a.rows == 0 || b.rows == 0) return hipSuccess;
    const Form form = form_of(a.rows, b.rows);
    if (form == Form::kFew) return launch_i8_few(a, b, out, gt, ld, st);
    return with_elem_type(gt, [&](auto g) {
        constexpr int GT = decltype(g)::value;
        switch (form) {
        case Form::kLarge: return launch_tiles<GT, 4, 2, 2, 4>(a, b, out, ld, st);
        case Form::kMiddle: return launch_tiles<GT, 2, 2, 2, 2>(a, b, out, ld, st);
        default: return launch_tiles<GT, 1, 1, 2, 2>(a, b, out, ld, st);
        }
    });
}

}  // namespace zo
