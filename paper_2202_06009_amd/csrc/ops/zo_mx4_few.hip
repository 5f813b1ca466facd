// zo_mx4_few.hip -- products of a few rows (a decode step) by a 4-bit matrix.
//
// The bound is reading the matrix once: 17/32 bytes an element (1 x 50257 x 1600 9.4 us,
// 4.6 TB/s; 11 rows 11.4 us, their quantisation before the stream).  A wave takes 16
// of its rows, 1 KiB a tile of 128 columns in one access per lane, and keeps
// eight tiles in flight; where the matrix has too few rows to occupy the GPU, the
// KS waves of a group share them, each a run of the tiles, and their sums are
// joined in a fixed order through shared memory.
//
// Up to 16 rows of activations, where they are few tiles (few_fused), are quantised by
// every workgroup for itself (FUSED): no second kernel, nothing written and read back.
#include "zo_mx4_device.h"

namespace zo {

constexpr int kWaves = 8, kAhead = 8;
// Tiles of 128 columns of quantised activations in shared memory: their codes and
// scale bytes beside the joined sums stay within 64 KiB.
constexpr int kFusedTiles = 52;

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

// The rows x (128 kt) activations in the operand's order: codes[t][lane], and a
// scale byte for each.  One block of 32 per thread and turn; columns that are not there
// are zeros, rows that are not there stay what they were: they reach no result.
template <int GX>
__device__ __forceinline__ void quantize_rows(const typename Elem<GX>::T *x, int rows,
                                              int64_t cols, int64_t ldx, int kt, u32x4 *codes,
                                              uint8_t *scales)
{
    constexpr int V = Elem<GX>::kVec, D = 32 / V;      // accesses of a block
#pragma unroll 2
    for (int b = threadIdx.x; b < kt * 4 * rows; b += kWaves * 64) {
        const int r = b % rows, k = b / rows, i = k * 16 + r;   // i = tile * 64 + lane
        const int64_t col = (int64_t)k * 32;
        u32x4 w[D];
        uint32_t a = 0;
#pragma unroll
        for (int d = 0; d < D; ++d) {
            w[d] = load16<GX>(x + r * ldx + col + d * V, cols - col - d * V);
#pragma unroll
            for (int q = 0; q < 4; ++q) a = mag<GX>(a, w[d][q]);
        }
        if constexpr (GX != GT_F32) a = max(a & 0xFFFFu, a >> 16);
        const uint32_t e = scale_byte<GX>(a);
        const float s = __uint_as_float(e << 23);
        u32x4 c;
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            uint32_t o = 0;
            if constexpr (GX == GT_F32) {
                o = convert2<GX, 0>(o, w[2 * d][0], w[2 * d][1], s);
                o = convert2<GX, 1>(o, w[2 * d][2], w[2 * d][3], s);
                o = convert2<GX, 2>(o, w[2 * d + 1][0], w[2 * d + 1][1], s);
                o = convert2<GX, 3>(o, w[2 * d + 1][2], w[2 * d + 1][3], s);
            } else {
                o = convert2<GX, 0>(o, w[d][0], 0, s);
                o = convert2<GX, 1>(o, w[d][1], 0, s);
                o = convert2<GX, 2>(o, w[d][2], 0, s);
                o = convert2<GX, 3>(o, w[d][3], 0, s);
            }
            c[d] = e == 255 ? 0 : o;
        }
        codes[i] = c;
        scales[i] = (uint8_t)e;
    }
}

// MB tiles of 16 rows of a by b.  A workgroup of 8 waves takes 8 / KS tiles of 16
// rows of b.  FUSED: a is x, quantised here.
template <int GX, int GT, int MB, int KS, bool FUSED>
__global__ __launch_bounds__(kWaves * 64) void k_mx4_few(
    Mx4View a, const typename Elem<GX>::T *__restrict__ x, int64_t ldx, Mx4View b,
    typename Elem<GT>::T *__restrict__ out, int64_t ld)
{
    extern __shared__ u32x4 lds[];       // FUSED: codes, scale bytes; then the sums
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int part = wave % KS;
    const int64_t tile = (int64_t)blockIdx.x * (kWaves / KS) + wave / KS;   // of 16 rows of b
    const int kt = (int)b.kt;
    u32x4 *codes = lds;
    uint8_t *scales = reinterpret_cast<uint8_t *>(lds + (FUSED ? kt * 64 : 0));
    f32x4 *sums = reinterpret_cast<f32x4 *>(scales + (FUSED ? kt * 64 : 0));
    const bool there = tile * 16 < b.rows;
    const int from = kt * part / KS, to = there ? kt * (part + 1) / KS : from;
    const uint8_t *wc = b.codes + (there ? tile : 0) * b.kt * 1024 + lane * 16;
    const uint8_t *ws = b.scales + (there ? tile / 4 : 0) * b.kt * 256 + lane * 4;
    const int shift = 8 * (int)(tile & 3);

    u32x4 w[kAhead];
    uint32_t e[kAhead];
    auto fetch = [&](int t0) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (t0 + u < to) {
                w[u] = *reinterpret_cast<const u32x4 *>(wc + (int64_t)(t0 + u) * 1024);
                e[u] = *reinterpret_cast<const uint32_t *>(ws + (int64_t)(t0 + u) * 256) >> shift;
            }
    };
    fetch(from);                         // in flight while x is quantised
    if constexpr (FUSED) {
        quantize_rows<GX>(x, (int)a.rows, a.cols, ldx, kt, codes, scales);
        __syncthreads();
    }
    f32x4 acc[MB] = {};
    for (int t0 = from; t0 < to; t0 += kAhead) {
        if (t0 > from) fetch(t0);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (t0 + u >= to) break;
            if constexpr (FUSED) {
                const int at = (t0 + u) * 64 + lane;
                acc[0] = mfma<0, 0>(w[u], codes[at], acc[0], e[u], scales[at]);
            } else {
                const uint32_t s =
                    *reinterpret_cast<const uint32_t *>(a.scales + (int64_t)(t0 + u) * 256 + lane * 4);
                const uint8_t *c = a.codes + (int64_t)(t0 + u) * 1024 + lane * 16;
                u32x4 f[MB];
#pragma unroll
                for (int i = 0; i < MB; ++i)
                    f[i] = *reinterpret_cast<const u32x4 *>(c + i * a.kt * 1024);
                acc[0] = mfma<0, 0>(w[u], f[0], acc[0], e[u], s);
                if constexpr (MB > 1) acc[1] = mfma<0, 1>(w[u], f[1], acc[1], e[u], s);
                if constexpr (MB > 2) {
                    acc[2] = mfma<0, 2>(w[u], f[2], acc[2], e[u], s);
                    acc[3] = mfma<0, 3>(w[u], f[3], acc[3], e[u], s);
                }
            }
        }
    }
    if constexpr (KS > 1) {
#pragma unroll
        for (int i = 0; i < MB; ++i) sums[(i * kWaves + wave) * 64 + lane] = acc[i];
        __syncthreads();
        if (part != 0) return;
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int p = 1; p < KS; ++p) {
                const f32x4 o = sums[(i * kWaves + wave + p) * 64 + lane];
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[i][q] += o[q];
            }
    }
    const int64_t n = tile * 16 + (lane >> 4) * 4;
    if (n >= b.rows) return;
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        const int64_t m = i * 16 + (lane & 15);
        if (m < a.rows) store_few<GT>(out + m * ld + n, acc[i], b.rows - n);
    }
}

// Waves that share 16 rows: enough that about two waves a SIMD are there, each
// with two tiles or more.
static int split_of(int64_t tiles, int64_t kt)
{
    int ks = 1;
    while (ks < kWaves && tiles * ks < 2048 && kt >= 4 * ks) ks *= 2;
    return ks;
}

static int64_t few_groups(int64_t tiles, int ks)
{
    return (tiles + kWaves / ks - 1) / (kWaves / ks);
}

bool mx4_few_fits(int64_t n, int64_t k)
{
    const int64_t tiles = (n + 15) / 16;
    return fits_a_launch(few_groups(tiles, split_of(tiles, (k + 127) / 128)), kWaves * 64);
}

template <int GX, int GT, int MB, bool FUSED>
static hipError_t launch_split(const Mx4View &a, const void *x, int64_t ldx, const Mx4View &b,
                               void *out, int64_t ld, hipStream_t st)
{
    const int64_t tiles = (b.rows + 15) / 16;
    const int ks = split_of(tiles, b.kt);
    const uint32_t lds = (FUSED ? (uint32_t)b.kt * 64 * 17 : 0) + (ks > 1 ? MB * kWaves * 1024 : 0);
    const auto *px = static_cast<const typename Elem<GX>::T *>(x);
    auto *po = static_cast<typename Elem<GT>::T *>(out);
    const auto kernel = ks == 1   ? k_mx4_few<GX, GT, MB, 1, FUSED>
                        : ks == 2 ? k_mx4_few<GX, GT, MB, 2, FUSED>
                        : ks == 4 ? k_mx4_few<GX, GT, MB, 4, FUSED>
                                  : k_mx4_few<GX, GT, MB, 8, FUSED>;
    return start(kernel, few_groups(tiles, ks), kWaves * 64, lds, st, a, px, ldx, b, po, ld);
}

hipError_t launch_mx4_few(const Mx4View &a, const Mx4View &b, void *out, int gt, int64_t ld,
                          hipStream_t st)
{
    return with_elem_type(gt, [&](auto g) {
        constexpr int GT = decltype(g)::value;
        if (a.rows <= 16)
            return launch_split<GT_F32, GT, 1, false>(a, nullptr, 0, b, out, ld, st);
        if (a.rows <= 32)
            return launch_split<GT_F32, GT, 2, false>(a, nullptr, 0, b, out, ld, st);
        return launch_split<GT_F32, GT, 4, false>(a, nullptr, 0, b, out, ld, st);
    });
}

// Every workgroup quantises all of x, so with many tile rows a kernel of its own is
// faster, the sooner the more workgroups there are beside their work: where eight waves
// share 16 rows of the matrix and there are more workgroups than CUs, from 200 tile rows
// on, otherwise from 400.  Measured, one kernel / two, us (rows x matrix; tile rows):
//   8 x 6400 x 2560 (160) 5.7 / 6.6; 11 x 6400 x 2560 (220) 6.7 / 6.5; 8 x 6400 x 4096 (256)
//   8.6 / 8.4; 8 x 6400 x 6400 (400) 12.1 / 10.5
//   8 x 4096 x 6400 (400) 8.1 / 9.6; 16 x 4096 x 4096 (512) 7.6 / 7.0; 16 x 1600 x 6400 (800)
//   9.8 / 8.0; 16 x 25600 x 2560 (320) 12.0 / 12.3; 16 x 50257 x 1600 (208) 12.1 / 14.5;
//   1 x 6400 x 1600 (13) 4.1 / 6.6
bool few_fused(int64_t rows, int64_t n, int64_t k)
{
    const int64_t kt = (k + 127) / 128, tiles = (n + 15) / 16;
    const int ks = split_of(tiles, kt);
    const bool crowded = ks == kWaves && few_groups(tiles, ks) > 256;
    return rows <= 16 && kt <= kFusedTiles && rows * kt <= (crowded ? 200 : 400);
}

hipError_t launch_mx4_few_fused(const void *x, int gx, int64_t rows, int64_t cols, int64_t ldx,
                                const Mx4View &b, void *out, int gt, int64_t ld, hipStream_t st)
{
    const Mx4View a = {nullptr, nullptr, rows, cols, b.kt};
    return with_elem_type(gx, [&](auto f) {
        return with_elem_type(gt, [&](auto g) {
            return launch_split<decltype(f)::value, decltype(g)::value, 1, true>(a, x, ldx, b, out,
                                                                                 ld, st);
        });
    });
}

}  // namespace zo
