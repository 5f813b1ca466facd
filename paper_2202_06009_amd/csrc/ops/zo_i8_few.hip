// zo_i8_few.hip -- products of a few rows (a decode step) by an 8-bit matrix.
//
// The bound is reading the matrix once, a byte an element.  A wave takes 16 of its rows and
// streams 64 columns of them in one access, 16 bytes a lane; the instruction is the 16 x 16 x
// 64 one, lane l holding row l % 16, elements 16 (l / 16) .. + 15, and of its four results
// lane l holds, for row l % 16 of the activations, columns 4 (l / 16) + 0..3.  Where the
// matrix has too few rows to occupy the GPU, the KS waves of a group share them, each a run
// of the columns, and their sums, which are exact, are joined through shared memory.
//
// Up to 16 rows of activations, where they are short (i8_few_fused), are quantised by every
// workgroup for itself (FUSED): no second kernel, nothing written and read back.
#include "zo_i8_device.h"

namespace zo {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 8, kAhead = 8;
// Bytes of quantised activations in shared memory, beside the joined sums.
constexpr int64_t kFusedBytes = 49152;

__device__ __forceinline__ i32x4 mfma16_i8(const u32x4 &a, const u32x4 &b, i32x4 acc)
{
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a),
                                                 __builtin_bit_cast(i32x4, b), acc, 0, 0, 0);
}

// The rows of activations in the operand's order, codes[64 columns][16 bytes of columns][row],
// and their scales: a row a wave at a time, read twice (the second time from the caches).
// Rows that are not there stay what they were: they reach no result.
template <int GX>
__device__ __forceinline__ void quantize_rows(const typename Elem<GX>::T *x, int rows,
                                              int64_t cols, int64_t ldx, int wide, int8_t *codes,
                                              float *scales)
{
    constexpr int V = Elem<GX>::kVec;
    const int lane = threadIdx.x & 63;
    for (int r = threadIdx.x >> 6; r < rows; r += kWaves) {
        const typename Elem<GX>::T *p = x + r * ldx;
        u32x4 m = {};
#pragma unroll 4
        for (int c = lane * V; c < cols; c += 64 * V) {
            const u32x4 w = load16<GX>(p + c, cols - c);
#pragma unroll
            for (int i = 0; i < 4; ++i) m[i] = packed_max<GX>(m[i], w[i]);
        }
        const Step s = step_of(wave_max(max_in<GX>(m)));
        if (lane == 0) scales[r] = s.s;
#pragma unroll 4
        for (int c = lane * V; c < wide; c += 64 * V) {
            u32x4 w = {0, 0, 0, 0};
            if (c < cols) w = load16<GX>(p + c, cols - c);
            float e[V];
#pragma unroll
            for (int i = 0; i < V; ++i) e[i] = elem_of<GX>(w, i);
            store_codes<V>(codes + (c / 16 * 16 + r) * 16 + c % 16, e, s);
        }
    }
}

// MB tiles of 16 rows of a by b.  A workgroup of 8 waves takes 8 / KS tiles of 16 rows of
// b.  FUSED: a is x, quantised here.
template <int GX, int GT, int MB, int KS, bool FUSED>
__global__ __launch_bounds__(kWaves * 64) void k_i8_few(
    I8View a, const typename Elem<GX>::T *__restrict__ x, int64_t ldx, I8View b,
    typename Elem<GT>::T *__restrict__ out, int64_t ld)
{
    extern __shared__ u32x4 lds[];       // the sums; FUSED: codes, scales
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int part = wave % KS;
    const int64_t tile = (int64_t)blockIdx.x * (kWaves / KS) + wave / KS;   // of 16 rows of b
    const int steps = (int)(b.wide / 64);
    i32x4 *sums = reinterpret_cast<i32x4 *>(lds);
    u32x4 *codes = lds + (KS > 1 ? MB * kWaves * 64 : 0);
    float *scales = reinterpret_cast<float *>(codes + (FUSED ? steps * 64 : 0));
    const bool there = tile * 16 < b.rows;
    const int from = steps * part / KS, to = there ? steps * (part + 1) / KS : from;
    // rows beyond the last stand for it; what is computed from them is not stored
    const int8_t *pb = b.codes + min(tile * 16 + (lane & 15), b.rows - 1) * b.wide + (lane >> 4) * 16;
    const int8_t *pa[MB];
    if constexpr (!FUSED)
#pragma unroll
        for (int i = 0; i < MB; ++i)
            pa[i] = a.codes + min((int64_t)(i * 16 + (lane & 15)), a.rows - 1) * a.wide + (lane >> 4) * 16;

    u32x4 w[kAhead];
    auto fetch = [&](int t0) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (t0 + u < to) w[u] = *reinterpret_cast<const u32x4 *>(pb + (int64_t)(t0 + u) * 64);
    };
    fetch(from);                         // in flight while x is quantised
    if constexpr (FUSED) {
        quantize_rows<GX>(x, (int)a.rows, a.cols, ldx, (int)b.wide,
                          reinterpret_cast<int8_t *>(codes), scales);
        __syncthreads();
    }
    i32x4 acc[MB] = {};
    for (int t0 = from; t0 < to; t0 += kAhead) {
        if (t0 > from) fetch(t0);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (t0 + u >= to) break;
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                const u32x4 f = FUSED ? codes[(t0 + u) * 64 + lane]
                                      : *reinterpret_cast<const u32x4 *>(pa[i] + (t0 + u) * 64);
                acc[i] = mfma16_i8(w[u], f, acc[i]);
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
            for (int p = 1; p < KS; ++p) acc[i] += sums[(i * kWaves + wave + p) * 64 + lane];
    }
    const int64_t n = tile * 16 + (lane >> 4) * 4;
    if (n >= b.rows) return;
    f32x4 sb;
#pragma unroll
    for (int q = 0; q < 4; ++q) sb[q] = steps > 0 ? b.scales[min(n + q, b.rows - 1)] : 0.0f;
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        const int64_t m = i * 16 + (lane & 15);
        if (m >= a.rows) continue;
        const float sa = steps == 0 ? 0.0f : FUSED ? scales[m] : a.scales[m];
        f32x4 v;
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = as_binary32<GT>((float)acc[i][q] * sa * sb[q]);
        store_few<GT>(out + m * ld + n, v, b.rows - n);
    }
}

// Waves that share 16 rows: enough that about two waves a SIMD are there, each with four
// steps or more.
static int split_of(int64_t tiles, int64_t steps)
{
    int ks = 1;
    while (ks < kWaves && tiles * ks < 2048 && steps >= 8 * ks) ks *= 2;
    return ks;
}

static int64_t few_groups(int64_t tiles, int ks)
{
    return (tiles + kWaves / ks - 1) / (kWaves / ks);
}

static int64_t steps_of(int64_t k) { return (k + 127) / 128 * 2; }

bool i8_few_fits(int64_t n, int64_t k)
{
    const int64_t tiles = (n + 15) / 16;
    return fits_a_launch(few_groups(tiles, split_of(tiles, steps_of(k))), kWaves * 64);
}

template <int GX, int GT, int MB, bool FUSED>
static hipError_t launch_split(const I8View &a, const void *x, int64_t ldx, const I8View &b,
                               void *out, int64_t ld, hipStream_t st)
{
    const int64_t tiles = (b.rows + 15) / 16;
    const int ks = split_of(tiles, b.wide / 64);
    const uint32_t lds = (FUSED ? (uint32_t)b.wide * 16 + 64 : 0) + (ks > 1 ? MB * kWaves * 1024 : 0);
    const auto *px = static_cast<const typename Elem<GX>::T *>(x);
    auto *po = static_cast<typename Elem<GT>::T *>(out);
    const auto kernel = ks == 1   ? k_i8_few<GX, GT, MB, 1, FUSED>
                        : ks == 2 ? k_i8_few<GX, GT, MB, 2, FUSED>
                        : ks == 4 ? k_i8_few<GX, GT, MB, 4, FUSED>
                                  : k_i8_few<GX, GT, MB, 8, FUSED>;
    return start(kernel, few_groups(tiles, ks), kWaves * 64, lds, st, a, px, ldx, b, po, ld);
}

hipError_t launch_i8_few(const I8View &a, const I8View &b, void *out, int gt, int64_t ld,
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

// Every workgroup quantises all of x: for few and short rows.
bool i8_few_fused(int64_t rows, int64_t n, int64_t k)
{
    (void)n;
    const int64_t wide = (k + 127) / 128 * 128;
    return rows <= 16 && wide * 16 <= kFusedBytes && rows * wide <= 16384;
}

hipError_t launch_i8_few_fused(const void *x, int gx, int64_t rows, int64_t cols, int64_t ldx,
                               const I8View &b, void *out, int gt, int64_t ld, hipStream_t st)
{
    const I8View a = {nullptr, nullptr, rows, cols, b.wide};
    return with_elem_type(gx, [&](auto f) {
        return with_elem_type(gt, [&](auto g) {
            return launch_split<decltype(f)::value, decltype(g)::value, 1, true>(a, x, ldx, b, out,
                                                                                 ld, st);
        });
    });
}

}  // namespace zo
