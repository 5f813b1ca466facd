// zo_i8_few.hip -- products of a few rows (a decode step) by an 8-bit matrix.
//
// The bound is reading the matrix once, a byte an element (1 x 50257 x 1600 16.3 us, 4.9 TB/s;
// 1 x 6400 x 1600 5.0 us, the launch and its latencies).  A wave takes 16 of its rows and
// streams 64 columns of them in one access, 16 bytes a lane; the instruction is the 16 x 16 x
// 64 one, lane l holding row l % 16, elements 16 (l / 16) .. + 15, and of its four results
// lane l holds, for row l % 16 of the activations, columns 4 (l / 16) + 0..3.  Where the
// matrix has too few rows to occupy the GPU, the KS waves of a group share them, each a run
// of the columns, and their sums, which are exact, are joined through shared memory.
//
// Up to 16 rows of activations, where they are short (i8_few_fused), are quantised by every
// workgroup for itself: no second kernel, nothing written and read back.
#include "zo_i8_device.h"

namespace zo {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 8, kAhead = 8;

__device__ __forceinline__ i32x4 mfma16_i8(const u32x4 &a, const u32x4 &b, i32x4 acc)
{
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a),
                                                 __builtin_bit_cast(i32x4, b), acc, 0, 0, 0);
}

// The rows of activations in shared memory, codes[16 columns][row][column], and their scales.
// The waves share a row where the rows are few; each keeps its first vectors of it in registers
// and reads the others twice.
template <int GX>
__device__ __forceinline__ void quantize_rows(const typename Elem<GX>::T *x, int rows, int cols,
                                              int64_t ldx, int wide, int8_t *codes, float *scales,
                                              uint32_t *tops)
{
    constexpr int V = Elem<GX>::kVec, HELD = 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int share = rows <= 1 ? 8 : rows <= 2 ? 4 : rows <= 4 ? 2 : 1;     // waves of a row
    const int part = wave % share, stride = share * 64 * V, first = (part * 64 + lane) * V;
    for (int r = wave / share; r < rows || share > 1; r += kWaves / share) {
        const typename Elem<GX>::T *p = x + min(r, rows - 1) * ldx;
        u32x4 held[HELD], m = {};
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int c = first + i * stride;
            held[i] = u32x4{0, 0, 0, 0};
            if (c < cols) held[i] = load16<GX>(p + c, cols - c);
        }
#pragma unroll
        for (int i = 0; i < HELD; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) m[q] = packed_max<GX>(m[q], held[i][q]);
        for (int c = first + HELD * stride; c < cols; c += stride) {
            const u32x4 w = load16<GX>(p + c, cols - c);
#pragma unroll
            for (int q = 0; q < 4; ++q) m[q] = packed_max<GX>(m[q], w[q]);
        }
        uint32_t top = wave_max(max_in<GX>(m));
        if (share > 1) {                        // the same for all
            if (lane == 0) tops[wave] = top;
            __syncthreads();
            for (int i = 0; i < share; ++i) top = max(top, tops[wave / share * share + i]);
        }
        const Step s = step_of(top);
        auto put = [&](const u32x4 &w, int c) __attribute__((always_inline)) {
            float e[V];
#pragma unroll
            for (int i = 0; i < V; ++i) e[i] = elem_of<GX>(w, i);
            store_codes<V>(codes + (c / 16 * rows + r) * 16 + c % 16, e, s);
        };
        if (r < rows) {
            if (part == 0 && lane == 0) scales[r] = s.s;
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                const int c = first + i * stride;
                if (c < wide) put(held[i], c);
            }
            for (int c = first + HELD * stride; c < wide; c += stride)
                put(c < cols ? load16<GX>(p + c, cols - c) : u32x4{0, 0, 0, 0}, c);
        }
        if (share > 1) break;                   // a row for every group of waves
    }
}

// Where the rows of a come from: their codes in memory, those copied into shared memory, or
// x, quantised here.
enum Source { kMemory, kCopied, kQuantised };

// MB tiles of 16 rows of a by b.  A workgroup of 8 waves takes 8 / KS tiles of 16 rows of
// b.
template <int GX, int GT, int MB, int KS, int FROM>
__global__ __launch_bounds__(kWaves * 64) void k_i8_few(
    I8View a, const typename Elem<GX>::T *__restrict__ x, int64_t ldx, I8View b,
    typename Elem<GT>::T *__restrict__ out, int64_t ld)
{
    extern __shared__ u32x4 lds[];       // the sums; codes, scales
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int part = wave % KS;
    const int64_t tile = (int64_t)blockIdx.x * (kWaves / KS) + wave / KS;   // of 16 rows of b
    const int steps = (int)(b.wide / 64), rows = (int)a.rows;
    i32x4 *sums = reinterpret_cast<i32x4 *>(lds);
    u32x4 *codes = lds + (KS > 1 ? MB * kWaves * 64 : 0);
    float *scales = reinterpret_cast<float *>(codes + (FROM == kQuantised ? steps * 4 * rows : 0));
    const bool there = tile * 16 < b.rows;
    const int from = steps * part / KS, to = there ? steps * (part + 1) / KS : from;
    // rows beyond the last stand for it; what is computed from them is not stored
    const int8_t *pb = b.codes + min(tile * 16 + (lane & 15), b.rows - 1) * b.wide + (lane >> 4) * 16;
    const int8_t *pa[MB];
    if constexpr (FROM == kMemory)
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
    const int64_t n = tile * 16 + (lane >> 4) * 4;
    f32x4 sb = {};
#pragma unroll
    for (int q = 0; q < 4; ++q)
        if (steps > 0) sb[q] = b.scales[min(n + q, b.rows - 1)];
    if constexpr (FROM == kQuantised) {
        quantize_rows<GX>(x, rows, (int)a.cols, ldx, (int)b.wide,
                          reinterpret_cast<int8_t *>(codes), scales,
                          reinterpret_cast<uint32_t *>(scales) + 16);
        __syncthreads();
    } else if constexpr (FROM == kCopied) {
        for (int r = wave; r < rows; r += kWaves)
#pragma unroll 4
            for (int c = lane; c < steps * 4; c += 64)
                codes[c * rows + r] = *reinterpret_cast<const u32x4 *>(a.codes + r * a.wide + c * 16);
        __syncthreads();
    }
    // a lane's place among the 16 columns' rows; lanes beyond the rows read the last one's
    int at[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) at[i] = (lane >> 4) * rows + min(i * 16 + (lane & 15), rows - 1);
    i32x4 acc[MB] = {};
    for (int t0 = from; t0 < to; t0 += kAhead) {
        if (t0 > from) fetch(t0);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (t0 + u >= to) break;
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                const u32x4 f = FROM != kMemory
                                    ? codes[(t0 + u) * 4 * rows + at[i]]
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
    if (n >= b.rows) return;
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        const int64_t m = i * 16 + (lane & 15);
        if (m >= a.rows) continue;
        const float sa = steps == 0 ? 0.0f : FROM == kQuantised ? scales[m] : a.scales[m];
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

template <int GX, int GT, int MB, int FROM>
static hipError_t launch_split(const I8View &a, const void *x, int64_t ldx, const I8View &b,
                               void *out, int64_t ld, hipStream_t st)
{
    const int64_t tiles = (b.rows + 15) / 16;
    const int ks = split_of(tiles, b.wide / 64);
    const uint32_t lds = (FROM != kMemory ? (uint32_t)(b.wide * a.rows) : 0) +
                         (FROM == kQuantised ? 128 : 0) + (ks > 1 ? MB * kWaves * 1024 : 0);
    const auto *px = static_cast<const typename Elem<GX>::T *>(x);
    auto *po = static_cast<typename Elem<GT>::T *>(out);
    const auto kernel = ks == 1   ? k_i8_few<GX, GT, MB, 1, FROM>
                        : ks == 2 ? k_i8_few<GX, GT, MB, 2, FROM>
                        : ks == 4 ? k_i8_few<GX, GT, MB, 4, FROM>
                                  : k_i8_few<GX, GT, MB, 8, FROM>;
    const hipError_t e = allow_lds(reinterpret_cast<const void *>(kernel), lds);
    if (e != hipSuccess) return e;
    return start(kernel, few_groups(tiles, ks), kWaves * 64, lds, st, a, px, ldx, b, po, ld);
}

// Codes that are copied into shared memory, beside the sums: a lane's 16 bytes of a row from
// memory for every tile of b are as many accesses as b's own (16 x 50257 x 1600 28.9 us, copied
// 17.8).
constexpr int64_t kCopiedBytes = 114688;

template <int GT, int MB>
static hipError_t launch_few(const I8View &a, const I8View &b, void *out, int64_t ld,
                             hipStream_t st)
{
    if (a.rows * a.wide <= kCopiedBytes)
        return launch_split<GT_F32, GT, MB, kCopied>(a, nullptr, 0, b, out, ld, st);
    return launch_split<GT_F32, GT, MB, kMemory>(a, nullptr, 0, b, out, ld, st);
}

hipError_t launch_i8_few(const I8View &a, const I8View &b, void *out, int gt, int64_t ld,
                         hipStream_t st)
{
    return with_elem_type(gt, [&](auto g) {
        constexpr int GT = decltype(g)::value;
        if (a.rows <= 16) return launch_few<GT, 1>(a, b, out, ld, st);
        return launch_few<GT, 2>(a, b, out, ld, st);
    });
}

// Every workgroup quantises all of x: for few and short rows.  One kernel / two, us (rows x
// matrix; KiB of codes): 1 x 6400 x 1600 (1.6) 5.0 / 6.9; 1 x 1600 x 6400 (6.3) 6.9 / 10.1; 8 x 6400
// x 1600 (13) 5.9 / 7.6; 4 x 1600 x 6400 (25) 9.2 / 10.7; 16 x 6400 x 1600 (26) 7.4 / 8.0; 8 x 4096 x
// 4096 (32) 9.7 / 9.2; 8 x 1600 x 6400 (50) 13.1 / 10.9.
bool i8_few_fused(int64_t rows, int64_t k)
{
    return rows <= 16 && rows * ((k + 127) / 128 * 128) <= 28672;
}

hipError_t launch_i8_few_fused(const void *x, int gx, int64_t rows, int64_t cols, int64_t ldx,
                               const I8View &b, void *out, int gt, int64_t ld, hipStream_t st)
{
    const I8View a = {nullptr, nullptr, rows, cols, b.wide};
    return with_elem_type(gx, [&](auto f) {
        return with_elem_type(gt, [&](auto g) {
            return launch_split<decltype(f)::value, decltype(g)::value, 1, kQuantised>(
                a, x, ldx, b, out, ld, st);
        });
    });
}

}  // namespace zo
