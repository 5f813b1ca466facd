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
#include "zo_mx4_device.h"

namespace zo {

// Calls f(integral_constant<0>) .. f(integral_constant<N - 1>).
template <int N, class F>
__device__ __forceinline__ void unroll(F &&f)
{
    if constexpr (N > 0) {
        unroll<N - 1>(f);
        f(std::integral_constant<int, N - 1>{});
    }
}

// Two adjacent 16 x 16 tiles of results, u of columns n .. n + 15 and v of the next
// 16: rows of 16 lanes swap halves so that a lane holds 8 consecutive columns (of
// u in lanes 0..15 and 32..47, of v in the others) and a row of the output gets 64
// (16-bit) or 128 bytes at once.
template <int GT>
__device__ __forceinline__ void store_pair(typename Elem<GT>::T *row, int64_t n, int64_t cols,
                                           bool inside, f32x4 u, f32x4 v, int lane)
{
    const int g = lane >> 4;
    if constexpr (GT == GT_F32) {
        // 16 bytes a lane as they are
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x4 &x = h ? v : u;
            const int64_t at = n + h * 16 + g * 4, nv = cols - at;
            if (!inside) continue;
            if (nv >= 4) {
                *reinterpret_cast<u32x4_a2 *>(row + at) = __builtin_bit_cast(u32x4, x);
            } else {
                for (int q = 0; q < 4; ++q)
                    if (q < nv) row[at + q] = __float_as_uint(x[q]);
            }
        }
    } else {
        u32x4 w;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t a = (uint32_t)narrow<GT>(u[2 * h]) |
                               (uint32_t)narrow<GT>(u[2 * h + 1]) << 16;
            const uint32_t b = (uint32_t)narrow<GT>(v[2 * h]) |
                               (uint32_t)narrow<GT>(v[2 * h + 1]) << 16;
            const auto s = __builtin_amdgcn_permlane16_swap(a, b, false, false);
            w[h] = s[0];
            w[2 + h] = s[1];
        }
        const int64_t at = n + (g & 1) * 16 + (g >> 1) * 8, nv = cols - at;
        if (!inside) return;
        if (nv >= 8) {
            *reinterpret_cast<u32x4_a2 *>(row + at) = w;
        } else {
            for (int q = 0; q < 8; ++q) {
                if (q >= nv) break;
                const uint32_t d = q < 2 ? w[0] : q < 4 ? w[1] : q < 6 ? w[2] : w[3];
                row[at + q] = (uint16_t)(d >> (16 * (q & 1)));
            }
        }
    }
}

// The workgroup's tile of the output.  Workgroups go to the 8 XCDs in turn, each
// of which has an L2 of its own: an XCD gets a contiguous run of tiles, walked
// down kBand rows of tiles at a time, so that its workgroups share operands.
constexpr uint32_t kXcds = 8, kBand = 8;
constexpr int64_t kCus = 256;

struct TileIndex {
    uint32_t m, n;
};

// Workgroup wg of `total` in an XCD's run.
__device__ __forceinline__ uint32_t run_index(uint32_t wg, uint32_t total)
{
    const uint32_t each = total / kXcds, more = total % kXcds, x = wg % kXcds;
    return x * each + min(x, more) + wg / kXcds;
}

__device__ __forceinline__ TileIndex tile_index(uint32_t id, uint32_t m_tiles, uint32_t n_tiles)
{
    const uint32_t band = id / (kBand * n_tiles), in = id % (kBand * n_tiles);
    const uint32_t height = min(kBand, m_tiles - band * kBand);
    return {band * kBand + in % height, in / height};
}

// Where the 1 KiB tile of 16 rows x 128 columns with row tile index rt begins, at
// column tile 0; row tiles beyond the matrix stand for the last that is stored
// (what is computed from them is not stored).
__device__ __forceinline__ const uint8_t *tile_at(const Mx4View &x, int64_t rt)
{
    const int64_t stored = (x.rows + 63) / 64 * 4;
    return x.codes + min(rt, stored - 1) * x.kt * 1024;
}

// The same for the scales of 64 rows.
__device__ __forceinline__ const uint8_t *scales_at(const Mx4View &x, int64_t group)
{
    const int64_t stored = (x.rows + 63) / 64;
    return x.scales + min(group, stored - 1) * x.kt * 256;
}

// 32 MT x 16 WN NT outputs per workgroup of 2 x WN waves, 16 MT x 16 NT per wave, the
// operands through shared memory in three buffers of one column tile each.
//
// A step multiplies one column tile.  Its first half (the wave's upper row tiles
// of a) runs from fragments that are in registers while the lower half's are
// read; then, past the step's one barrier, the second half runs while the next
// step's first fragments are read from the next buffer (each of b's as soon as its
// last product is under way), the tiles that were loaded two steps ago are written
// to the buffer after that, and loads into their registers are issued: two steps
// of loads are in flight, about what the memory's latency takes.
// ODD: an odd number of steps (the register sets go round by twos).
//
// The outputs begin at row tile m_tile and column tile n_tile (of 16).
template <int GT, int MT, int NT, int WN, bool ODD>
__device__ __forceinline__ void product_tile(const Mx4View &a, const Mx4View &b,
                                             typename Elem<GT>::T *__restrict__ out, int64_t ld,
                                             int64_t m_tile, int64_t n_tile, u32x4 *lds)
{
    static_assert(MT % 4 == 0 && NT % 4 == 0, "whole groups of 64 rows per wave");
    constexpr int CHUNKS = 2 * MT + WN * NT, WAVES = 2 * WN;     // 1 KiB tiles of a step
    constexpr int MINE = CHUNKS / WAVES;
    constexpr int MS = MT / 4, NS = NT / 4, HALF = MT / 2;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int steps = (int)a.kt;

    // this wave's share of the loads: chunk c < 2 MT is of a, the others of b
    const uint8_t *src[MINE];
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
        const int c = i * WAVES + wave;
        src[i] = c < 2 * MT ? tile_at(a, m_tile + c) : tile_at(b, n_tile + (c - 2 * MT));
    }
    const uint8_t *sa[MS], *sb[NS];
#pragma unroll
    for (int g = 0; g < MS; ++g) sa[g] = scales_at(a, m_tile / 4 + wm * MS + g);
#pragma unroll
    for (int g = 0; g < NS; ++g) sb[g] = scales_at(b, n_tile / 4 + wn * NS + g);

    // set R holds the tiles and scales of the steps congruent to R modulo 2
    u32x4 stage[2][MINE];
    uint32_t ea[2][MS], eb[2][NS];
    auto fetch = [&](auto set, int t) {
        constexpr int R = decltype(set)::value;
        const int64_t at = min(t, steps - 1);
#pragma unroll
        for (int i = 0; i < MINE; ++i)
            stage[R][i] = *reinterpret_cast<const u32x4 *>(src[i] + at * 1024 + lane * 16);
    };
    auto read_scales = [&](auto set, int t) {
        constexpr int R = decltype(set)::value;
        const int64_t at = min(t, steps - 1);
#pragma unroll
        for (int g = 0; g < MS; ++g)
            ea[R][g] = *reinterpret_cast<const uint32_t *>(sa[g] + at * 256 + lane * 4);
#pragma unroll
        for (int g = 0; g < NS; ++g)
            eb[R][g] = *reinterpret_cast<const uint32_t *>(sb[g] + at * 256 + lane * 4);
    };
    auto put = [&](auto set, int buf) {
        constexpr int R = decltype(set)::value;
#pragma unroll
        for (int i = 0; i < MINE; ++i)
            lds[(buf * CHUNKS + i * WAVES + wave) * 64 + lane] = stage[R][i];
    };
    u32x4 fa[MT], fb[NT];
    auto read_a = [&](int buf, auto i) {
        constexpr int I = decltype(i)::value;
        fa[I] = lds[(buf * CHUNKS + wm * MT + I) * 64 + lane];
    };
    auto read_b = [&](int buf, auto j) {
        constexpr int J = decltype(j)::value;
        fb[J] = lds[(buf * CHUNKS + 2 * MT + wn * NT + J) * 64 + lane];
    };
    f32x4 acc[MT][NT] = {};
    // the products of half the row tiles with column tile j
    auto multiply = [&](auto set, auto from, auto j) {
        unroll<HALF>([&](auto i) {
            constexpr int R = decltype(set)::value;
            constexpr int I = decltype(from)::value + decltype(i)::value;
            constexpr int J = decltype(j)::value;
            acc[I][J] = mfma<J % 4, I % 4>(fb[J], fa[I], acc[I][J], eb[R][J / 4], ea[R][I / 4]);
        });
    };
    using Zero = std::integral_constant<int, 0>;
    using One = std::integral_constant<int, 1>;
    using Lower = std::integral_constant<int, HALF>;
    // step t, t congruent to `now` modulo 2, in buffer t modulo 3
    int buf = 0;
    auto step = [&](auto now, int t) {
        const int next = buf == 2 ? 0 : buf + 1, after = next == 2 ? 0 : next + 1;
        unroll<NT>([&](auto j) {
            constexpr int J = decltype(j)::value;
            if constexpr (J < HALF) read_a(buf, std::integral_constant<int, HALF + J>{});
            multiply(now, Zero{}, j);
            __builtin_amdgcn_sched_barrier(0);
        });
        __syncthreads();                        // every wave's tiles of step t + 1 are there
        unroll<NT>([&](auto j) {
            constexpr int J = decltype(j)::value;
            if constexpr (J < HALF) read_a(next, j);
            if constexpr (J == NT / 2 - 1) put(now, after);
            if constexpr (J == NT / 2) fetch(now, t + 4);
            multiply(now, Lower{}, j);
            read_b(next, j);
            __builtin_amdgcn_sched_barrier(0);
        });
        read_scales(now, t + 2);
        buf = next;
    };

    if (steps > 0) {
        fetch(Zero{}, 0);
        fetch(One{}, 1);
        read_scales(Zero{}, 0);
        read_scales(One{}, 1);
        put(Zero{}, 0);
        fetch(Zero{}, 2);
        put(One{}, 1);
        fetch(One{}, 3);
        __syncthreads();
        unroll<NT>([&](auto j) { read_b(0, j); });
        unroll<HALF>([&](auto i) { read_a(0, i); });
        int t = 0;
        for (; t + 1 < steps; t += 2) {
            step(Zero{}, t);
            step(One{}, t + 1);
        }
        if constexpr (ODD) step(Zero{}, t);
    }

    const int64_t m0 = m_tile * 16 + wm * MT * 16 + (lane & 15);
    const int64_t n0 = n_tile * 16 + wn * NT * 16;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t m = m0 + i * 16;
#pragma unroll
        for (int j = 0; j < NT; j += 2)
            store_pair<GT>(out + m * ld, n0 + j * 16, b.rows, m < a.rows, acc[i][j], acc[i][j + 1],
                           lane);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// One tile a workgroup.
template <int GT, int MT, int NT, int WN, bool ODD>
__global__ __launch_bounds__(128 * WN, 2) void k_mx4_product(
    Mx4View a, Mx4View b, typename Elem<GT>::T *__restrict__ out, int64_t ld, uint32_t m_tiles,
    uint32_t n_tiles)
{
    extern __shared__ u32x4 lds[];                               // [3][CHUNKS][64]
    const TileIndex tile = tile_index(run_index(blockIdx.x, m_tiles * n_tiles), m_tiles, n_tiles);
    product_tile<GT, MT, NT, WN, ODD>(a, b, out, ld, (int64_t)tile.m * 2 * MT,
                                      (int64_t)tile.n * WN * NT, lds);
}

// Tiles of 256 x 256, of which the first `whole` take one workgroup each and the
// others, too few for a round of the GPU, two of 128 rows each.
template <int GT, bool ODD>
__global__ __launch_bounds__(512, 2) void k_mx4_product_large(
    Mx4View a, Mx4View b, typename Elem<GT>::T *__restrict__ out, int64_t ld, uint32_t m_tiles,
    uint32_t n_tiles, uint32_t whole)
{
    extern __shared__ u32x4 lds[];
    if (blockIdx.x < whole) {
        const TileIndex tile = tile_index(run_index(blockIdx.x, whole), m_tiles, n_tiles);
        product_tile<GT, 8, 4, 4, ODD>(a, b, out, ld, (int64_t)tile.m * 16, (int64_t)tile.n * 16,
                                       lds);
    } else {
        const uint32_t half = blockIdx.x - whole;
        const TileIndex tile = tile_index(whole + half / 2, m_tiles, n_tiles);
        product_tile<GT, 4, 4, 4, ODD>(a, b, out, ld, (int64_t)tile.m * 16 + half % 2 * 8,
                                       (int64_t)tile.n * 16, lds);
    }
}

// Shared memory beyond 64 KiB has to be asked for.
static hipError_t allow_lds(const void *kernel, uint32_t lds)
{
    if (lds <= 65536) return hipSuccess;
    return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
}

template <int GT, int MT, int NT, int WN>
static hipError_t launch_tiles(const Mx4View &a, const Mx4View &b, void *out, int64_t ld,
                               hipStream_t st)
{
    constexpr uint32_t lds = 3 * (2 * MT + WN * NT) * 1024;
    const int64_t nt = (b.rows + 16 * WN * NT - 1) / (16 * WN * NT);
    const int64_t mt = (a.rows + 32 * MT - 1) / (32 * MT), tiles = mt * nt;
    if (tiles > INT32_MAX || a.kt > INT32_MAX) return hipErrorInvalidValue;
    const auto kernel =
        a.kt % 2 ? k_mx4_product<GT, MT, NT, WN, true> : k_mx4_product<GT, MT, NT, WN, false>;
    const hipError_t e = allow_lds(reinterpret_cast<const void *>(kernel), lds);
    if (e != hipSuccess) return e;
    kernel<<<dim3((uint32_t)tiles), 128 * WN, lds, st>>>(
        a, b, static_cast<typename Elem<GT>::T *>(out), ld, (uint32_t)mt, (uint32_t)nt);
    return hipGetLastError();
}

template <int GT>
static hipError_t launch_large(const Mx4View &a, const Mx4View &b, void *out, int64_t ld,
                               hipStream_t st)
{
    constexpr uint32_t lds = 3 * 32 * 1024;
    const int64_t mt = (a.rows + 255) / 256, nt = (b.rows + 255) / 256, tiles = mt * nt;
    if (tiles > INT32_MAX || a.kt > INT32_MAX) return hipErrorInvalidValue;
    const int64_t rest = tiles % kCus;
    const int64_t whole = rest <= kCus / 2 && tiles > kCus ? tiles - rest : tiles;
    const auto kernel = a.kt % 2 ? k_mx4_product_large<GT, true> : k_mx4_product_large<GT, false>;
    const hipError_t e = allow_lds(reinterpret_cast<const void *>(kernel), lds);
    if (e != hipSuccess) return e;
    kernel<<<dim3((uint32_t)(whole + 2 * (tiles - whole))), 512, lds, st>>>(
        a, b, static_cast<typename Elem<GT>::T *>(out), ld, (uint32_t)mt, (uint32_t)nt,
        (uint32_t)whole);
    return hipGetLastError();
}

hipError_t launch_mx4_product(const Mx4View &a, const Mx4View &b, void *out, int gt, int64_t ld,
                              hipStream_t st)
{
    if (a.rows == 0 || b.rows == 0) return hipSuccess;
    if (a.rows <= kFewRows) return launch_mx4_few(a, b, out, gt, ld, st);
    const auto count = [&](int64_t m, int64_t n) {
        return (a.rows + m - 1) / m * ((b.rows + n - 1) / n);
    };
    return with_elem_type(gt, [&](auto g) {
        constexpr int GT = decltype(g)::value;
        if (count(256, 256) >= 224) return launch_large<GT>(a, b, out, ld, st);
        if (count(128, 128) >= 144) return launch_tiles<GT, 4, 4, 2>(a, b, out, ld, st);
        return launch_tiles<GT, 4, 4, 1>(a, b, out, ld, st);
    });
}

}  // namespace zo
