// zo_mx4_gemm.hip -- products of microscaled 4-bit matrices on the scaled matrix
// instruction (32 x 32 x 64, E2M1 operands, binary32 accumulators).  By itself, two waves a
// SIMD on random operands that stay in registers, it gives 6.3 PFLOP/s over 1 to 14 ms and
// the 16 x 16 x 128 form 6.8 (both 9.6 on operands that are all alike: the clock follows
// the bits that change); in this kernel this form was a few percent faster.
//
// Operand layout of the instruction: lane l holds row l % 32, elements
// 32 (l / 32) .. + 31 of the 64 (16 bytes), and their scale byte, one of the four bytes
// of a register.  An mx4 matrix (zo_ops.h) keeps these 16 bytes in tiles of 16 rows x
// 128 columns, block after block of 32 columns: two adjacent tiles hold two fragments
// of 32 rows x 64 columns, and 16 lanes read 256 contiguous bytes.  A lane's scale
// dword serves rows r % 16 + 16 {0, 1, 2, 3} of 64: shifted right by 8 in the lanes of
// the upper 16 rows, its bytes 0 and 2 are those of the two fragments.
//
// With b's rows as the first operand, a lane's results are runs of four columns of one
// row of the output.
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

// 32 rows of a wave's results, NF fragments of 32 columns, through this wave's part of
// shared memory (no other wave's business), so that a store writes whole runs of 128 or 256
// bytes: 16-byte chunk c of row r is kept at c ^ (r % 8).  16-bit results: the wave's
// halves swap runs of four, so that a lane holds 8 consecutive columns.  rows, cols: how
// many of them are there; STREAM: past the caches (see streamed).  Straight from the
// registers, 32 bytes of each row: 8192 x 6400 by 128 31 us in 16 bits, 60 in 32; so 27 and 46.
template <int GT, bool STREAM, int NF>
__device__ __forceinline__ void store_rows(typename Elem<GT>::T *out, int64_t ld, int64_t rows,
                                           int64_t cols, const f32x16 (&v)[NF], u32x4 *mine)
{
    constexpr int V = Elem<GT>::kVec, C = 32 * NF / V;     // 16-byte chunks of a row
    const int lane = threadIdx.x & 63, r = lane & 31, half = lane >> 5;
#pragma unroll
    for (int j = 0; j < NF; ++j) {
        if constexpr (GT == GT_F32) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                mine[r * C + ((j * 8 + q * 2 + half) ^ (r & 7))] =
                    u32x4{__float_as_uint(v[j][4 * q]), __float_as_uint(v[j][4 * q + 1]),
                          __float_as_uint(v[j][4 * q + 2]), __float_as_uint(v[j][4 * q + 3])};
        } else {
#pragma unroll
            for (int q = 0; q < 4; q += 2) {
                u32x4 w;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t x = (uint32_t)narrow<GT>(v[j][4 * q + 2 * h]) |
                                       (uint32_t)narrow<GT>(v[j][4 * q + 2 * h + 1]) << 16;
                    const uint32_t y = (uint32_t)narrow<GT>(v[j][4 * q + 4 + 2 * h]) |
                                       (uint32_t)narrow<GT>(v[j][4 * q + 5 + 2 * h]) << 16;
                    const auto s = __builtin_amdgcn_permlane32_swap(x, y, false, false);
                    w[h] = s[0];
                    w[2 + h] = s[1];
                }
                mine[r * C + ((j * 4 + q + half) ^ (r & 7))] = w;
            }
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int i = 0; i < C / 2; ++i) {
        const int row = i * (64 / C) + lane / C, c = lane % C;
        const u32x4 w = mine[row * C + (c ^ (row & 7))];
        typename Elem<GT>::T *to = out + row * ld + c * V;
        const int64_t nv = row < rows ? cols - c * V : 0;
        if (nv >= V) {
            u32x4_a2 *const p = reinterpret_cast<u32x4_a2 *>(to);
            if constexpr (STREAM)
                __builtin_nontemporal_store(w, p);
            else
                *p = w;
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e < nv)
                    to[e] = (typename Elem<GT>::T)(GT == GT_F32 ? w[e & 3]
                                                                : w[e / 2] >> (16 * (e & 1)));
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
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
// Measured: 16384 x 16384 by 8192 1.14 ms (3.9 PFLOP/s), 8192 x 6400 by 1600 67 us, 8192 x
// 1600 by 6400 56 us.  Bound: copies of the kernel that leave work out took, in this order,
// 0.79 ms (5.6 PFLOP/s), 45 and 40 us without any operand traffic, 0.84 ms, 44 and 42 us
// without the loads and the writes to shared memory, 1.10 ms, 62 and 54 us without the
// reads from it: the loads (32 KiB a step through the L1, about 30 bytes a clock) take the
// most beside the matrix pipe.
// Four waves of 128 x 128 read less of shared memory but leave no registers for loads
// in flight (1.5 ms); workgroups of 128 x 256, two a CU, spill (1.8 ms).
//
// The outputs begin at row tile m_tile and column tile n_tile (of 16).
template <int GT, int MT, int NT, int WN, bool ODD, bool STREAM>
__device__ __forceinline__ void product_tile(const Mx4View &a, const Mx4View &b,
                                             typename Elem<GT>::T *__restrict__ out, int64_t ld,
                                             int64_t m_tile, int64_t n_tile, u32x4 *lds)
{
    static_assert(MT % 4 == 0 && NT % 4 == 0, "whole groups of 64 rows per wave");
    constexpr int CHUNKS = 2 * MT + WN * NT, WAVES = 2 * WN;     // 1 KiB tiles of a step
    constexpr int MINE = CHUNKS / WAVES;
    constexpr int MS = MT / 4, NS = NT / 4;                      // groups of 64 rows
    constexpr int MF = MT / 2, NF = NT / 2, HALF = MF / 2;       // fragments of 32 rows
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

    // lane's place in a fragment: row half and 32-column block of the 64
    const int upper = lane >> 4 & 1, block = lane >> 5;
    const int frag_at = upper * 64 + block * 16 + (lane & 15);
    const int scale_at = (block * 16 + (lane & 15)) * 4;

    // set R holds the tiles and scales of the steps congruent to R modulo 2
    u32x4 stage[2][MINE];
    uint32_t ea[2][MS][2], eb[2][NS][2];      // the scales of both halves of a column tile
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
        for (int p = 0; p < 2; ++p) {
#pragma unroll
            for (int g = 0; g < MS; ++g)
                ea[R][g][p] = *reinterpret_cast<const uint32_t *>(sa[g] + at * 256 + p * 128 +
                                                                  scale_at);
#pragma unroll
            for (int g = 0; g < NS; ++g)
                eb[R][g][p] = *reinterpret_cast<const uint32_t *>(sb[g] + at * 256 + p * 128 +
                                                                  scale_at);
        }
    };
    auto put = [&](auto set, int buf) {
        constexpr int R = decltype(set)::value;
#pragma unroll
        for (int i = 0; i < MINE; ++i)
            lds[(buf * CHUNKS + i * WAVES + wave) * 64 + lane] = stage[R][i];
    };
    u32x4 fa[MF][2], fb[NF][2];
    auto read_a = [&](int buf, auto i) {
        constexpr int I = decltype(i)::value;
#pragma unroll
        for (int p = 0; p < 2; ++p)
            fa[I][p] = lds[(buf * CHUNKS + wm * MT + 2 * I) * 64 + p * 32 + frag_at];
    };
    auto read_b = [&](int buf, auto j) {
        constexpr int J = decltype(j)::value;
#pragma unroll
        for (int p = 0; p < 2; ++p)
            fb[J][p] = lds[(buf * CHUNKS + 2 * MT + wn * NT + 2 * J) * 64 + p * 32 + frag_at];
    };
    f32x16 acc[MF][NF] = {};
    // the products of half the row fragments with column fragment j
    auto multiply = [&](auto set, auto from, auto j) {
        unroll<2>([&](auto p) {
            unroll<HALF>([&](auto i) {
                constexpr int R = decltype(set)::value, P = decltype(p)::value;
                constexpr int I = decltype(from)::value + decltype(i)::value;
                constexpr int J = decltype(j)::value;
                acc[I][J] = mfma32<J % 2 * 2, I % 2 * 2>(fb[J][P], fa[I][P], acc[I][J],
                                                         eb[R][J / 2][P], ea[R][I / 2][P]);
            });
        });
    };
    using Zero = std::integral_constant<int, 0>;
    using One = std::integral_constant<int, 1>;
    using Lower = std::integral_constant<int, HALF>;
    // step t, t congruent to `now` modulo 2, in buffer t modulo 3
    int buf = 0;
    auto step = [&](auto now, int t) {
        constexpr int R = decltype(now)::value;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
#pragma unroll
            for (int g = 0; g < MS; ++g) ea[R][g][p] >>= upper * 8;
#pragma unroll
            for (int g = 0; g < NS; ++g) eb[R][g][p] >>= upper * 8;
        }
        const int next = buf == 2 ? 0 : buf + 1, after = next == 2 ? 0 : next + 1;
        unroll<NF>([&](auto j) {
            constexpr int J = decltype(j)::value;
            if constexpr (J < HALF) read_a(buf, std::integral_constant<int, HALF + J>{});
            multiply(now, Zero{}, j);
            __builtin_amdgcn_sched_barrier(0);
        });
        __syncthreads();                        // every wave's tiles of step t + 1 are there
        unroll<NF>([&](auto j) {
            constexpr int J = decltype(j)::value;
            if constexpr (J < HALF) read_a(next, j);
            if constexpr (J == NF / 2 - 1) put(now, after);
            if constexpr (J == NF / 2) fetch(now, t + 4);
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
        unroll<NF>([&](auto j) { read_b(0, j); });
        unroll<HALF>([&](auto i) { read_a(0, i); });
        int t = 0;
        for (; t + 1 < steps; t += 2) {
            step(Zero{}, t);
            step(One{}, t + 1);
        }
        if constexpr (ODD) step(Zero{}, t);
    }

    __syncthreads();                            // every wave has read its last operands
    static_assert(3 * CHUNKS >= WAVES * 2 * NT, "room for 32 binary32 rows of every wave");
    const int64_t m0 = m_tile * 16 + wm * MT * 16, n0 = n_tile * 16 + wn * NT * 16;
#pragma unroll
    for (int i = 0; i < MF; ++i) {
        store_rows<GT, STREAM>(out + (m0 + i * 32) * ld + n0, ld, a.rows - m0 - i * 32,
                               b.rows - n0, acc[i], lds + wave * (NT * 4 * 32));
        __builtin_amdgcn_sched_barrier(0);
    }
}

// One tile a workgroup.
template <int GT, int MT, int NT, int WN, bool ODD, bool STREAM>
__global__ __launch_bounds__(128 * WN, 2) void k_mx4_product(
    Mx4View a, Mx4View b, typename Elem<GT>::T *__restrict__ out, int64_t ld, uint32_t m_tiles,
    uint32_t n_tiles)
{
    extern __shared__ u32x4 lds[];                               // [3][CHUNKS][64]
    const TileIndex tile = tile_index(run_index(blockIdx.x, m_tiles * n_tiles), m_tiles, n_tiles);
    product_tile<GT, MT, NT, WN, ODD, STREAM>(a, b, out, ld, (int64_t)tile.m * 2 * MT,
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
        product_tile<GT, 8, 4, 4, ODD, false>(a, b, out, ld, (int64_t)tile.m * 16,
                                              (int64_t)tile.n * 16, lds);
    } else {
        const uint32_t half = blockIdx.x - whole;
        const TileIndex tile = tile_index(whole + half / 2, m_tiles, n_tiles);
        product_tile<GT, 4, 4, 4, ODD, false>(a, b, out, ld, (int64_t)tile.m * 16 + half % 2 * 8,
                                       (int64_t)tile.n * 16, lds);
    }
}

// Whether results are stored past the caches: where rows begin on lines of 128 bytes.
// The small tiles' products are short, and the lines they leave in the L2 are written at
// the end: 2047 x 4096 by 512 8.2 us against 9.6.  Rows off the lines would be written in
// parts: 4096 x 4100 by 512 23.6 us against 19.6.  The large tiles gain nothing
// (8192 x 6400 by 1600 67.2 against 64.8).
template <int GT>
static bool streamed(const void *out, int64_t ld)
{
    const uint64_t row = (uint64_t)ld * sizeof(typename Elem<GT>::T);
    return ((reinterpret_cast<uintptr_t>(out) | row) & 127) == 0;
}

// Shared memory beyond 64 KiB has to be asked for.
static hipError_t allow_lds(const void *kernel, uint32_t lds)
{
    if (lds <= 65536) return hipSuccess;
    return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
}

template <int GT, int MT, int NT, int WN, bool STREAM>
static hipError_t launch_tiles(const Mx4View &a, const Mx4View &b, void *out, int64_t ld,
                               hipStream_t st)
{
    constexpr uint32_t lds = 3 * (2 * MT + WN * NT) * 1024;
    const int64_t nt = (b.rows + 16 * WN * NT - 1) / (16 * WN * NT);
    const int64_t mt = (a.rows + 32 * MT - 1) / (32 * MT), tiles = mt * nt;
    const auto kernel = a.kt % 2 ? k_mx4_product<GT, MT, NT, WN, true, STREAM>
                                 : k_mx4_product<GT, MT, NT, WN, false, STREAM>;
    const hipError_t e = allow_lds(reinterpret_cast<const void *>(kernel), lds);
    if (e != hipSuccess) return e;
    return start(kernel, tiles, 128 * WN, lds, st, a, b, static_cast<typename Elem<GT>::T *>(out),
                 ld, (uint32_t)mt, (uint32_t)nt);
}

// How many of the large tiles are not halved.
static int64_t whole_tiles(int64_t tiles)
{
    const int64_t rest = tiles % kCus;
    return rest <= kCus / 2 && tiles > kCus ? tiles - rest : tiles;
}

template <int GT>
static hipError_t launch_large(const Mx4View &a, const Mx4View &b, void *out, int64_t ld,
                               hipStream_t st)
{
    constexpr uint32_t lds = 3 * 32 * 1024;
    const int64_t mt = (a.rows + 255) / 256, nt = (b.rows + 255) / 256, tiles = mt * nt;
    const int64_t whole = whole_tiles(tiles);
    const auto kernel = a.kt % 2 ? k_mx4_product_large<GT, true> : k_mx4_product_large<GT, false>;
    const hipError_t e = allow_lds(reinterpret_cast<const void *>(kernel), lds);
    if (e != hipSuccess) return e;
    return start(kernel, 2 * tiles - whole, 512, lds, st, a, b,
                 static_cast<typename Elem<GT>::T *>(out), ld, (uint32_t)mt, (uint32_t)nt,
                 (uint32_t)whole);
}

enum class Form { kFew, kLarge, kMiddle, kSmall };

static int64_t tiles_of(int64_t m, int64_t n, int64_t tile_m, int64_t tile_n)
{
    return (m + tile_m - 1) / tile_m * ((n + tile_n - 1) / tile_n);
}

// Large tiles need less of memory and LDS per product and take a CU each; of 128 x 128 a
// CU takes three.  Large ones pay where they make one round of the GPU and the others
// more than one, or from one and a half rounds on, if the steps are many for the time that
// a workgroup, alone on its CU, takes to write its results (the more so in 32 bits on lines,
// where the others' stores go past the caches); with many steps, from two thirds of a
// round on.  Otherwise 128 x 128 while that occupies half of the GPU, then 128 x 64.
// Measured both sides in a graph, outputs in turn, us, large / 128 x 128:
//   175 tiles, 6400 x 1600: 16 bits by 1600 20.5 / 18.2, by 6400 1% under; 32 bits by 6400
//   57.9 / 57.0; 196 off the lines, 812 x 12547 by 4640 49.9 / 54.0; 192, 6144 x 2048 by 1600
//   19.9 / 18.8; 320, 5120 x 4096 by 2560 48.4 / 42.0
//   200 (800 of the others), 10208 x 1239 by 4007 45.6 / 53.4; 208, 6656 x 2048: 16 bits by
//   1024 17.1 / 17.9; 32 bits by 1280 23.5 / 23.9; 224, 8192 x 1600 by 6400 55.6 / 74.2
//   16 bits on lines: 8192 x 6400 by 1024 54.1 / 51.0, by 2560 2% under; 10240 x 4096 by 1280
//   52.1 / 46.9, by 4096 2% under; 8192 x 4096 by 1600 45.1 / 47.9
//   32 bits on lines: 8192 x 4096 by 2560 77.9 / 70.9, by 4096 102.7 / 103.7
//   off the lines: 4096 x 50257 in 16 bits by 1024 240 / 256, in 32 328 / 362; 8192 x 4098 in
//   32 bits by 768 49.5 / 57.2
// 128 x 128 / 128 x 64: 144 tiles, 1152 x 2048 by 1600 9.0 / 10.6; 128, 2047 x 1024 by 4096
// 16.6 / 15.0, by 512 6.1 / 5.7.
static Form form_of(int64_t m, int64_t n, int64_t kt, bool f32, bool stream)
{
    if (m <= kFewRows) return Form::kFew;
    const int64_t large = tiles_of(m, n, 256, 256), middle = tiles_of(m, n, 128, 128);
    const bool fills = large <= kCus ? middle > 3 * kCus : large >= kCus * 3 / 2;
    const int64_t steps = !stream        ? (f32 ? 3 : 8)
                          : large > kCus ? (f32 ? 32 : 16)
                                         : (f32 ? 10 : 8);
    if (fills && kt >= steps) return Form::kLarge;
    if (large >= 168 && large <= kCus && kt >= 32 && !(f32 && stream)) return Form::kLarge;
    return middle >= 144 ? Form::kMiddle : Form::kSmall;
}

bool mx4_product_fits(int64_t m, int64_t n, int64_t k, int gt, const void *out, int64_t ld)
{
    if (m == 0 || n == 0) return true;
    const bool stream = gt == GT_F32 ? streamed<GT_F32>(out, ld) : streamed<GT_BF16>(out, ld);
    switch (form_of(m, n, (k + 127) / 128, gt == GT_F32, stream)) {
    case Form::kFew: return mx4_few_fits(n, k);
    case Form::kLarge: {
        const int64_t tiles = tiles_of(m, n, 256, 256);
        return fits_a_launch(2 * tiles - whole_tiles(tiles), 512);
    }
    case Form::kMiddle: return fits_a_launch(tiles_of(m, n, 128, 128), 256);
    default: return fits_a_launch(tiles_of(m, n, 128, 64), 128);
    }
}

hipError_t launch_mx4_product(const Mx4View &a, const Mx4View &b, void *out, int gt, int64_t ld,
                              hipStream_t st)
{
    if (a.rows == 0 || b.rows == 0) return hipSuccess;
    if (a.rows <= kFewRows) return launch_mx4_few(a, b, out, gt, ld, st);
    return with_elem_type(gt, [&](auto g) {
        constexpr int GT = decltype(g)::value;
        const bool stream = streamed<GT>(out, ld);
        switch (form_of(a.rows, b.rows, a.kt, GT == GT_F32, stream)) {
        case Form::kLarge: return launch_large<GT>(a, b, out, ld, st);
        case Form::kMiddle:
            return stream ? launch_tiles<GT, 4, 4, 2, true>(a, b, out, ld, st)
                          : launch_tiles<GT, 4, 4, 2, false>(a, b, out, ld, st);
        default:
            return stream ? launch_tiles<GT, 4, 4, 1, true>(a, b, out, ld, st)
                          : launch_tiles<GT, 4, 4, 1, false>(a, b, out, ld, st);
        }
    });
}

}  // namespace zo
