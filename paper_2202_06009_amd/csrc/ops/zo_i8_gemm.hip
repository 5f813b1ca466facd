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

// This wave's loads but the last N have arrived and its reads of shared memory are done,
// then the barrier: what all waves' loads brought is there, what they read may be replaced.
template <int N>
__device__ __forceinline__ void wait_barrier()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <int N>
using Int = std::integral_constant<int, N>;

// 32 MF WR x 32 NF WC outputs per workgroup of WR x WC waves, 32 MF x 32 NF a wave.
//
// A step multiplies 128 columns of both operands, in four slices of 32, out of one of S
// buffers in shared memory; the loads of the steps after it go straight into the others, whole
// lines of 128 bytes a row (rows of 64 bytes load at half the rate: 28 bytes a clock and CU
// against 56).  The buffers are arrays of their own: the compiler then knows that a read of one
// need not wait for loads into another.  A row's eight chunks of 16 bytes stand at
// c ^ (row % 8), so that the 32 rows of a fragment read all banks alike: the loads place chunk
// after chunk, so a lane fetches the chunk that belongs in its place.
//
// Loads and fragment reads are placed one by one between the products: issued in a burst, a
// wave's eight loads of a step hold its matrix instructions up until the address unit has taken
// them (8192 x 8192 by 8192: 487 us in bursts, 434 so).  A slice's products run from fragments
// that were read during the slice before; the last slice's run past the step's one barrier,
// among the reads of the next buffer.  The loads of a step are issued among the first slices
// (TAIL: how many slices before the last are left without), so that they have the rest of it.
//
// Measured, us: 8192 x 8192 by 8192 434 (2.5 POP/s), 8192 x 6400 by 1600 98, 8192 x 1600 by
// 6400 80, 6400 x 1600 by 8192 87.  By itself the instruction gives 3.45 POP/s on random
// operands that stay in registers (4.3 on operands that are all alike: the clock follows the
// bits that change).  Bound: copies of the kernel that leave work out took, of the 487 us, 326
// without any operand traffic, 376 without the loads, 432 without the fragment reads.
template <int GT, int MF, int NF, int WR, int WC, int S, int TAIL, int OCC, bool STREAM>
__global__ __launch_bounds__(64 * WR * WC, OCC) void k_i8_product(
    I8View a, I8View b, typename Elem<GT>::T *__restrict__ out, int64_t ld, uint32_t m_tiles,
    uint32_t n_tiles)
{
    constexpr int WAVES = WR * WC, BM = 32 * MF * WR, BN = 32 * NF * WC, ROWS = BM + BN;
    constexpr int MINE = ROWS / 8 / WAVES, OF_A = BM / 8 / WAVES;   // a wave's loads of 8 rows
    constexpr int SIZE = ROWS * 8, READS = MF + NF, PRODUCTS = MF * NF;
    static_assert(BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0, "whole loads for every wave");
    static_assert(S >= 2 && S <= 4 && MINE * (S - 2) < 64, "what the wait can count");
    __shared__ u32x4 buf0[SIZE], buf1[SIZE], buf2[S > 2 ? SIZE : 1], buf3[S > 3 ? SIZE : 1];
    const TileIndex tile = tile_index(run_index(blockIdx.x, m_tiles * n_tiles), m_tiles, n_tiles);
    const int64_t m0 = (int64_t)tile.m * BM, n0 = (int64_t)tile.n * BN;
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WC, wn = wave % WC;
    const int steps = (int)(a.wide / 128);
    auto buf = [&](auto i) __attribute__((always_inline)) -> u32x4 * {
        constexpr int N = decltype(i)::value;
        return N == 0 ? buf0 : N == 1 ? buf1 : N == 2 ? buf2 : buf3;
    };

    // rows beyond the last stand for it; what is computed from them is not stored.  Within a
    // tile 32 bits hold the offsets: 256 rows of at most 2^17 bytes
    uint32_t off[MINE];
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
        const int64_t r = ((i < OF_A ? i : i - OF_A) * WAVES + wave) * 8 + lane / 8;
        off[i] = (uint32_t)((i < OF_A ? min(r, a.rows - 1 - m0) : min(r, b.rows - 1 - n0)) * a.wide) +
                 ((lane & 7) ^ (lane >> 3)) * 16;
    }
    const int8_t *from_a = a.codes + m0 * a.wide, *from_b = b.codes + n0 * a.wide;
    auto load = [&](auto i, u32x4 *to, uint32_t at) __attribute__((always_inline)) {
        constexpr int P = decltype(i)::value;
        load_lds((P < OF_A ? from_a : from_b) + at + off[P], to + (P * WAVES + wave) * 64);
    };
    auto fetch = [&](u32x4 *to, uint32_t at) __attribute__((always_inline)) {
        unroll<MINE>([&](auto i) __attribute__((always_inline)) { load(i, to, at); });
    };

    const int row_a = (wm * 32 * MF + (lane & 31)) * 8, row_b = (BM + wn * 32 * NF + (lane & 31)) * 8;
    i32x16 acc[MF][NF] = {};
    u32x4 fa[2][MF], fb[2][NF];
    // fragment n of slice k into set k % 2, in the order b0 a0 b1 a1 ...
    auto read = [&](const u32x4 *from, auto k, auto n) __attribute__((always_inline)) {
        constexpr int K = decltype(k)::value, N = decltype(n)::value;
        constexpr int PAIRED = 2 * (MF < NF ? MF : NF);
        constexpr bool OF_B = N < PAIRED ? N % 2 == 0 : NF > MF;
        constexpr int I = N < PAIRED ? N / 2 : N - PAIRED / 2;
        const int c = (2 * K + half) ^ (lane & 7);
        if constexpr (OF_B)
            fb[K & 1][I] = from[row_b + I * 256 + c];
        else
            fa[K & 1][I] = from[row_a + I * 256 + c];
    };
    // the products of slice k; among them the reads of slice `next` from `from` and the loads
    // P0 .. P1 - 1 into `to`
    auto slice = [&](auto k, auto next, const u32x4 *from, bool reads, auto p0, auto p1, u32x4 *to,
                     bool loads, uint32_t at) __attribute__((always_inline)) {
        constexpr int R = decltype(k)::value & 1, P0 = decltype(p0)::value;
        constexpr int NP = decltype(p1)::value - P0, LAST = PRODUCTS > 1 ? PRODUCTS - 1 : 1;
        unroll<PRODUCTS>([&](auto n) __attribute__((always_inline)) {
            constexpr int N = decltype(n)::value, I = N / NF, J = N % NF;
            acc[I][J] = mfma_i8(fb[R][J], fa[R][I], acc[I][J]);
            __builtin_amdgcn_sched_barrier(0);
            constexpr int A = N * READS / LAST, B = (N + 1) * READS / LAST;
            constexpr int A1 = A < READS ? A : READS, B1 = B < READS ? B : READS;
            if (reads)
                unroll<B1 - A1>([&](auto q) __attribute__((always_inline)) {
                    read(from, next, Int<A1 + decltype(q)::value>{});
                });
            constexpr int L0 = N * NP / PRODUCTS, L1 = (N + 1) * NP / PRODUCTS;
            if (loads)
                unroll<L1 - L0>([&](auto q) __attribute__((always_inline)) {
                    load(Int<P0 + L0 + decltype(q)::value>{}, to, at);
                });
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    // step t in buffer B = t % S; the loads of step t + S - 1 go into the one of step t - 1
    auto step = [&](auto b, int t) __attribute__((always_inline)) {
        constexpr int B = decltype(b)::value, SLICES = 3 - TAIL;
        u32x4 *now = buf(Int<B>{}), *next = buf(Int<(B + 1) % S>{}), *last = buf(Int<(B + S - 1) % S>{});
        const bool more = t + S - 1 < steps;
        unroll<3>([&](auto k) __attribute__((always_inline)) {
            constexpr int K = decltype(k)::value;
            slice(k, Int<K + 1>{}, now, true, Int<(K < SLICES ? MINE * K / SLICES : MINE)>{},
                  Int<(K < SLICES ? MINE * (K + 1) / SLICES : MINE)>{}, last, more,
                  (uint32_t)(t + S - 1) * 128);
        });
        if (more)
            wait_barrier<MINE *(S - 2)>();
        else
            wait_barrier<0>();
        __builtin_amdgcn_sched_barrier(0);
        slice(Int<3>{}, Int<0>{}, next, t + 1 < steps, Int<0>{}, Int<0>{}, now, false, 0);
    };
    if (steps > 0) {
        fetch(buf0, 0);
        if (S > 2 && steps > 1) fetch(buf1, 128);
        if (S > 3 && steps > 2) fetch(buf2, 256);
        if (steps >= S - 1)
            wait_barrier<MINE *(S - 2)>();
        else
            wait_barrier<0>();
        unroll<READS>([&](auto n) __attribute__((always_inline)) { read(buf0, Int<0>{}, n); });
        int t = 0;
        for (; t + S <= steps; t += S)
            unroll<S>([&](auto u) __attribute__((always_inline)) { step(u, t + decltype(u)::value); });
        unroll<S - 1>([&](auto u) __attribute__((always_inline)) {
            if (t + decltype(u)::value < steps) step(u, t + decltype(u)::value);
        });
    }
    __syncthreads();                            // every wave has read its last operands

    constexpr int FIT = SIZE / (NF * 256);      // waves whose 32 binary32 rows fit a buffer
    static_assert(2 * FIT >= WAVES, "room for every wave in two buffers");
    u32x4 *mine = wave < FIT ? buf0 + wave * (NF * 256) : buf1 + (wave - FIT) * (NF * 256);
    const int64_t mw = m0 + wm * 32 * MF, nw = n0 + wn * 32 * NF;
    f32x4 sb[NF][4];
#pragma unroll
    for (int j = 0; j < NF; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t n = nw + j * 32 + q * 8 + half * 4 + e;
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

template <int GT, int MF, int NF, int WR, int WC, int S, int TAIL, int OCC>
static hipError_t launch_tiles(const I8View &a, const I8View &b, void *out, int64_t ld,
                               hipStream_t st)
{
    constexpr int BM = 32 * MF * WR, BN = 32 * NF * WC;
    const int64_t mt = (a.rows + BM - 1) / BM, nt = (b.rows + BN - 1) / BN;
    const auto kernel = streamed<GT>(out, ld) ? k_i8_product<GT, MF, NF, WR, WC, S, TAIL, OCC, true>
                                              : k_i8_product<GT, MF, NF, WR, WC, S, TAIL, OCC, false>;
    return start(kernel, mt * nt, 64 * WR * WC, 0, st, a, b,
                 static_cast<typename Elem<GT>::T *>(out), ld, (uint32_t)mt, (uint32_t)nt);
}

// The forms, and what they take (ns): a workgroup's step where it has its CU to itself, where
// the CU is full (one of 256 x 256 fills it, two of the others), and what comes before and after
// the steps.  Fitted to the measured us (POP/s where the GPU is full):
//                        256x256  192x128  128x128  128x64   64x64
//   8192 x 8192 by 8192   434      485      501      660      824
//   8192 x 6400 by 1600   105       98      107      124      165
//   8192 x 1600 by 6400    80      111       94      113      135
//   6400 x 1600 by 8192    89       86      107      108      130
//   2047 x 4096 by 1024    17.4     15.5     12.7     16.4     20.4
//   2047 x 1024 by 4096    45       30.5     26.1     16.9     14.8
//   4096 x 1024 by 2047    26.6     18.3     13.1     12.8     16.6
//    100 x 6400 by 1600    21.3     13.2     10.4      7.5      6.2
enum class Form { kFew, k256, k192, k128, k64, k64x64 };

struct FormCost {
    Form form;
    int64_t rows, cols, a_cu, alone, full, ends;
};
constexpr FormCost kForms[] = {
    {Form::k256, 256, 256, 1, 1550, 1550, 6500}, {Form::k192, 192, 128, 2, 950, 1380, 3000},
    {Form::k128, 128, 128, 2, 800, 970, 3000},   {Form::k64, 128, 64, 2, 500, 640, 2500},
    {Form::k64x64, 64, 64, 2, 330, 400, 2000},
};

static int64_t tiles_of(int64_t m, int64_t n, int64_t tile_m, int64_t tile_n)
{
    return (m + tile_m - 1) / tile_m * ((n + tile_n - 1) / tile_n);
}

static Form form_of(int64_t m, int64_t n, int64_t steps)
{
    if (m <= kI8FewRows) return Form::kFew;
    Form best = Form::k256;
    int64_t least = INT64_MAX;
    for (const FormCost &f : kForms) {
        const int64_t tiles = tiles_of(m, n, f.rows, f.cols), rounds = tiles / (kCus * f.a_cu);
        const int64_t rest = tiles % (kCus * f.a_cu);
        int64_t cost = rounds * (steps * f.full + f.ends);
        if (rest) cost += steps * (rest <= kCus ? f.alone : f.full) + f.ends;
        if (cost < least) {
            least = cost;
            best = f.form;
        }
    }
    return best;
}

bool i8_product_fits(int64_t m, int64_t n, int64_t k)
{
    if (m == 0 || n == 0) return true;
    const Form form = form_of(m, n, (k + 127) / 128);
    if (form == Form::kFew) return i8_few_fits(n, k);
    for (const FormCost &f : kForms)
        if (f.form == form)
            return fits_a_launch(tiles_of(m, n, f.rows, f.cols), form == Form::k256 ? 512 : 256);
    return false;
}

hipError_t launch_i8_product(const I8View &a, const I8View &b, void *out, int gt, int64_t ld,
                             hipStream_t st)
{
    if (a.rows == 0 || b.rows == 0) return hipSuccess;
    const Form form = form_of(a.rows, b.rows, a.wide / 128);
    if (form == Form::kFew) return launch_i8_few(a, b, out, gt, ld, st);
    return with_elem_type(gt, [&](auto g) {
        constexpr int GT = decltype(g)::value;
        switch (form) {
        case Form::k256: return launch_tiles<GT, 4, 2, 2, 4, 2, 2, 2>(a, b, out, ld, st);
        case Form::k192: return launch_tiles<GT, 3, 2, 2, 2, 2, 2, 2>(a, b, out, ld, st);
        case Form::k128: return launch_tiles<GT, 2, 2, 2, 2, 2, 1, 2>(a, b, out, ld, st);
        case Form::k64: return launch_tiles<GT, 2, 1, 2, 2, 3, 1, 2>(a, b, out, ld, st);
        default: return launch_tiles<GT, 1, 1, 2, 2, 4, 1, 2>(a, b, out, ld, st);
        }
    });
}

}  // namespace zo
