// zo_norm.hip -- the residual's addition with the root-mean-square norm, into the inputs'
// type and into 8-bit rows, and its gradients.
//
// Bound by memory: every input read once, every output written once.  A row stays in the
// registers of its threads (a wave for short rows, four of them a workgroup) between the
// sum of squares and the outputs.  The codes of h weight are those of h rstd weight, so
// that the largest magnitude is known with the sum of squares: one reduction a row.
#include "zo_i8_device.h"

namespace zo {

// Elements of the weight, widened; 0 beyond the nv that are there.
template <int WT, int K>
__device__ __forceinline__ void read_weight(const typename Elem<WT>::T *w, int64_t nv,
                                            float (&v)[K])
{
    constexpr int V = Elem<WT>::kVec;
#pragma unroll
    for (int h = 0; h < K / V; ++h) {
        u32x4 b = {0, 0, 0, 0};
        if (nv > h * V) b = load16<WT>(w + h * V, nv - h * V);
#pragma unroll
        for (int q = 0; q < V; ++q) v[h * V + q] = elem_of<WT>(b, q);
    }
}

struct NormArgs {
    const void *x, *residual, *weight;
    void *h, *out;
    float *rstd;
    I8View q;
    int64_t rows, cols, ldx, ldr, ldh, ldo;
    float eps, inv_cols;
};

// 1 / sqrt(x) to within a step of binary32: the instruction's value, off by one or two, and
// one Newton step.  x is a normal number or infinite (then 0) or NaN.
__device__ __forceinline__ float inverse_root(float x)
{
    const float y = __builtin_amdgcn_rsqf(x);
    const float e = __builtin_fmaf(-x * y, y, 1.0f);
    return x < INFINITY ? __builtin_fmaf(0.5f * y, e, y) : y;
}

// What h is scaled by before it is multiplied with `rs` (1 and rstd but for extreme rows).
struct Rstd {
    float rstd, pre, rs;
};

// Of rows whose squares binary32 does not hold: from h scaled by a power of two.
template <int GT, int TH, int NV>
__device__ Rstd extreme_rstd(const u32x4 (&w)[NV], float plain, float cols, float eps, float *sum,
                             uint32_t *top)
{
    u32x4 m = {};
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < 4; ++i) m[i] = packed_max<GT>(m[i], w[v][i]);
    const uint32_t a = row_max<TH>(max_in<GT>(m), top);
    if (a == 0 || a >= kInfBits) return {plain, 1.0f, plain};
    const int e = max((int)(a >> 23), 1) - 127;          // exponent of the largest
    const float pre = __builtin_ldexpf(1.0f, -e);
    float ss = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int q = 0; q < Elem<GT>::kVec; ++q) {
            const float y = elem_of<GT>(w[v], q) * pre;
            ss = __builtin_fmaf(y, y, ss);
        }
    ss = row_sum<TH>(ss, sum);
    const double rstd =
        1.0 / __builtin_sqrt(__builtin_ldexp((double)ss / (double)cols, 2 * e) + (double)eps);
    return {(float)rstd, pre, (float)__builtin_ldexp(rstd, e)};
}

// h of a thread's vectors times pre, rs and the weight.
template <int GT, int TH, int NV>
__device__ __forceinline__ void put_out(typename Elem<GT>::T *out, const u32x4 (&w)[NV],
                                        const float (&g)[NV][Elem<GT>::kVec], float pre, float rs,
                                        int cols, int t)
{
    constexpr int K = Elem<GT>::kVec;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        u32x4 x = w[v];
        repack<GT>(x);
        float e[K];
#pragma unroll
        for (int q = 0; q < K; ++q) e[q] = elem_of<GT>(x, q) * pre * rs * g[v][q];
        store_vector<GT>(out, pack16<GT>(e), (v * TH + t) * K, cols);
    }
}

// A row by TH threads: the weight and the row stay in registers.  Workgroups that went on to
// further rows, their loads ahead, were slower (8192 x 1600 bfloat16, all outputs: 27.3 us
// against 24.7).
template <int GT, int WT, int TH, int NV>
__global__ __launch_bounds__(TH == 64 ? 256 : TH) void k_norm(NormArgs a)
{
    using T = typename Elem<GT>::T;
    constexpr int K = Elem<GT>::kVec, TEAMS = TH == 64 ? 4 : 1, NW = TH / 64;
    __shared__ float sum[2][NW];
    __shared__ uint32_t top[2][NW];
    const int t = threadIdx.x % TH, cols = (int)a.cols;
    const int64_t row = (int64_t)blockIdx.x * TEAMS + threadIdx.x / TH;
    if (row >= a.rows) return;                           // whole waves, without barriers
    u32x4 h[NV], o[NV];
    load_row<GT, TH>(h, static_cast<const T *>(a.x) + row * a.ldx, cols, t);
    if (a.residual)
        load_row<GT, TH>(o, static_cast<const T *>(a.residual) + row * a.ldr, cols, t);
    const auto *weight = static_cast<const typename Elem<WT>::T *>(a.weight);
    float g[NV][K];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * TH + t) * K;
        read_weight<WT, K>(weight + c, cols - c, g[v]);
    }
    if (a.residual)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float e[K];
#pragma unroll
            for (int q = 0; q < K; ++q) e[q] = elem_of<GT>(h[v], q) + elem_of<GT>(o[v], q);
            h[v] = pack16<GT>(e);
        }
    float ss = 0.0f;
    uint32_t most = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
        for (int q = 0; q < K; ++q) {
            const float x = elem_of<GT>(h[v], q);
            ss = __builtin_fmaf(x, x, ss);
            most = max(most, mag_bits(x * g[v][q]));
        }
        if (a.h)
            store_vector<GT>(static_cast<T *>(a.h) + row * a.ldh, h[v], (v * TH + t) * K, cols);
        __builtin_amdgcn_sched_barrier(0);
    }
    ss = wave_reduce<OpSum>(ss);
    most = wave_max(most);
    if constexpr (TH > 64) {
        if ((threadIdx.x & 63) == 0) {
            sum[0][threadIdx.x >> 6] = ss;
            top[0][threadIdx.x >> 6] = most;
        }
        __syncthreads();
        ss = group_get<OpSum, NW>(sum[0]);
        most = top[0][0];
#pragma unroll
        for (int i = 1; i < NW; ++i) most = max(most, top[0][i]);
    }
    const float plain = inverse_root(ss * a.inv_cols + a.eps);
    Rstd r = {plain, 1.0f, plain};
    if (!(ss < 0x1p120f) || (ss < 0x1p-60f && a.eps < 0x1p-60f))
        r = extreme_rstd<GT, TH, NV>(h, plain, (float)cols, a.eps, sum[1], top[1]);
    if (a.rstd && t == 0) a.rstd[row] = r.rstd;
    if (a.out) {
        T *out = static_cast<T *>(a.out) + row * a.ldo;
        if (r.pre == 1.0f)
            put_out<GT, TH>(out, h, g, 1.0f, r.rs, cols, t);
        else
            put_out<GT, TH>(out, h, g, r.pre, r.rs, cols, t);
    }
    if (a.q.codes) {
        const Step s = step_of(most);
        if (t == 0) a.q.scales[row] = s.s * r.rstd;
        int8_t *codes = a.q.codes + row * a.q.wide;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * TH + t) * K;
            float e[K];
            repack<GT>(h[v]);
#pragma unroll
            for (int q = 0; q < K; ++q) e[q] = elem_of<GT>(h[v], q) * g[v][q];
            if (c < a.q.wide) store_codes<K>(codes + c, e, s);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

template <int N>
using Int = std::integral_constant<int, N>;

// Calls f(threads of a row, vectors of a thread) for rows of `cols` elements.  GRAD: as the
// backward pass takes them, which keeps more of a row in its registers.  Measured, bfloat16,
// us: forward, 8192 x 1600 with 64 x 4 29.7, 128 x 2 25.2, 256 x 1 24.7; backward, 8192 x 1600
// 128 x 2 27.6, 256 x 1 28.0; 3200 x 4096 256 x 2 29.1, 512 x 1 27.8; 1600 x 8192 512 x 2 33.4,
// 1024 x 1 32.7.
template <int GT, bool GRAD, class F>
static hipError_t with_team(int64_t cols, F &&f)
{
    const int64_t vecs = (cols + 127) / 128 * (128 / Elem<GT>::kVec);
    if (vecs <= 64) return f(Int<64>{}, Int<1>{});
    if (vecs <= 128) return f(Int<64>{}, Int<2>{});
    if (vecs <= 256) return f(Int<(GRAD ? 128 : 256)>{}, Int<(GRAD ? 2 : 1)>{});
    if (vecs <= 512) return f(Int<(GRAD ? 512 : 256)>{}, Int<(GRAD ? 1 : 2)>{});
    if (vecs <= 1024) return f(Int<(GRAD ? 1024 : 512)>{}, Int<(GRAD ? 1 : 2)>{});
    if (vecs <= 2048) return f(Int<1024>{}, Int<2>{});
    if constexpr (GT == GT_F32)                          // 32768 columns at most
        if (vecs > 4096) return f(Int<1024>{}, Int<8>{});
    return f(Int<1024>{}, Int<4>{});
}

// Calls f(element type, weight's type).
template <class F>
static hipError_t with_types(int32_t dtype, int32_t weight, F &&f)
{
    return with_elem_type(dtype, [&](auto g) {
        if (weight == GT_F32) return f(g, std::integral_constant<int, GT_F32>{});
        return f(g, g);
    });
}

hipError_t launch_norm(const zo_norm &a, const I8View &q, hipStream_t st)
{
    return with_types(a.dtype, a.weight_dtype, [&](auto g, auto wg) {
        constexpr int GT = decltype(g)::value, WT = decltype(wg)::value;
        using T = typename Elem<GT>::T;
        return with_team<GT, false>(a.cols, [&](auto th, auto nv) {
            constexpr int TH = decltype(th)::value, NV = decltype(nv)::value;
            constexpr int TEAMS = TH == 64 ? 4 : 1;
            hipError_t e = hipSuccess;
            for (int64_t r = 0; r < a.rows && e == hipSuccess; r += kLaunchRows) {
                const int64_t part = a.rows - r < kLaunchRows ? a.rows - r : kLaunchRows;
                NormArgs n = {static_cast<const T *>(a.x) + r * a.ldx,
                              a.residual ? static_cast<const T *>(a.residual) + r * a.ldr : nullptr,
                              a.weight,
                              a.h ? static_cast<T *>(a.h) + r * a.ldh : nullptr,
                              a.out ? static_cast<T *>(a.out) + r * a.ldo : nullptr,
                              a.rstd ? a.rstd + r : nullptr,
                              q, part, a.cols, a.ldx, a.ldr, a.ldh, a.ldo, a.eps,
                              1.0f / (float)a.cols};
                if (q.codes) {
                    n.q.codes += r * q.wide;
                    n.q.scales += r;
                }
                e = start(k_norm<GT, WT, TH, NV>, (part + TEAMS - 1) / TEAMS, TH == 64 ? 256 : TH,
                          0, st, n);
            }
            return e;
        });
    });
}

// ---------------------------------------------------------------------------

struct NormGradArgs {
    const void *dy, *h, *weight, *dh;
    const float *rstd;
    void *dx;
    float *dw;                   // [blocks][cols], or the result of one block
    int64_t rows, cols, lddy, ldh, lddh, lddx, per;
    float inv_cols;
};

// Rows [blockIdx.x * per, + per), by TEAMS teams of TH threads: dx, and the rows' part of dw in
// registers.  The workgroups are few, as their parts of dw go through memory, so a team keeps a
// row ahead on its way, and the weight in registers (8192 x 1600 bfloat16 with dh: without 33.3
// us, dy and h ahead 30.0, dh too 27.2, of which the joining of dw takes 4).
template <int GT, int WT, int TH, int NV, int TEAMS>
__global__ __launch_bounds__(TH *TEAMS, 2) void k_norm_grad(NormGradArgs a)
{
    using T = typename Elem<GT>::T;
    constexpr int K = Elem<GT>::kVec, NW = TH / 64;
    __shared__ float sum[2][TEAMS][NW];
    __shared__ float joined[TEAMS > 1 ? TEAMS - 1 : 1][TEAMS > 1 ? TH * NV * K : 1];
    const int t = threadIdx.x % TH, team = threadIdx.x / TH, cols = (int)a.cols;
    const int64_t from = blockIdx.x * a.per, to = min(a.rows, from + a.per);
    const int turns = (int)((to - from + TEAMS - 1) / TEAMS);
    const auto *weight = static_cast<const typename Elem<WT>::T *>(a.weight);
    constexpr bool HELD = NV <= 2;               // the weight in registers, a row ahead
    float dw[NV][K] = {}, g[HELD ? NV : 1][K];
    auto weight_of = [&](int v, float(&w)[K]) __attribute__((always_inline)) {
        const int c = (v * TH + t) * K;
        read_weight<WT, K>(weight + c, cols - c, w);
    };
    u32x4 d[NV], h[NV], o[NV], d1[HELD ? NV : 1], h1[HELD ? NV : 1], o1[HELD ? NV : 1];
    float rstd1 = 0.0f;
    // a team without a row has none of its elements, and stores nothing
    auto row_of = [&](int turn) { return min(from + turn * TEAMS + team, to - 1); };
    auto size_of = [&](int turn) { return from + turn * TEAMS + team < to ? cols : 0; };
    auto fetch = [&](int turn, auto &d, auto &h, auto &o, float &rstd) __attribute__((always_inline)) {
        const int64_t r = row_of(turn);
        load_row<GT, TH>(d, static_cast<const T *>(a.dy) + r * a.lddy, size_of(turn), t);
        load_row<GT, TH>(h, static_cast<const T *>(a.h) + r * a.ldh, size_of(turn), t);
        rstd = a.rstd[r];
        if (a.dh && a.dx)
            load_row<GT, TH>(o, static_cast<const T *>(a.dh) + r * a.lddh, size_of(turn), t);
    };
    if constexpr (HELD) {
        fetch(0, d1, h1, o1, rstd1);
#pragma unroll
        for (int v = 0; v < NV; ++v) weight_of(v, g[v]);
    }
    for (int turn = 0; turn < turns; ++turn) {
        const int64_t r = row_of(turn);
        float rstd;
        if constexpr (HELD) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                d[v] = d1[v];
                h[v] = h1[v];
                o[v] = o1[v];
            }
            rstd = rstd1;
        } else {
            fetch(turn, d, h, o, rstd);
        }
        if constexpr (HELD)
            if (turn + 1 < turns) fetch(turn + 1, d1, h1, o1, rstd1);
        float dot = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float(&w)[K] = g[HELD ? v : 0];
            if constexpr (!HELD) weight_of(v, w);
#pragma unroll
            for (int q = 0; q < K; ++q) {
                const float y = elem_of<GT>(d[v], q), n = elem_of<GT>(h[v], q) * rstd;
                dot = __builtin_fmaf(y * w[q], n, dot);
                dw[v][q] = __builtin_fmaf(y, n, dw[v][q]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (!a.dx) continue;                     // the same for all
        dot = wave_reduce<OpSum>(dot);
        if constexpr (TH > 64) {
            float *s = sum[turn & 1][team];
            if ((t & 63) == 0) s[t >> 6] = dot;
            __syncthreads();
            dot = group_get<OpSum, NW>(s);
        }
        const float mean = dot * a.inv_cols;
        T *px = static_cast<T *>(a.dx) + r * a.lddx;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float(&w)[K] = g[HELD ? v : 0];
            if constexpr (!HELD) weight_of(v, w);
            float e[K];
            repack<GT>(d[v]);
            repack<GT>(h[v]);
#pragma unroll
            for (int q = 0; q < K; ++q) {
                const float n = elem_of<GT>(h[v], q) * rstd;
                const float x = __builtin_fmaf(-n, mean, elem_of<GT>(d[v], q) * w[q]);
                e[q] = a.dh ? __builtin_fmaf(rstd, x, elem_of<GT>(o[v], q)) : rstd * x;
            }
            store_vector<GT>(px, pack16<GT>(e), (v * TH + t) * K, size_of(turn));
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if (!a.dw) return;
    if constexpr (TEAMS > 1) {
        if (team > 0)
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int q = 0; q < K; ++q) joined[team - 1][(v * K + q) * TH + t] = dw[v][q];
        __syncthreads();
        if (team > 0) return;
#pragma unroll 1
        for (int k = 0; k < TEAMS - 1; ++k)
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int q = 0; q < K; ++q) dw[v][q] += joined[k][(v * K + q) * TH + t];
    }
    float *to_dw = a.dw + (int64_t)blockIdx.x * cols;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * TH + t) * K;
#pragma unroll
        for (int q = 0; q < K; ++q)
            if (c + q < cols) to_dw[c + q] = dw[v][q];
    }
}

// dw from the blocks' parts: 16 columns a workgroup, the blocks in 64 slices, joined by
// twos.
__global__ __launch_bounds__(1024) void k_norm_dw(const float *__restrict__ work, int64_t blocks,
                                                  int64_t cols, float *__restrict__ dw)
{
    __shared__ float s[64][16];
    const int i = threadIdx.x & 15, slice = threadIdx.x >> 4;
    const int64_t c = (int64_t)blockIdx.x * 16 + i;
    float v = 0.0f;
    if (c < cols)
#pragma unroll 8
        for (int64_t b = slice; b < blocks; b += 64) v += work[b * cols + c];
    s[slice][i] = v;
    for (int half = 32; half; half /= 2) {
        __syncthreads();
        if (slice < half) s[slice][i] = v = v + s[slice + half][i];
    }
    if (slice == 0 && c < cols) dw[c] = v;
}

static int64_t rows_a_block(int64_t rows)
{
    const int64_t most = rows / 16 + 64 < 512 ? rows / 16 + 64 : 512;
    return (rows + most - 1) / most;
}

int64_t norm_grad_blocks(int64_t rows)
{
    if (rows == 0) return 0;
    const int64_t per = rows_a_block(rows);
    return (rows + per - 1) / per;
}

hipError_t launch_norm_grad(const zo_norm_back &a, hipStream_t st)
{
    const int64_t blocks = a.dw ? norm_grad_blocks(a.rows) : 0;
    if (a.rows > 0) {
        const hipError_t e = with_types(a.dtype, a.weight_dtype, [&](auto g, auto wg) {
            constexpr int GT = decltype(g)::value, WT = decltype(wg)::value;
            using T = typename Elem<GT>::T;
            return with_team<GT, true>(a.cols, [&](auto th, auto nv) {
                constexpr int TH = decltype(th)::value, NV = decltype(nv)::value;
                constexpr int TEAMS = TH < 256 ? 256 / TH : 1;
                const auto kernel = k_norm_grad<GT, WT, TH, NV, TEAMS>;
                NormGradArgs n = {a.dy, a.h, a.weight, a.dh, a.rstd, a.dx,
                                  blocks == 1 ? a.dw : static_cast<float *>(a.work),
                                  a.rows, a.cols, a.lddy, a.ldh, a.lddh, a.lddx,
                                  rows_a_block(a.rows), 1.0f / (float)a.cols};
                if (a.dw) return start(kernel, blocks, TH * TEAMS, 0, st, n);
                hipError_t e = hipSuccess;
                n.dw = nullptr;
                n.per = TEAMS;
                for (int64_t r = 0; r < a.rows && e == hipSuccess; r += kLaunchRows) {
                    n.rows = a.rows - r < kLaunchRows ? a.rows - r : kLaunchRows;
                    n.dy = static_cast<const T *>(a.dy) + r * a.lddy;
                    n.h = static_cast<const T *>(a.h) + r * a.ldh;
                    n.dh = a.dh ? static_cast<const T *>(a.dh) + r * a.lddh : nullptr;
                    n.rstd = a.rstd + r;
                    n.dx = static_cast<T *>(a.dx) + r * a.lddx;
                    e = start(kernel, (n.rows + TEAMS - 1) / TEAMS, TH * TEAMS, 0, st, n);
                }
                return e;
            });
        });
        if (e != hipSuccess) return e;
    }
    if (!a.dw || blocks == 1) return hipSuccess;
    return start(k_norm_dw, (a.cols + 15) / 16, 1024, 0, st, static_cast<const float *>(a.work),
                 blocks, a.cols, a.dw);
}

}  // namespace zo
