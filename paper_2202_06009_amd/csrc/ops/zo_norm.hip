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
    float eps;
};

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

template <int GT, int WT, int TH, int NV>
__global__ __launch_bounds__(TH < 256 ? 256 : TH) void k_norm(NormArgs a)
{
    using T = typename Elem<GT>::T;
    constexpr int K = Elem<GT>::kVec, TEAMS = TH < 256 ? 256 / TH : 1, NW = TH / 64;
    __shared__ float sum[2][NW];
    __shared__ uint32_t top[2][NW];
    const int t = threadIdx.x % TH;
    const int64_t row = (int64_t)blockIdx.x * TEAMS + (TEAMS > 1 ? threadIdx.x / TH : 0);
    if (row >= a.rows) return;                           // whole waves, without barriers
    const T *x = static_cast<const T *>(a.x) + row * a.ldx;
    const auto *weight = static_cast<const typename Elem<WT>::T *>(a.weight);
    const int64_t cols = a.cols;
    u32x4 w[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int64_t c = (int64_t)(v * TH + t) * K;
        w[v] = u32x4{0, 0, 0, 0};
        if (c < cols) w[v] = load16<GT>(x + c, cols - c);
    }
    if (a.residual) {
        const T *r = static_cast<const T *>(a.residual) + row * a.ldr;
        u32x4 o[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int64_t c = (int64_t)(v * TH + t) * K;
            o[v] = u32x4{0, 0, 0, 0};
            if (c < cols) o[v] = load16<GT>(r + c, cols - c);
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float e[K];
#pragma unroll
            for (int q = 0; q < K; ++q) e[q] = elem_of<GT>(w[v], q) + elem_of<GT>(o[v], q);
            w[v] = pack16<GT>(e);
        }
    }
    if (a.h) {
        T *h = static_cast<T *>(a.h) + row * a.ldh;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int64_t c = (int64_t)(v * TH + t) * K;
            if (c < cols) store16<GT>(h + c, w[v], cols - c);
        }
    }
    float ss = 0.0f;
    uint32_t most = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int64_t c = (int64_t)(v * TH + t) * K;
#pragma unroll
        for (int q = 0; q < K; ++q) {
            const float h = elem_of<GT>(w[v], q);
            ss = __builtin_fmaf(h, h, ss);
        }
        if (a.q.codes) {
            float g[K];
            read_weight<WT, K>(weight + c, cols - c, g);
#pragma unroll
            for (int q = 0; q < K; ++q) most = max(most, mag_bits(elem_of<GT>(w[v], q) * g[q]));
        }
    }
    ss = row_sum<TH>(ss, sum[0]);
    const float plain = 1.0f / sqrtf(ss / (float)cols + a.eps);
    Rstd r = {plain, 1.0f, plain};
    if (!(ss < 0x1p120f) || (ss < 0x1p-60f && a.eps < 0x1p-60f))
        r = extreme_rstd<GT, TH, NV>(w, plain, (float)cols, a.eps, sum[1], top[0]);
    if (a.rstd && t == 0) a.rstd[row] = r.rstd;
    if (a.out) {
        T *out = static_cast<T *>(a.out) + row * a.ldo;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int64_t c = (int64_t)(v * TH + t) * K;
            float g[K], e[K];
            read_weight<WT, K>(weight + c, cols - c, g);
#pragma unroll
            for (int q = 0; q < K; ++q) e[q] = elem_of<GT>(w[v], q) * r.pre * r.rs * g[q];
            if (c < cols) store16<GT>(out + c, pack16<GT>(e), cols - c);
        }
    }
    if (a.q.codes) {
        const Step s = step_of(row_max<TH>(most, top[1]));
        if (t == 0) a.q.scales[row] = s.s * r.rstd;
        int8_t *codes = a.q.codes + row * a.q.wide;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int64_t c = (int64_t)(v * TH + t) * K;
            float g[K], e[K];
            read_weight<WT, K>(weight + c, cols - c, g);
#pragma unroll
            for (int q = 0; q < K; ++q) e[q] = elem_of<GT>(w[v], q) * g[q];
            if (c < a.q.wide) store_codes<K>(codes + c, e, s);
        }
    }
}

// Calls f(threads of a row, vectors of a thread) for rows of `cols` elements.
template <int GT, class F>
static hipError_t with_team(int64_t cols, F &&f)
{
    using std::integral_constant;
    const int64_t vecs = (cols + 127) / 128 * (128 / Elem<GT>::kVec);
    if (vecs <= 64) return f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    if (vecs <= 128) return f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    if (vecs <= 256) return f(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    if (vecs <= 512) return f(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    if (vecs <= 1024) return f(integral_constant<int, 256>{}, integral_constant<int, 4>{});
    if constexpr (GT == GT_F32)                          // 32768 columns at most
        if (vecs > 4096) return f(integral_constant<int, 1024>{}, integral_constant<int, 8>{});
    return f(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
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
        return with_team<GT>(a.cols, [&](auto th, auto nv) {
            constexpr int TH = decltype(th)::value, NV = decltype(nv)::value;
            constexpr int TEAMS = TH < 256 ? 256 / TH : 1;
            hipError_t e = hipSuccess;
            for (int64_t r = 0; r < a.rows && e == hipSuccess; r += kLaunchRows) {
                const int64_t part = a.rows - r < kLaunchRows ? a.rows - r : kLaunchRows;
                NormArgs n = {static_cast<const T *>(a.x) + r * a.ldx,
                              a.residual ? static_cast<const T *>(a.residual) + r * a.ldr : nullptr,
                              a.weight,
                              a.h ? static_cast<T *>(a.h) + r * a.ldh : nullptr,
                              a.out ? static_cast<T *>(a.out) + r * a.ldo : nullptr,
                              a.rstd ? a.rstd + r : nullptr,
                              q, part, a.cols, a.ldx, a.ldr, a.ldh, a.ldo, a.eps};
                if (q.codes) {
                    n.q.codes += r * q.wide;
                    n.q.scales += r;
                }
                e = start(k_norm<GT, WT, TH, NV>, (part + TEAMS - 1) / TEAMS, TH < 256 ? 256 : TH,
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
};

// Rows [blockIdx.x * per, + per): dx, and the rows' part of dw in registers.
template <int GT, int WT, int TH, int NV>
__global__ __launch_bounds__(TH < 256 ? 256 : TH) void k_norm_grad(NormGradArgs a)
{
    using T = typename Elem<GT>::T;
    constexpr int K = Elem<GT>::kVec, TEAMS = TH < 256 ? 256 / TH : 1, NW = TH / 64;
    __shared__ float sum[2][NW];
    __shared__ float joined[TEAMS > 1 ? TEAMS - 1 : 1][TEAMS > 1 ? TH * NV * K : 1];
    const int t = threadIdx.x % TH, team = TEAMS > 1 ? threadIdx.x / TH : 0;
    const int64_t cols = a.cols, from = blockIdx.x * a.per, to = min(a.rows, from + a.per);
    const auto *weight = static_cast<const typename Elem<WT>::T *>(a.weight);
    float dw[NV][K] = {};
    int turn = 0;
    for (int64_t r = from + team; r < to; r += TEAMS, turn ^= 1) {
        const T *pd = static_cast<const T *>(a.dy) + r * a.lddy;
        const T *ph = static_cast<const T *>(a.h) + r * a.ldh;
        u32x4 d[NV], h[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int64_t c = (int64_t)(v * TH + t) * K;
            d[v] = h[v] = u32x4{0, 0, 0, 0};
            if (c < cols) {
                d[v] = load16<GT>(pd + c, cols - c);
                h[v] = load16<GT>(ph + c, cols - c);
            }
        }
        const float rstd = a.rstd[r];
        float dot = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int64_t c = (int64_t)(v * TH + t) * K;
            float w[K];
            read_weight<WT, K>(weight + c, cols - c, w);
#pragma unroll
            for (int q = 0; q < K; ++q) {
                const float y = elem_of<GT>(d[v], q), n = elem_of<GT>(h[v], q) * rstd;
                dot = __builtin_fmaf(y * w[q], n, dot);
                dw[v][q] = __builtin_fmaf(y, n, dw[v][q]);
            }
        }
        const float mean = row_sum<TH>(dot, sum[turn]) / (float)cols;
        if (!a.dx) continue;
        T *px = static_cast<T *>(a.dx) + r * a.lddx;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int64_t c = (int64_t)(v * TH + t) * K;
            if (c >= cols) continue;
            u32x4 o = {0, 0, 0, 0};
            if (a.dh) o = load16<GT>(static_cast<const T *>(a.dh) + r * a.lddh + c, cols - c);
            float w[K], e[K];
            read_weight<WT, K>(weight + c, cols - c, w);
#pragma unroll
            for (int q = 0; q < K; ++q) {
                const float n = elem_of<GT>(h[v], q) * rstd;
                const float g = __builtin_fmaf(-n, mean, elem_of<GT>(d[v], q) * w[q]);
                e[q] = a.dh ? __builtin_fmaf(rstd, g, elem_of<GT>(o, q)) : rstd * g;
            }
            store16<GT>(px + c, pack16<GT>(e), cols - c);
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
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int q = 0; q < K; ++q)
#pragma unroll
                for (int k = 0; k < TEAMS - 1; ++k) dw[v][q] += joined[k][(v * K + q) * TH + t];
    }
    float *to_dw = a.dw + blockIdx.x * cols;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int64_t c = (int64_t)(v * TH + t) * K;
#pragma unroll
        for (int q = 0; q < K; ++q)
            if (c + q < cols) to_dw[c + q] = dw[v][q];
    }
}

// dw from the blocks' parts: 32 columns a workgroup, the blocks in 32 slices, joined in a
// fixed order.
__global__ __launch_bounds__(1024) void k_norm_dw(const float *__restrict__ work, int64_t blocks,
                                                  int64_t cols, float *__restrict__ dw)
{
    __shared__ float s[32][32];
    const int i = threadIdx.x & 31, slice = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + i;
    float v = 0.0f;
    if (c < cols)
#pragma unroll 8
        for (int64_t b = slice; b < blocks; b += 32) v += work[b * cols + c];
    s[slice][i] = v;
    __syncthreads();
    if (slice == 0 && c < cols) {
#pragma unroll
        for (int k = 1; k < 32; ++k) v += s[k][i];
        dw[c] = v;
    }
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
    const int64_t blocks = norm_grad_blocks(a.rows);
    if (blocks > 0) {
        const hipError_t e = with_types(a.dtype, a.weight_dtype, [&](auto g, auto wg) {
            constexpr int GT = decltype(g)::value, WT = decltype(wg)::value;
            return with_team<GT>(a.cols, [&](auto th, auto nv) {
                constexpr int TH = decltype(th)::value, NV = decltype(nv)::value;
                const NormGradArgs n = {a.dy, a.h, a.weight, a.dh, a.rstd, a.dx,
                                        !a.dw || blocks == 1 ? a.dw : static_cast<float *>(a.work),
                                        a.rows, a.cols, a.lddy, a.ldh, a.lddh, a.lddx,
                                        rows_a_block(a.rows)};
                return start(k_norm_grad<GT, WT, TH, NV>, blocks, TH < 256 ? 256 : TH, 0, st, n);
            });
        });
        if (e != hipSuccess) return e;
    }
    if (!a.dw || blocks == 1) return hipSuccess;
    return start(k_norm_dw, (a.cols + 31) / 32, 1024, 0, st, static_cast<const float *>(a.work),
                 blocks, a.cols, a.dw);
}

}  // namespace zo
