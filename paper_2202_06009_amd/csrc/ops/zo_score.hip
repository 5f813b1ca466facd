// zo_score.hip -- log probabilities of tokens, the rows' entropies and most likely
// alternatives, and the gradient of the logits.
//
// With m the row's largest logit, t = (z - m) log2(e) / tau and e = 2^t:
//   S = sum e, U = sum e t; log p = (z - m) / tau - ln S, entropy = ln S - ln 2 U / S.
// The difference comes first, so that logits of any size keep their distances.  Terms of
// t below kLeast add nothing to either sum (2^t is 0), so t is clamped there in U and
// logits of -infinity need no case of their own.
//
// One workgroup per row; the bound is reading the logits once (k_score: the row stays in
// registers).  The alternatives are found as zo_top.hip finds them.
#include "zo_top_device.h"

namespace zo {

constexpr float kLeast = -256.0f;

// A row's results.
struct RowScore {
    float m, log_s, entropy;
};

__device__ __forceinline__ float log_prob(float z, const RowScore &r, float tau)
{
    if (r.log_s != r.log_s) return NAN;
    return z == -INFINITY ? -INFINITY : (z - r.m) / tau - r.log_s;
}

struct PutScore {
    const zo_score &a;
    int64_t row;
    RowScore r;
    __device__ __forceinline__ void operator()(int rank, uint64_t key) const
    {
        a.values[row * a.top + rank] = log_prob(key_value((uint32_t)(key >> 32)), r, a.tau);
        a.columns[row * a.top + rank] = (int32_t)~(uint32_t)key;
    }
};

// From the sums; s of NaN: a NaN or +infinity is among the logits.
__device__ __forceinline__ RowScore row_score(float m, float s, float u)
{
    if (s != s) return {NAN, NAN, NAN};
    if (m == -INFINITY) return {m, m, 0.0f};
    const float log_s = logf(s);
    return {m, log_s, fmaxf(log_s - kLn2 * (u / s), 0.0f)};
}

// The row's token, or -1, and its logit.
struct Token {
    int32_t at;
    float z;
};

template <int GT>
__device__ __forceinline__ Token read_token(const zo_score &a, int64_t row,
                                            const typename Elem<GT>::T *z)
{
    int32_t at = a.tokens ? a.tokens[row] : -1;
    if (at < 0 || at >= a.vocab) at = -1;
    return {at, at >= 0 ? widen<GT>(z[at]) : 0.0f};
}

// By one thread.
__device__ __forceinline__ void put_row(const zo_score &a, int64_t row, const RowScore &r,
                                        const Token &token)
{
    if (a.tokens) a.logp[row] = token.at >= 0 ? log_prob(token.z, r, a.tau) : 0.0f;
    if (a.stats) {
        a.stats[row * 3] = r.m;
        a.stats[row * 3 + 1] = r.log_s;
        a.stats[row * 3 + 2] = r.entropy;
    }
}

__device__ __forceinline__ void add_term(float z, float b, float c, float &s, float &u)
{
    const float t = (z - b) * c, e = exp2_hw(t);
    s += e;
    u = __builtin_fmaf(e, fmaxf(t, kLeast), u);
}

template <int GT, int TH, int NV>
__global__ __launch_bounds__(TH, TH == 768 ? 6 : 4) void k_score(zo_score a)
{
    constexpr int K = Elem<GT>::kVec, NW = TH / 64;
    __shared__ TopShared<TH> sh;
    __shared__ float more[NW];
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x, V = a.vocab;
    const auto *z = static_cast<const typename Elem<GT>::T *>(a.z) + row * a.ldz;
    const Token token = read_token<GT>(a, row, z);
    Resident<GT, TH, NV> x;
    x.load(z, V);
    for (int i = tid; i < 256; i += TH) sh.hist[i] = 0;
    if (tid == 0) sh.sel[3] = 0;

    GroupMaxima m = {x.last, {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, 0};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        if (v * TH < x.vecs)                             // the same for all threads
            m.of[v % kGroups] = fmaxf(m.of[v % kGroups], max_of<GT>(x.w[v]));
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        m.all = fmaxf(m.all, m.of[g]);
        if (x.at(g) < x.vecs) m.there |= 1u << g;
    }
    group_put<OpMax>(m.all, sh.red[0]);
    __syncthreads();
    const float M = group_get<OpMax, NW>(sh.red[0]), b = M == -INFINITY ? 0.0f : M;
    const float c = log2_factor(a.tau);
    float s = 0.0f, u = 0.0f;
    add_term(x.last, b, c, s, u);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        repack<GT>(x.w[v]);
        if (v * TH < x.vecs) {
#pragma unroll
            for (int q = 0; q < K; ++q) add_term(elem_of<GT>(x.w[v], q), b, c, s, u);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    group_put<OpSum>(s, sh.red[2]);
    group_put<OpSum>(u, more);

    // as k_top
    const int groups = min(x.vecs, a.top <= TH / kGroups ? TH : TH * kGroups);
    const bool all = 2 * a.top > groups && V <= kRoom, unbound = !all && groups < a.top;
    uint32_t least = 0;
    if (a.top == 0 || all || unbound)
        __syncthreads();
    else
        least = find_bound<TH>(sh, (uint32_t)a.top, M, m);
    const float total = group_get<OpSum, NW>(sh.red[2]);
    const RowScore r = row_score(M, total, group_get<OpSum, NW>(more));
    if (tid == 0) put_row(a, row, r, token);
    if (a.top == 0) return;
    bool counted = total != total || unbound;
    if (!counted) {                                      // collect
        const float bound = key_value(least);
        if (x.has_last(V) && (all || x.last >= bound)) offer<TH>(sh, x.last, x.last_column());
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            repack<GT>(x.w[v]);
            if (x.at(v) < x.vecs && (all || max_of<GT>(x.w[v]) >= bound)) {
#pragma unroll
                for (int q = 0; q < K; ++q) {
                    const float e = elem_of<GT>(x.w[v], q);
                    if (all || e >= bound) offer<TH>(sh, e, x.at(v) * K + q);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        __syncthreads();
        counted = sh.sel[3] > kRoom;
    }
    if (counted)
        select_row<GT, TH>(z, V, a.top, sh, PutScore{a, row, r});
    else
        sort_out<TH>(sh, (int)sh.sel[3], a.top, PutScore{a, row, r});
}

// Rows that do not fit registers: the largest logits of the groups first, then, in a second
// read, the sums and the candidates.
template <int GT>
__global__ __launch_bounds__(1024) void k_score_long(zo_score a)
{
    constexpr int TH = 1024, NW = TH / 64, K = Elem<GT>::kVec;
    __shared__ TopShared<TH> sh;
    __shared__ float more[NW];
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x, V = a.vocab;
    const auto *z = static_cast<const typename Elem<GT>::T *>(a.z) + row * a.ldz;
    const Token token = read_token<GT>(a, row, z);
    const float c = log2_factor(a.tau);
    for (int i = tid; i < 256; i += TH) sh.hist[i] = 0;
    if (tid == 0) sh.sel[3] = 0;
    GroupMaxima m = {-INFINITY, {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, 0};
    for (int64_t i0 = (int64_t)tid * K; i0 < V; i0 += kGroups * TH * K) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int64_t i = i0 + g * TH * K;
            m.of[g] = fmaxf(m.of[g],
                            max_of<GT>(load16<GT>(z + i, V - i, kNegInf<GT> & kElemMask<GT>)));
            if (i < V) m.there |= 1u << g;
        }
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) m.all = fmaxf(m.all, m.of[g]);
    group_put<OpMax>(m.all, sh.red[0]);
    __syncthreads();
    const float M = group_get<OpMax, NW>(sh.red[0]), b = M == -INFINITY ? 0.0f : M;
    const bool wanted = a.top > 0;
    const float bound = wanted ? key_value(find_bound<TH>(sh, (uint32_t)a.top, M, m)) : 0.0f;
    float s = 0.0f, u = 0.0f;
    for (int64_t i = (int64_t)tid * K; i < V; i += TH * K) {
        const u32x4 w = load16<GT>(z + i, V - i, kNegInf<GT> & kElemMask<GT>);
#pragma unroll
        for (int q = 0; q < K; ++q) add_term(elem_of<GT>(w, q), b, c, s, u);
        if (wanted && max_of<GT>(w) >= bound) {
#pragma unroll
            for (int q = 0; q < K; ++q) {
                const float e = elem_of<GT>(w, q);
                if (e >= bound && i + q < V) offer<TH>(sh, e, i + q);
            }
        }
    }
    group_put<OpSum>(s, sh.red[2]);
    group_put<OpSum>(u, more);
    __syncthreads();
    const float total = group_get<OpSum, NW>(sh.red[2]);
    const RowScore r = row_score(M, total, group_get<OpSum, NW>(more));
    if (tid == 0) put_row(a, row, r, token);
    if (!wanted) return;
    const uint32_t n = sh.sel[3];
    if (total != total || n > kRoom)
        select_row<GT, TH>(z, V, a.top, sh, PutScore{a, row, r});
    else
        sort_out<TH>(sh, (int)n, a.top, PutScore{a, row, r});
}

static hipError_t launch_rows(const zo_score &a, int gt, hipStream_t st)
{
    return with_elem_type(gt, [&](auto g) {
        constexpr int GT = decltype(g)::value;
        const int64_t vecs = a.vocab / Elem<GT>::kVec;
        auto go = [&](auto th, auto nv) {
            constexpr int TH = decltype(th)::value, NV = decltype(nv)::value;
            return start(k_score<GT, TH, NV>, a.rows, TH, 0, st, a);
        };
        using std::integral_constant;
        if (vecs > 1024 * 16) return start(k_score_long<GT>, a.rows, 1024, 0, st, a);
        // as for the top logits
        if (a.top <= 256 && vecs <= 256 * 4)
            return go(integral_constant<int, 256>{}, integral_constant<int, 4>{});
        if (a.top <= 256 && vecs <= 256 * 8)
            return go(integral_constant<int, 256>{}, integral_constant<int, 8>{});
        if (a.top <= 512 && vecs <= 512 * 8)
            return go(integral_constant<int, 512>{}, integral_constant<int, 8>{});
        if (a.top <= 768 && vecs <= 768 * 9)
            return go(integral_constant<int, 768>{}, integral_constant<int, 9>{});
        if (a.top <= 768 && vecs <= 768 * 11)
            return go(integral_constant<int, 768>{}, integral_constant<int, 11>{});
        return go(integral_constant<int, 1024>{}, integral_constant<int, 16>{});
    });
}

hipError_t launch_score(const zo_score &a, hipStream_t st)
{
    const int64_t size = a.dtype == GT_F32 ? 4 : 2;
    for (int64_t r = 0; r < a.rows; r += kLaunchRows) {
        zo_score part = a;
        part.rows = a.rows - r < kLaunchRows ? a.rows - r : kLaunchRows;
        part.z = static_cast<const char *>(a.z) + r * a.ldz * size;
        if (a.tokens) {
            part.tokens += r;
            part.logp += r;
        }
        if (a.stats) part.stats += r * 3;
        if (a.top) {
            part.values += r * a.top;
            part.columns += r * a.top;
        }
        const hipError_t e = launch_rows(part, a.dtype, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// ---------------------------------------------------------------------------

constexpr int kGradVecs = 4;

// With t as above less log2 S, p = 2^t and log p = ln 2 t:
//   dz = p (k0 + k1 t) / tau, k0 = -(dlogp + dentropy entropy), k1 = -ln 2 dentropy,
// and at the token's column dlogp (1 - p) by expm1: 1 - p keeps its digits.
// Workgroup (row, run of 256 kGradVecs vectors).
template <int GT>
__global__ __launch_bounds__(256) void k_score_grad(zo_score_back a, uint32_t runs)
{
    using T = typename Elem<GT>::T;
    constexpr int K = Elem<GT>::kVec;
    const int64_t row = blockIdx.x / runs, V = a.vocab;
    const int64_t first = ((int64_t)(blockIdx.x % runs) * 256 * kGradVecs + threadIdx.x) * K;
    const T *z = static_cast<const T *>(a.z) + row * a.ldz;
    T *dz = static_cast<T *>(a.dz) + row * a.lddz;
    int32_t token = a.tokens ? a.tokens[row] : -1;
    if (token < 0 || token >= V) token = -1;
    const float dlogp = a.dlogp && token >= 0 ? a.dlogp[row] : 0.0f;
    const float dh = a.dentropy ? a.dentropy[row] : 0.0f;
    const float m = a.stats[row * 3], log_s = a.stats[row * 3 + 1], h = a.stats[row * 3 + 2];
    const bool nothing = (dlogp == 0.0f && dh == 0.0f) || m == -INFINITY, bad = log_s != log_s;
    if (nothing || bad) {
        float e[K];
#pragma unroll
        for (int q = 0; q < K; ++q) e[q] = nothing ? 0.0f : NAN;
#pragma unroll
        for (int v = 0; v < kGradVecs; ++v) {
            const int64_t i = first + v * 256 * K;
            if (i < V) store16<GT>(dz + i, pack16<GT>(e), V - i);
        }
        return;
    }
    const float c = log2_factor(a.tau), l2 = log_s * kLog2e;
    const float k0 = -(dlogp + dh * h), k1 = -kLn2 * dh, scale = 1.0f / a.tau;
    u32x4 w[kGradVecs];
#pragma unroll
    for (int v = 0; v < kGradVecs; ++v) {
        const int64_t i = first + v * 256 * K;
        if (i < V) w[v] = load16<GT>(z + i, V - i);
    }
#pragma unroll
    for (int v = 0; v < kGradVecs; ++v) {
        const int64_t i = first + v * 256 * K;
        if (i >= V) continue;
        float e[K];
#pragma unroll
        for (int q = 0; q < K; ++q) {
            const float t = fmaxf(__builtin_fmaf(elem_of<GT>(w[v], q) - m, c, -l2), kLeast);
            e[q] = exp2_hw(t) * __builtin_fmaf(k1, t, k0) * scale;
        }
        if (token >= i && token < i + K) {
#pragma unroll
            for (int q = 0; q < K; ++q)
                if (token == i + q) {
                    const float x = elem_of<GT>(w[v], q);
                    const float lp = x == -INFINITY ? x : (x - m) / a.tau - log_s;
                    const float t = fmaxf(lp * kLog2e, kLeast);
                    e[q] = (-dlogp * expm1f(lp) - dh * exp2_hw(t) * (t * kLn2 + h)) * scale;
                }
        }
        store16<GT>(dz + i, pack16<GT>(e), V - i);
    }
}

hipError_t launch_score_grad(const zo_score_back &a, hipStream_t st)
{
    return with_elem_type(a.dtype, [&](auto g) {
        constexpr int GT = decltype(g)::value, RUN = 256 * kGradVecs * Elem<GT>::kVec;
        using T = typename Elem<GT>::T;
        const int64_t runs = (a.vocab + RUN - 1) / RUN, most = ((1 << 22) + runs - 1) / runs;
        for (int64_t r = 0; r < a.rows; r += most) {
            zo_score_back part = a;
            part.rows = a.rows - r < most ? a.rows - r : most;
            part.z = static_cast<const T *>(a.z) + r * a.ldz;
            part.dz = static_cast<T *>(a.dz) + r * a.lddz;
            part.stats += r * 3;
            if (a.tokens) part.tokens += r;
            if (a.dlogp) part.dlogp += r;
            if (a.dentropy) part.dentropy += r;
            const hipError_t e =
                start(k_score_grad<GT>, part.rows * runs, 256, 0, st, part, (uint32_t)runs);
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    });
}

}  // namespace zo
