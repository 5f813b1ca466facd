// zo_top.hip -- the largest logits of every row, their columns, and the row's
// log-sum-exp.
//
// One workgroup per row; the bound is reading the logits once.  A row that fits
// the registers of the workgroup stays there (k_top); its k largest are found
// from a bound below them: of G groups of the row, k have a maximum of at least
// the k-th largest group maximum, so the row has at least k logits of at least
// that, and few more when G is several times k.  The group maxima are counted in
// 256 bins of the integer order of their bits (twice, the second time within
// the bin that holds the k-th, when the first leaves many), the logits in and
// above the bin found are collected, and sorted by one 64-bit key: the value's
// order above the complement of the column, so that of equal logits the lowest
// column comes first and no order of the collection shows.
//
// Rows that do not fit are read twice (k_top_long).  Rows on which this collects
// more than it has room for (ties, masks) and rows with NaN or +infinity are
// counted digit by digit from memory (select_row): exact for everything, several
// reads, and equal logits meet in one counter.  4096 x 50257 bfloat16, 64 wanted: 142 us;
// with a NaN in every row 1.3 ms, rows of one value or masked but for 40 columns 3.1 ms.
#include "zo_top_device.h"

namespace zo {

// Writes a row's result.
struct PutLogit {
    float *values;
    int32_t *columns;
    __device__ __forceinline__ PutLogit(const TopArgs &a, int64_t row)
        : values(a.values + row * a.top), columns(a.columns + row * a.top)
    {
    }
    __device__ __forceinline__ void operator()(int rank, uint64_t key) const
    {
        values[rank] = key_value((uint32_t)(key >> 32));
        columns[rank] = (int32_t)~(uint32_t)key;
    }
};

// log(sum) from the pieces: largest logit m, s = sum of 2^(z c - r).
__device__ __forceinline__ float lse_of(float m, float s, float tau, bool nan)
{
    if (nan) return NAN;
    if (m == INFINITY || m == -INFINITY) return m;
    return m / tau + logf(s);
}

// The log-sum-exp of any row, from memory: the differences first, then the
// factor, so that no product overflows and no reference is needed beforehand.
template <int GT, int TH>
__device__ void lse_row(const TopArgs &a, int64_t row, TopShared<TH> &s)
{
    constexpr int K = Elem<GT>::kVec;
    const int64_t V = a.vocab;
    const auto *z = static_cast<const typename Elem<GT>::T *>(a.z) + row * a.ld;
    const float c = log2_factor(a.tau);
    float m = -INFINITY, sum = 0.0f;
    bool nan = false;
    for (int64_t i = (int64_t)threadIdx.x * K; i < V; i += TH * K) {
        const u32x4 w = load16<GT>(z + i, V - i, kNegInf<GT> & kElemMask<GT>);
        const float mv = fmaxf(m, max_of<GT>(w));
        if (m != mv) {
            sum *= m == -INFINITY ? 0.0f : exp2_hw((m - mv) * c);
            m = mv;
        }
#pragma unroll
        for (int q = 0; q < K; ++q) {
            const float v = elem_of<GT>(w, q);
            nan |= v != v;
            if (m != -INFINITY) sum += exp2_hw((v - m) * c);
        }
    }
    __syncthreads();
    group_put<OpMax>(m, s.red[0]);
    group_put<OpMax>(nan ? 1.0f : 0.0f, s.red[1]);
    __syncthreads();
    const float M = group_get<OpMax, TH / 64>(s.red[0]);
    group_put<OpSum>(m == -INFINITY ? 0.0f : sum * exp2_hw((m - M) * c), s.red[2]);
    __syncthreads();
    if (threadIdx.x == 0)
        a.lse[row] = lse_of(M, group_get<OpSum, TH / 64>(s.red[2]), a.tau,
                            group_get<OpMax, TH / 64>(s.red[1]) > 0.0f);
}

// Rows that do not fit registers: the same with a second read of the row, the sums
// from the differences (as lse_row).
template <int GT>
__global__ __launch_bounds__(1024) void k_top_long(TopArgs a)
{
    constexpr int TH = 1024, NW = TH / 64, K = Elem<GT>::kVec;
    __shared__ TopShared<TH> s;
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x, V = a.vocab;
    const auto *z = static_cast<const typename Elem<GT>::T *>(a.z) + row * a.ld;
    const float c = log2_factor(a.tau);
    for (int i = tid; i < 256; i += TH) s.hist[i] = 0;
    if (tid == 0) s.sel[3] = 0;
    GroupMaxima m = {-INFINITY, {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, 0};
    float sum = 0.0f;
    for (int64_t i0 = (int64_t)tid * K; i0 < V; i0 += kGroups * TH * K) {
        u32x4 w[kGroups];
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int64_t i = i0 + g * TH * K;
            w[g] = load16<GT>(z + i, V - i, kNegInf<GT> & kElemMask<GT>);
            if (i < V) m.there |= 1u << g;
        }
        float top = m.all;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const float v = max_of<GT>(w[g]);
            m.of[g] = fmaxf(m.of[g], v);
            top = fmaxf(top, v);
        }
        if (top != m.all) {
            sum *= m.all == -INFINITY ? 0.0f : exp2_hw((m.all - top) * c);
            m.all = top;
        }
        const float b = m.all == -INFINITY ? 0.0f : m.all;
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
            for (int q = 0; q < K; ++q) sum += exp2_hw((elem_of<GT>(w[g], q) - b) * c);
    }
    group_put<OpMax>(m.all, s.red[0]);
    __syncthreads();
    const float M = group_get<OpMax, NW>(s.red[0]);
    if (m.all != -INFINITY) sum *= exp2_hw((m.all - M) * c);
    group_put<OpSum>(sum, s.red[2]);
    const uint32_t least = find_bound<TH>(s, (uint32_t)a.top, M, m);
    const float total = group_get<OpSum, NW>(s.red[2]);
    if (total != total) {                                // NaN or an infinity is about
        if (a.lse) lse_row<GT, TH>(a, row, s);
        select_row<GT, TH>(z, V, a.top, s, PutLogit(a, row));
        return;
    }
    if (a.lse && tid == 0) a.lse[row] = lse_of(M, total, a.tau, false);
    const float bound = key_value(least);
    for (int64_t i = (int64_t)tid * K; i < V; i += TH * K) {
        const u32x4 w = load16<GT>(z + i, V - i, kNegInf<GT> & kElemMask<GT>);
        if (max_of<GT>(w) >= bound) {
#pragma unroll
            for (int q = 0; q < K; ++q) {
                const float v = elem_of<GT>(w, q);
                if (v >= bound && i + q < V) offer<TH>(s, v, i + q);
            }
        }
    }
    __syncthreads();
    const uint32_t n = s.sel[3];
    if (n > kRoom)
        select_row<GT, TH>(z, V, a.top, s, PutLogit(a, row));
    else
        sort_out<TH>(s, (int)n, a.top, PutLogit(a, row));
}

template <int GT, int TH, int NV>
__global__ __launch_bounds__(TH, TH == 768 ? 6 : 4) void k_top(TopArgs a)
{
    constexpr int K = Elem<GT>::kVec, NW = TH / 64;
    __shared__ TopShared<TH> s;
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x, V = a.vocab;
    Resident<GT, TH, NV> x;
    const auto *z = static_cast<const typename Elem<GT>::T *>(a.z) + row * a.ld;
    x.load(z, V);
    for (int i = tid; i < 256; i += TH) s.hist[i] = 0;
    if (tid == 0) s.sel[3] = 0;

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
    group_put<OpMax>(m.all, s.red[0]);
    __syncthreads();
    const float M = group_get<OpMax, NW>(s.red[0]);

    // sum of 2^(c z - r); its NaN also tells of a row with NaN or +infinity (the
    // maxima pass over NaN)
    const float c = log2_factor(a.tau), r = reference(M, c);
    float sum = term(x.last, c, r);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        repack<GT>(x.w[v]);
        if (v * TH < x.vecs) {
#pragma unroll
            for (int q = 0; q < K; ++q) sum += term(elem_of<GT>(x.w[v], q), c, r);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    group_put<OpSum>(sum, s.red[2]);

    // where the groups are not several times as many as are wanted, every logit of a
    // short row is a candidate; fewer groups than wanted logits bound nothing
    const int groups = min(x.vecs, a.top <= TH / kGroups ? TH : TH * kGroups);
    const bool all = 2 * a.top > groups && V <= kRoom, unbound = !all && groups < a.top;
    uint32_t least = 0;
    if (all || unbound)
        __syncthreads();
    else
        least = find_bound<TH>(s, (uint32_t)a.top, M, m);
    const float total = group_get<OpSum, NW>(s.red[2]);
    // from 2^31 on the rounding of r is many exponents
    const bool plain = total == total && fabsf(r) < 0x1p31f;
    bool counted = total != total || unbound;
    if (a.lse && plain && tid == 0) a.lse[row] = lse_of(M, total, a.tau, false);
    if (!counted) {                                      // collect
        const float bound = key_value(least);
        if (x.has_last(V) && (all || x.last >= bound)) offer<TH>(s, x.last, x.last_column());
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            repack<GT>(x.w[v]);
            if (x.at(v) < x.vecs && (all || max_of<GT>(x.w[v]) >= bound)) {
#pragma unroll
                for (int q = 0; q < K; ++q) {
                    const float e = elem_of<GT>(x.w[v], q);
                    if (all || e >= bound) offer<TH>(s, e, x.at(v) * K + q);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        __syncthreads();
        counted = s.sel[3] > kRoom;
    }
    if (counted)
        select_row<GT, TH>(z, V, a.top, s, PutLogit(a, row));
    else
        sort_out<TH>(s, (int)s.sel[3], a.top, PutLogit(a, row));
    if (a.lse && !plain) lse_row<GT, TH>(a, row, s);     // the row's registers are free
}

template <int GT, int TH, int NV>
static hipError_t launch_k_top(const TopArgs &a, hipStream_t st)
{
    return start(k_top<GT, TH, NV>, a.rows, TH, 0, st, a);
}

static hipError_t launch_rows(const TopArgs &a, int gt, hipStream_t st)
{
    return with_elem_type(gt, [&](auto g) {
        constexpr int GT = decltype(g)::value;
        const int64_t vecs = a.vocab / Elem<GT>::kVec;
        if (vecs > 1024 * 16) return start(k_top_long<GT>, a.rows, 1024, 0, st, a);
        // the more are wanted, the more threads: about 4 groups a logit or more.  Long
        // rows: two workgroups of 768 threads a CU, 24 waves (4096 x 50257 bfloat16, 64
        // wanted: 138 us; of 512 with 16 waves 159, of 256 with 12 waves 175, of 1024
        // with 32 waves and too few registers 184)
        if (a.top <= 256 && vecs <= 256 * 4) return launch_k_top<GT, 256, 4>(a, st);
        if (a.top <= 256 && vecs <= 256 * 8) return launch_k_top<GT, 256, 8>(a, st);
        if (a.top <= 512 && vecs <= 512 * 8) return launch_k_top<GT, 512, 8>(a, st);
        if (a.top <= 768 && vecs <= 768 * 9) return launch_k_top<GT, 768, 9>(a, st);
        if (a.top <= 768 && vecs <= 768 * 11) return launch_k_top<GT, 768, 11>(a, st);
        return launch_k_top<GT, 1024, 16>(a, st);
    });
}

hipError_t launch_top_logits(const TopArgs &a, int gt, hipStream_t st)
{
    const int64_t size = gt == GT_F32 ? 4 : 2;
    for (int64_t r = 0; r < a.rows; r += kLaunchRows) {
        const int64_t rows = a.rows - r < kLaunchRows ? a.rows - r : kLaunchRows;
        const TopArgs part = {static_cast<const char *>(a.z) + r * a.ld * size,
                              rows,
                              a.vocab,
                              a.ld,
                              a.top,
                              a.tau,
                              a.values + r * a.top,
                              a.columns + r * a.top,
                              a.lse ? a.lse + r : nullptr};
        const hipError_t e = launch_rows(part, gt, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace zo
