// zo_score.hip -- log probabilities of tokens, the rows' entropies and most likely
// alternatives, and the gradient of the logits.
//
// With m the row's largest logit, t = (z - m) log2(e) / tau and e = 2^t:
//   S = sum e, U = sum e t; log p = (z - m) / tau - ln S, entropy = ln S - ln 2 U / S.
// Where one logit has more than half of the probability, S - 1 is summed apart from its 1, and
// ln S is log1p of that: log p of that token keeps its digits, and 1 - p in the gradient.
// A logit of -infinity adds nothing to either sum: where the product of 0 and -infinity has
// made U a NaN, the vector is taken again with t clamped to kLeast.
#include "zo_top_device.h"

namespace zo {

constexpr float kLeast = -256.0f;

// Distances over tau, from k z - k m: with a k of 1/4 for a tau of 1 or more the difference of the
// largest numbers stays within binary32, and the factor of the largest tau within its normal
// numbers.  Below 1 a distance that passes binary32 does so over tau too.
struct Slope {
    float k, c;                  // c = log2(e) / (k tau)

    __device__ __forceinline__ explicit Slope(float tau)
        : k(tau < 1.0f ? 1.0f : 0.25f), c(kLog2e / (k * tau))
    {
    }
    // k (z - m), and t of it.
    __device__ __forceinline__ float apart(float z, float m) const
    {
        return __builtin_fmaf(z, k, -(k * m));
    }
    __device__ __forceinline__ float octaves(float z, float m) const { return apart(z, m) * c; }
};

// A row's results.
struct RowScore {
    float m, log_s, entropy;
};

__device__ __forceinline__ float log_prob(float z, const RowScore &r, float tau)
{
    const Slope by(tau);
    if (r.log_s != r.log_s) return NAN;
    return z == -INFINITY ? -INFINITY : by.apart(z, r.m) / (by.k * tau) - r.log_s;
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

// From the sums, and s - 1 where s is below 2; s of NaN: a NaN or +infinity is among the logits.
__device__ __forceinline__ RowScore row_score(float m, float s, float rest, float u)
{
    if (s != s) return {NAN, NAN, NAN};
    if (m == -INFINITY) return {m, m, 0.0f};
    const float log_s = s < 2.0f ? log1pf(rest) : logf(s);
    return {m, log_s, fmaxf(log_s - kLn2 * (u / s), 0.0f)};
}

// Largest of a vector's elements: 16-bit ones two at a time by their bits, whose order as
// signed integers is that of the numbers where the result is positive, and as unsigned ones the
// opposite among negative numbers.  NaN passes as any
// number: a row with one is not told from these.
typedef int16_t i16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pk_max(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(i16x2, a),
                                                                  __builtin_bit_cast(i16x2, b)));
}

__device__ __forceinline__ uint32_t pk_least(uint32_t a, uint32_t b)
{
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(u16x2, a),
                                                                  __builtin_bit_cast(u16x2, b)));
}

template <int GT>
__device__ __forceinline__ float largest_of(const u32x4 &w)
{
    if constexpr (GT == GT_F32) {
        return max_of<GT>(w);
    } else {
        uint32_t m = pk_max(pk_max(w[0], w[1]), pk_max(w[2], w[3]));
        m = pk_max(m, m >> 16);
        if (m & 0x8000u) {
            m = pk_least(pk_least(w[0], w[1]), pk_least(w[2], w[3]));
            m = pk_least(m, m >> 16);
        }
        return widen<GT>((uint16_t)m);
    }
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

__device__ __forceinline__ void add_term(float z, float b, const Slope &by, float &s, float &u)
{
    const float t = by.octaves(z, b), e = exp2_hw(t);
    s += e;
    u = __builtin_fmaf(e, fmaxf(t, kLeast), u);
}

// The same of the row's largest logit m, less the 1 that it is itself.
__device__ __forceinline__ void add_other(float z, float m, const Slope &by, float &s,
                                          float &u)
{
    add_term(z == m ? -INFINITY : z, m, by, s, u);
}

// A vector's terms about b.
template <int GT>
__device__ __forceinline__ void add_vector(const u32x4 &w, float b, const Slope &by, float &s,
                                           float &u)
{
    const float s0 = s, u0 = u;
#pragma unroll
    for (int q = 0; q < Elem<GT>::kVec; ++q) {
        const float t = by.octaves(elem_of<GT>(w, q), b), e = exp2_hw(t);
        s += e;
        u = __builtin_fmaf(e, t, u);
    }
    if (u != u) {
        s = s0;
        u = u0;
#pragma unroll
        for (int q = 0; q < Elem<GT>::kVec; ++q) add_term(elem_of<GT>(w, q), b, by, s, u);
    }
}

// The sums about a larger logit than they were: u and s d are both below 0, so nothing cancels.
// From -infinity they are 0, or a NaN.
__device__ __forceinline__ void move_base(float from, float to, const Slope &by, float &s,
                                          float &u)
{
    if (from == -INFINITY) return;
    const float d = fmaxf(by.octaves(from, to), kLeast), f = exp2_hw(d);
    u = f * __builtin_fmaf(s, d, u);
    s *= f;
}

// A row by TH threads, in one read.  The sums are those of 1024 lanes, of which a thread is
// one, two or four: lane l takes the vectors l, l + 1024, ... of the row and sums about the
// largest logit of the row's first 1024 vectors, or a larger one of its own; the sums of waves of
// 64 lanes are joined in order.  So a row's results
// are the same bits however many rows there are and whatever else is wanted.  No logit is larger
// than what its lane sums about: a term is at most 1, the row's largest exactly, so S >= 1 and no
// log probability is above 0.  About each lane's own first vector a base would move with most of
// a wave's vectors; beyond the first 1024 hardly any holds a larger one.
//
// Every N-th of a lane's vectors belongs to the same group, four groups a thread.  The groups'
// maxima bound the k-th largest logit from below, and only those that reach the bound, few more
// than are wanted, are read again for the candidates.
//
// Nothing of the row stays in the registers, so that a CU has 2048 threads with several loads
// each under way: 4096 x 50304 bfloat16 without alternatives 81 us, with 20 104; with the row in
// registers, two workgroups of 768 threads a CU, 95 and 126.  Bound by vector instructions and
// memory alike: the floor of one read is 64.
template <int GT, int TH>
__global__ __launch_bounds__(TH, 8) void k_score(zo_score a)
{
    constexpr int LANES = 1024 / TH, NW = TH / 64, K = Elem<GT>::kVec, G = kGroups, N = G / LANES;
    __shared__ TopShared<TH> sh;
    __shared__ float red[2][16];
    const int tid = threadIdx.x;
    const int vecs = (int)(a.vocab / K);
    const int64_t row = blockIdx.x, V = a.vocab, whole = (int64_t)vecs * K;
    const auto *z = static_cast<const typename Elem<GT>::T *>(a.z) + row * a.ldz;
    const Token token = read_token<GT>(a, row, z);
    const Slope by(a.tau);
    GroupMaxima m = {-INFINITY, {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, 0};
    float base[LANES], s[LANES] = {}, u[LANES] = {};
#pragma unroll
    for (int l = 0; l < LANES; ++l) base[l] = -INFINITY;
    for (int j = 0; j < vecs; j += 1024 * N) {
        u32x4 w[N][LANES];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int l = 0; l < LANES; ++l) {
                // without a condition, past the end the last vector: behind a branch each load
                // would wait for the one before
                const int i = min(j + n * 1024 + l * TH + tid, vecs - 1);
                w[n][l] = *reinterpret_cast<const u32x4_a2 *>(z + (int64_t)i * K);
            }
        if (j == 0) {                                    // w[0]: the first 1024 vectors
            float top = largest_of<GT>(w[0][0]);
#pragma unroll
            for (int l = 1; l < LANES; ++l) top = fmaxf(top, largest_of<GT>(w[0][l]));
            group_put<OpMax>(top, sh.red[2]);
            __syncthreads();
            top = group_get<OpMax, NW>(sh.red[2]);
#pragma unroll
            for (int l = 0; l < LANES; ++l) base[l] = top;
        }
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int l = 0; l < LANES; ++l)
                if (j + n * 1024 + l * TH + tid < vecs) {
                    const int g = n * LANES + l;
                    const float top = largest_of<GT>(w[n][l]);
                    m.of[g] = fmaxf(m.of[g], top);
                    m.there |= 1u << g;
                    if (top > base[l]) {
                        move_base(base[l], top, by, s[l], u[l]);
                        base[l] = top;
                    }
                    add_vector<GT>(w[n][l], base[l] == -INFINITY ? 0.0f : base[l], by, s[l], u[l]);
                }
    }
    // one each of the V % K logits that are left
    const bool has_last = whole + tid < V;
    const float last = has_last ? widen<GT>(z[whole + tid]) : -INFINITY;
    if (has_last) {
        if (last > base[0]) {
            move_base(base[0], last, by, s[0], u[0]);
            base[0] = last;
        }
        add_term(last, base[0] == -INFINITY ? 0.0f : base[0], by, s[0], u[0]);
    }
    for (int i = tid; i < 256; i += TH) sh.hist[i] = 0;
    if (tid == 0) sh.sel[3] = 0;
    m.all = last;
#pragma unroll
    for (int g = 0; g < G; ++g) m.all = fmaxf(m.all, m.of[g]);
    group_put<OpMax>(m.all, sh.red[0]);
    __syncthreads();
    const float M = group_get<OpMax, NW>(sh.red[0]);
#pragma unroll
    for (int l = 0; l < LANES; ++l) {
        move_base(base[l], M, by, s[l], u[l]);
        group_put<OpSum>(s[l], red[0] + l * NW);
        group_put<OpSum>(u[l], red[1] + l * NW);
    }
    __syncthreads();
    const float total = group_get<OpSum, 16>(red[0]);
    float rest = 0.0f, mean = group_get<OpSum, 16>(red[1]);
    // S below 2: one logit alone is the largest, as another would add 1, and S has lost the last
    // digits of the others to its 1.  The wave of the lane that has it takes that lane's logits
    // again, one a thread, without it (4096 x 50304 bfloat16 with only such rows 86 us, the lane by
    // itself 93, S as it is 79)
    if (total < 2.0f && M > -INFINITY) {                 // the same for all
        __syncthreads();
#pragma unroll
        for (int l = 0; l < LANES; ++l) {
            float top = l == 0 ? last : -INFINITY;
#pragma unroll
            for (int n = 0; n < N; ++n) top = fmaxf(top, m.of[n * LANES + l]);
            if (const uint64_t mine = __ballot(top == M)) {
                const int at = __ffsll((unsigned long long)mine) - 1, id = tid & 63;
                const int first = l * TH + tid - id + at;        // the lane
                float so = 0.0f, uo = 0.0f;
                for (int k = id; first + k / K * 1024 < vecs; k += 64)
                    add_other(widen<GT>(z[(int64_t)(first + k / K * 1024) * K + k % K]), M, by, so,
                              uo);
                if (l == 0 && id == at) add_other(last, M, by, so, uo);
                so = wave_reduce<OpSum>(so);
                uo = wave_reduce<OpSum>(uo);
                if (id == at) {
                    s[l] = so;
                    u[l] = uo;
                }
            }
            group_put<OpSum>(s[l], red[0] + l * NW);
            group_put<OpSum>(u[l], red[1] + l * NW);
        }
        __syncthreads();
        rest = group_get<OpSum, 16>(red[0]);
        mean = group_get<OpSum, 16>(red[1]);
    }

    // where the groups are not several times as many as are wanted, every logit of a short row
    // is a candidate; fewer groups than wanted logits bound nothing
    const int groups = min(vecs, a.top <= TH / G ? TH : TH * G);
    const bool all = 2 * a.top > groups && V <= kRoom, unbound = !all && groups < a.top;
    uint32_t least = 0;
    if (a.top > 0 && !all && !unbound) least = find_bound<TH>(sh, (uint32_t)a.top, M, m);
    const RowScore r = row_score(M, total, rest, mean);
    if (tid == 0) put_row(a, row, r, token);
    if (a.top == 0) return;
    bool counted = total != total || unbound;
    if (!counted) {                                      // collect
        const float bound = key_value(least);
        if (has_last && (all || last >= bound)) offer<TH>(sh, last, whole + tid);
        auto take = [&](int i) __attribute__((always_inline)) {
            const u32x4 w = *reinterpret_cast<const u32x4_a2 *>(z + (int64_t)i * K);
#pragma unroll
            for (int q = 0; q < K; ++q) {
                const float e = elem_of<GT>(w, q);
                if (all || e >= bound) offer<TH>(sh, e, (int64_t)i * K + q);
            }
        };
#pragma unroll
        for (int g = 0; g < G; ++g)
            if (all || m.of[g] >= bound)
                for (int i = tid + g * TH; i < vecs; i += G * TH) take(i);
        __syncthreads();
        counted = sh.sel[3] > kRoom;
    }
    if (counted)
        select_row<GT, TH>(z, V, a.top, sh, PutScore{a, row, r});
    else
        sort_out<TH>(sh, (int)sh.sel[3], a.top, PutScore{a, row, r});
}

// 1024 vectors at most are one for each lane.  Of long rows, four workgroups of 512 threads a
// CU, or, where a CU has no more than two rows, of 1024: 4096 x 50304 bfloat16, 20 wanted, 104 us
// against 123; 3 x 50257 binary32, 5 wanted, 12.8 against 10.6.  More wanted logits need the
// groups of 1024 threads.
static hipError_t launch_rows(const zo_score &a, int gt, hipStream_t st)
{
    return with_elem_type(gt, [&](auto g) {
        constexpr int GT = decltype(g)::value;
        const int64_t vecs = a.vocab / Elem<GT>::kVec;
        if (a.top <= 256 && vecs <= 1024) return start(k_score<GT, 256>, a.rows, 256, 0, st, a);
        if (a.top <= 256 && a.rows > 512) return start(k_score<GT, 512>, a.rows, 512, 0, st, a);
        return start(k_score<GT, 1024>, a.rows, 1024, 0, st, a);
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
//   dz = p (k0 + k1 t) / (k tau), k0 = -k (dlogp + dentropy entropy), k1 = -k ln 2 dentropy,
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
    const Slope by(a.tau);
    const float l2 = log_s * kLog2e, scale = 1.0f / (by.k * a.tau);
    const float ga = by.k * dlogp, gh = by.k * dh, k0 = -(ga + gh * h), k1 = -kLn2 * gh;
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
            const float d = by.apart(elem_of<GT>(w[v], q), m);
            const float t = fmaxf(__builtin_fmaf(d, by.c, -l2), kLeast);
            e[q] = exp2_hw(t) * __builtin_fmaf(k1, t, k0) * scale;
        }
        if (token >= i && token < i + K) {
#pragma unroll
            for (int q = 0; q < K; ++q)
                if (token == i + q) {
                    const float x = elem_of<GT>(w[v], q);
                    const float lp = log_prob(x, RowScore{m, log_s, h}, a.tau);
                    const float t = fmaxf(lp * kLog2e, kLeast);
                    e[q] = (-ga * expm1f(lp) - gh * exp2_hw(t) * (t * kLn2 + h)) * scale;
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
