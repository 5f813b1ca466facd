// zo_distill.hip -- the distillation loss from a teacher's top logits and the
// gradient of the student's logits.
//
// One workgroup per row, one pass over memory: the row stays in registers
// (k_distill) between the statistics and the gradient, so that a row costs one
// read and one write.  S (the columns of the used slots) is marked by a bit per
// column in shared memory; its logits are taken out of the row (as -infinity)
// and belong to the threads that hold the slots.  All sums over the rest, of
//   e_i = 2^(c z_i - b), c = log2(e) / tau, b = the rest's own largest c z, rounded,
// are then the rest's own, with no 1 - sum: q_i / q_r = e_i / sum e keeps its
// digits however little the rest holds.  The gradient of the rest is e_i times
// one factor of the row, and at tau = 1 and tau = 2 the label's softmax follows
// from the same e_i (e_i, e_i^2): one exponential per logit in each of the two
// sweeps instead of two.
//
// c z - b is one fused operation, rounded relative to itself; b's own rounding
// is common to every term and cancels.  Where that rounding is itself many
// exponents (the products of the row's largest logits are 2^31 or more) and in rows
// that do not fit registers (k_distill_long, two reads), the difference z - b is
// formed first, b being the largest logit itself (FAR).  4096 x 50257 bfloat16 with the
// teacher's log-sum-exp: 211 us, 319 us where every row's rest is masked by the type's
// lowest value and read again for it.
#include "zo_ops_device.h"

namespace zo {

constexpr int kMaxTop = 1024;

// What 1 - sum p is known to, its terms being rounded exponentials of numbers
// around 10: where the student has nothing outside S, or less than 2^-32768 (masks of
// -1e9 or a type's lowest value: the logarithm would make the rounding the loss), less
// than this is nothing.
constexpr float kRestRounding = 0x1p-16f, kNothing = -32768.0f;

// The base b of a sum whose largest logit is m; 0 for an empty sum.
template <bool FAR>
__device__ __forceinline__ float base_of(float m, float c)
{
    return m == -INFINITY ? 0.0f : FAR ? m : m * c;
}

// log2 of e for logit z.
template <bool FAR>
__device__ __forceinline__ float above(float z, float c, float b)
{
    return FAR ? (z - b) * c : __builtin_fmaf(z, c, -b);
}

// log2 of the factor from base b to base to.
template <bool FAR>
__device__ __forceinline__ float between(float b, float to, float c)
{
    return FAR ? (b - to) * c : b - to;
}

// ln of the same.
template <bool FAR>
__device__ __forceinline__ float log_between(float b, float to, float c, float tau)
{
    return FAR ? (b - to) / tau : between<FAR>(b, to, c) * kLn2;
}

// ln of e about the row's largest logit m, from l, its log2: from the difference itself
// where its product with log2(e) / tau may have passed binary32 (a label or a slot at the
// type's lowest value).
__device__ __forceinline__ float log_above(float z, float m, float tau, float l)
{
    return l < -0x1p100f ? (z - m) / tau : l * kLn2;
}

// How the label's softmax (tau = 1) follows from e: as e (and where no labels are
// given), as e^2, by an exponential of its own.
enum LabelForm { kSame, kSquare, kOwn };

// The teacher's slots of a row: their columns (-1: unused), the two logits, and,
// once the row's statistics are known, the two probabilities.  In shared memory:
// the registers hold the row.  Slot j belongs to thread j modulo TH.
template <int TH>
struct DistillShared {
    int32_t col[kMaxTop];
    float u[kMaxTop], z[kMaxTop], p[kMaxTop], q[kMaxTop];
    float red[12][TH / 64];
    int dup;
};

template <int TH>
struct Row {
    static constexpr int NW = TH / 64;
    int64_t row, V;
    float w, c;              // weight, log2(e) / tau
    int32_t y;               // label, or -1
    float zy;
    bool tail;
    int top;
    // Calls f(j) for the thread's used slots.
    template <class F>
    __device__ __forceinline__ void slots(const DistillShared<TH> &s, F &&f) const
    {
        for (int j = threadIdx.x; j < top; j += TH)
            if (s.col[j] >= 0) f(j);
    }
};

// What a row's gradient follows from, besides its logits.
struct Stats {
    float b_out, b_all, b_one;          // bases: outside S, all, all at tau = 1
    float s_out, s_all, s_one;          // and sums
    float share;                        // q_i = share e_i outside S
    float pr;                           // teacher's mass outside S
    float gk, ge;                       // factors of the two parts
    bool kd, none, no_rest;
};

// log2 of the exponential at tau = 1 for logit z, about the largest of all.
template <bool FAR, LabelForm F>
__device__ __forceinline__ float above_one(float z, float c, const Stats &t)
{
    if constexpr (F == kOwn) return above<FAR>(z, kLog2e, t.b_one);
    return (F == kSquare ? 2.0f : 1.0f) * above<FAR>(z, c, t.b_all);
}

__device__ __forceinline__ bool is_marked(const uint32_t *bits, int64_t i)
{
    return bits[i >> 5] >> (i & 31) & 1;
}

// The marks of the kVec columns from column i (a multiple of kVec) on.
template <int GT>
__device__ __forceinline__ uint32_t marks_of(const uint32_t *bits, int64_t i)
{
    const uint32_t byte = reinterpret_cast<const uint8_t *>(bits)[i >> 3];
    return GT == GT_F32 ? byte >> (i & 4) & 15u : byte;
}

// The row's scalars; its slots, S marked.  Synchronises; false: weight 0.
template <int GT, int TH>
__device__ __forceinline__ bool read_row(const zo_distill &a, Row<TH> &R, DistillShared<TH> &s,
                                         uint32_t *bits, const typename Elem<GT>::T *z)
{
    const int tid = threadIdx.x;
    R.row = blockIdx.x;
    R.V = a.vocab;
    R.top = a.top;
    R.c = log2_factor(a.tau);
    R.tail = a.teacher_lse != nullptr;
    R.w = a.row_weight ? a.row_weight[R.row] : 1.0f;
    if (R.w == 0.0f) return false;
    R.y = a.labels && a.ce_weight != 0.0f ? a.labels[R.row] : -1;
    if (R.y < 0 || R.y >= R.V) R.y = -1;
    R.zy = R.y >= 0 ? widen<GT>(z[R.y]) : 0.0f;
    for (int i = tid; i < (int)((R.V + 31) / 32); i += TH) bits[i] = 0;
    if (tid == 0) s.dup = 0;
    for (int j = tid; j < a.top; j += TH) {
        const int32_t col = a.columns[R.row * a.top + j];
        const bool used = col >= 0 && col < R.V;
        s.col[j] = used ? col : -1;
        s.u[j] = used ? a.values[R.row * a.top + j] : -INFINITY;
        s.z[j] = used ? widen<GT>(z[col]) : -INFINITY;
    }
    __syncthreads();
    R.slots(s, [&](int j) {
        const int32_t col = s.col[j];
        if (atomicOr(&bits[col >> 5], 1u << (col & 31)) >> (col & 31) & 1) s.dup = 1;
    });
    __syncthreads();
    if (s.dup) {                        // of equal columns the first counts
        // judged from the columns as they were, noted in p, then applied
        for (int j = tid; j < a.top; j += TH) {
            bool again = false;
            for (int i = 0; i < j; ++i) again |= s.col[i] == s.col[j];
            s.p[j] = again ? 1.0f : 0.0f;
        }
        __syncthreads();
        for (int j = tid; j < a.top; j += TH)
            if (s.p[j] != 0.0f) {
                s.col[j] = -1;
                s.u[j] = s.z[j] = -INFINITY;
            }
    }
    return true;
}

// Joins the threads' sums outside S (s_out about b_out; at tau = 1: s1 about b1,
// unless it follows from e) with the slots; writes the loss.  m_in: the slots'
// largest logit, um the largest teacher's.  Synchronises.
template <bool FAR, LabelForm F, int TH>
__device__ __forceinline__ Stats statistics(const zo_distill &a, const Row<TH> &R,
                                            DistillShared<TH> &s, float m_out, float m_in,
                                            float um, float s_out, float s1)
{
    constexpr int NW = Row<TH>::NW;
    Stats t;
    const float m_all = fmaxf(m_out, m_in), c = R.c;
    t.b_out = base_of<FAR>(m_out, c);
    t.b_all = base_of<FAR>(m_all, c);
    t.b_one = base_of<FAR>(m_all, kLog2e);
    t.gk = R.w * a.kd_weight * a.tau;
    t.ge = R.w * a.ce_weight;
    t.kd = a.kd_weight != 0.0f && (R.tail || um != -INFINITY);
    const float lse = R.tail ? a.teacher_lse[R.row] : 0.0f, u0 = R.tail ? 0.0f : um;
    // log p up to the sum of p, kept in s.p
    float s_in = 0.0f, one_in = 0.0f, psum = 0.0f;
    R.slots(s, [&](int j) {
        const float u = s.u[j], z = s.z[j];
        const float logp = u == -INFINITY ? -INFINITY : (u - u0) / a.tau - lse;
        s.p[j] = logp;
        psum += expf(logp);
        s_in += exp2_hw(above<FAR>(z, c, t.b_all));
        if constexpr (F == kSquare)
            one_in += exp2_hw(2.0f * above<FAR>(z, c, t.b_all));
        else if constexpr (F == kOwn)
            one_in += exp2_hw(above<FAR>(z, kLog2e, t.b_one));
    });
    group_put<OpSum>(s_out, s.red[4]);
    group_put<OpSum>(s1, s.red[5]);
    group_put<OpSum>(s_in, s.red[6]);
    group_put<OpSum>(one_in, s.red[7]);
    group_put<OpSum>(psum, s.red[8]);
    __syncthreads();
    t.s_out = group_get<OpSum, NW>(s.red[4]);
    s1 = group_get<OpSum, NW>(s.red[5]);
    s_in = group_get<OpSum, NW>(s.red[6]);
    one_in = group_get<OpSum, NW>(s.red[7]);
    psum = group_get<OpSum, NW>(s.red[8]);
    t.no_rest = m_out == -INFINITY && t.s_out == 0.0f;
    t.none = t.no_rest && m_in == -INFINITY && s_in == 0.0f;
    const float log_to_all = m_out == -INFINITY ? 0.0f : between<FAR>(t.b_out, t.b_all, c);
    const float to_all = exp2_hw(log_to_all);
    t.s_all = t.s_out * to_all + s_in;
    t.share = t.none ? 0.0f : to_all / t.s_all;
    if constexpr (F == kSame)
        t.s_one = t.s_all;
    else if constexpr (F == kSquare)
        t.s_one = s1 * exp2_hw(2.0f * log_to_all) + one_in;
    else
        t.s_one = s1 + one_in;
    t.pr = 0.0f;
    if (R.tail) {
        t.pr = fmaxf(0.0f, 1.0f - psum);
        if ((t.no_rest || log_to_all < kNothing) && t.pr < kRestRounding) t.pr = 0.0f;
    }
    const float log_p = R.tail ? 0.0f : logf(psum), log_all = logf(t.s_all);
    // p log(p / q) - p + q for each outcome: what is added sums to 0 over all
    // outcomes, and a term is then small where p is near q
    float kl = 0.0f, qsum = 0.0f;
    R.slots(s, [&](int j) {
        const float z = s.z[j], l = above<FAR>(z, c, t.b_all), logp = s.p[j] - log_p;
        const float p = expf(logp), q = t.none ? 0.0f : exp2_hw(l) / t.s_all;
        s.p[j] = p;
        s.q[j] = q;
        if (p == 0.0f)
            kl += q;
        else if (t.none || z == -INFINITY)
            kl += INFINITY;
        else
            kl += p * (logp - (log_above(z, m_all, a.tau, l) - log_all)) - p + q;
        qsum += q;
    });
    for (float *x : {&t.b_out, &t.b_all, &t.b_one, &t.s_out, &t.s_all, &t.s_one, &t.share, &t.pr,
                     &t.gk, &t.ge})
        *x = uniform(*x);
    if (!a.loss) return t;
    group_put<OpSum>(kl, s.red[9]);
    group_put<OpSum>(qsum, s.red[10]);
    __syncthreads();
    if (threadIdx.x == 0) {
        kl = group_get<OpSum, NW>(s.red[9]);
        qsum = group_get<OpSum, NW>(s.red[10]);
        if (R.tail) {
            // log(pr / qr) from the logarithms where qr is near the end of binary32 or past it
            const float qr = t.s_out * t.share;
            if (t.pr > 0.0f && t.no_rest)
                kl += INFINITY;
            else if (t.pr > 0.0f && qr < 0x1p-100f)
                kl += t.pr * (logf(t.pr) - (log_between<FAR>(t.b_out, t.b_all, c, a.tau) +
                                            logf(t.s_out / t.s_all))) - t.pr + qr;
            else if (t.pr > 0.0f)
                kl += t.pr * logf(t.pr / qr) - t.pr + qr;
            else
                kl += qr;
            kl += fmaxf(0.0f, psum - 1.0f);
        } else if (!t.none) {
            kl += 1.0f - qsum;
        }
        float l = 0.0f;
        if (t.kd)                       // tau^2 may be 0 in binary32
            l = kl == INFINITY ? a.kd_weight * kl : a.kd_weight * a.tau * a.tau * kl;
        if (R.y >= 0) {
            const float lz = log_above(R.zy, m_all, 1.0f, above_one<FAR, F>(R.zy, c, t));
            l += a.ce_weight * (R.zy == -INFINITY ? INFINITY : logf(t.s_one) - lz);
        }
        a.loss[R.row] = R.w * l;
    }
    return t;
}

// The gradient outside S and off the label at logit z, as e times the row's
// factors; f_out: gradient per e, f_one: the label's softmax per its exponential.
template <bool FAR, LabelForm FORM>
__device__ __forceinline__ float rest_value(float z, float c, const Stats &t, float f_out,
                                            float f_one)
{
    const float e = exp2_hw(above<FAR>(z, c, t.b_out));
    if constexpr (FORM == kSame)
        return f_out * e;
    else if constexpr (FORM == kSquare)
        return e * __builtin_fmaf(f_one, e, f_out);
    else
        return __builtin_fmaf(f_out, e, f_one * exp2_hw(above<FAR>(z, kLog2e, t.b_one)));
}

// Of kVec logits.
template <int GT, bool FAR, LabelForm FORM>
__device__ __forceinline__ u32x4 rest_gradient(const u32x4 &w, float c, const Stats &t,
                                               float f_out, float f_one)
{
    float d[Elem<GT>::kVec];
#pragma unroll
    for (int q = 0; q < Elem<GT>::kVec; ++q)
        d[q] = rest_value<FAR, FORM>(elem_of<GT>(w, q), c, t, f_out, f_one);
    return pack16<GT>(d);
}

// Factors of rest_value.
template <bool FAR, LabelForm F>
__device__ __forceinline__ void rest_factors(const Stats &t, bool label, float c, float &f_out,
                                             float &f_one)
{
    f_out = !t.kd || t.no_rest ? 0.0f : t.gk * (t.share - t.pr / t.s_out);
    f_one = 0.0f;
    if (!label || t.no_rest) return;
    if constexpr (F == kSame)
        f_out += t.ge * t.share;
    else if constexpr (F == kSquare)
        f_one = t.ge * exp2_hw(2.0f * between<FAR>(t.b_out, t.b_all, c)) / t.s_one;
    else
        f_one = t.ge / t.s_one;
}

// The gradient at the slots and at the label, over what the sweep left there.
// Synchronises first.
template <int GT, bool FAR, LabelForm F, int TH>
__device__ __forceinline__ void slot_gradient(const Row<TH> &R, const DistillShared<TH> &s,
                                              const Stats &t, float f_out, float f_one,
                                              const uint32_t *bits, typename Elem<GT>::T *dz)
{
    __syncthreads();
    R.slots(s, [&](int j) {
        const int32_t col = s.col[j];
        float d = t.kd ? t.gk * (s.q[j] - s.p[j]) : 0.0f;
        if (R.y >= 0) {
            const float l = above_one<FAR, F>(s.z[j], R.c, t);
            d += t.ge * ((t.none ? 0.0f : exp2_hw(l) / t.s_one) - (col == R.y ? 1.0f : 0.0f));
        }
        dz[col] = narrow<GT>(d);
    });
    if (threadIdx.x == 0 && R.y >= 0 && !is_marked(bits, R.y))
        dz[R.y] = narrow<GT>(rest_value<FAR, F>(R.zy, R.c, t, f_out, f_one) - t.ge);
}

// The thread's slots' largest logits.
template <int TH>
__device__ __forceinline__ void slot_maxima(const Row<TH> &R, const DistillShared<TH> &s,
                                            float &m_in, float &um)
{
    m_in = um = -INFINITY;
    R.slots(s, [&](int j) {
        m_in = fmaxf(m_in, s.z[j]);
        um = fmaxf(um, s.u[j]);
    });
}

template <int GT, int TH>
__device__ __forceinline__ void skip_row(const zo_distill &a, int64_t row,
                                         typename Elem<GT>::T *dz)
{
    constexpr int K = Elem<GT>::kVec;
    if (a.loss && threadIdx.x == 0) a.loss[row] = 0.0f;
    if (a.dz)
        for (int64_t i = (int64_t)threadIdx.x * K; i < a.vocab; i += TH * K)
            store16<GT>(dz + i, u32x4{0, 0, 0, 0}, a.vocab - i);
}

// A row from memory: the differences first (FAR), one sweep with the running
// maximum, one for the gradient.
template <int GT, LabelForm F, int TH>
__device__ void far_row(const zo_distill &a, const Row<TH> &R, DistillShared<TH> &s,
                        const uint32_t *bits, const typename Elem<GT>::T *z,
                        typename Elem<GT>::T *dz)
{
    constexpr int K = Elem<GT>::kVec, NW = TH / 64;
    const float c = R.c;
    float m = -INFINITY, sum = 0.0f, one = 0.0f, m_in, um;
    slot_maxima(R, s, m_in, um);
    // the row's last logits count as a vector filled up with -infinity
    for (int64_t i = (int64_t)threadIdx.x * K; i < R.V; i += TH * K) {
        const u32x4 w = load16<GT>(z + i, R.V - i, kNegInf<GT> & kElemMask<GT>);
        const uint32_t marks = marks_of<GT>(bits, i);
        float x[K], mv = m;
#pragma unroll
        for (int q = 0; q < K; ++q) {
            x[q] = marks >> q & 1 ? -INFINITY : elem_of<GT>(w, q);
            mv = fmaxf(mv, x[q]);
        }
        if (mv != m) {
            if (m != -INFINITY) {
                const float by = exp2_hw((m - mv) * c);
                sum *= by;
                if constexpr (F == kSquare) one *= by * by;
                if constexpr (F == kOwn) one *= exp2_hw((m - mv) * kLog2e);
            }
            m = mv;
        }
        const float b = base_of<true>(m, c);
#pragma unroll
        for (int q = 0; q < K; ++q) {
            const float e = exp2_hw((x[q] - b) * c);
            sum += e;
            if constexpr (F == kSquare) one = __builtin_fmaf(e, e, one);
            if constexpr (F == kOwn) one += exp2_hw((x[q] - b) * kLog2e);
        }
    }
    __syncthreads();
    group_put<OpMax>(m, s.red[0]);
    group_put<OpMax>(m_in, s.red[1]);
    group_put<OpMax>(um, s.red[2]);
    __syncthreads();
    const float m_out = group_get<OpMax, NW>(s.red[0]);
    m_in = group_get<OpMax, NW>(s.red[1]);
    um = group_get<OpMax, NW>(s.red[2]);
    if (m != -INFINITY) {
        sum *= exp2_hw((m - m_out) * c);
        if constexpr (F == kSquare) one *= exp2_hw(2.0f * (m - m_out) * c);
        if constexpr (F == kOwn) one *= exp2_hw((m - fmaxf(m_out, m_in)) * kLog2e);
    }
    const Stats t = statistics<true, F>(a, R, s, m_out, m_in, um, sum, one);
    if (!a.dz) return;
    float f_out, f_one;
    rest_factors<true, F>(t, R.y >= 0, c, f_out, f_one);
    for (int64_t i = (int64_t)threadIdx.x * K; i < R.V; i += TH * K) {
        const u32x4 w = load16<GT>(z + i, R.V - i, kNegInf<GT> & kElemMask<GT>);
        store16<GT>(dz + i, rest_gradient<GT, true, F>(w, c, t, f_out, f_one), R.V - i);
    }
    slot_gradient<GT, true, F>(R, s, t, f_out, f_one, bits, dz);
}

template <int GT, LabelForm F>
__global__ __launch_bounds__(1024) void k_distill_long(zo_distill a)
{
    using T = typename Elem<GT>::T;
    constexpr int TH = 1024;
    extern __shared__ uint32_t bits[];
    __shared__ DistillShared<TH> s;
    const T *z = static_cast<const T *>(a.z) + (int64_t)blockIdx.x * a.ldz;
    T *dz = static_cast<T *>(a.dz) + (int64_t)blockIdx.x * a.lddz;   // if a.dz
    Row<TH> R;
    if (!read_row<GT, TH>(a, R, s, bits, z)) {
        skip_row<GT, TH>(a, blockIdx.x, dz);
        return;
    }
    far_row<GT, F, TH>(a, R, s, bits, z, dz);
}

// One logit's e and its share of the sum at tau = 1.
template <LabelForm F>
__device__ __forceinline__ void add_terms(float z, float c, float b, float b1, float &sum,
                                          float &one)
{
    const float e = exp2_hw(above<false>(z, c, b));
    sum += e;
    if constexpr (F == kSquare) one = __builtin_fmaf(e, e, one);
    if constexpr (F == kOwn) one += exp2_hw(above<false>(z, kLog2e, b1));
}

template <int GT, LabelForm F, int TH, int NV>
__global__ __launch_bounds__(TH, 4) void k_distill(zo_distill a)
{
    using T = typename Elem<GT>::T;
    constexpr int K = Elem<GT>::kVec, NW = TH / 64;
    extern __shared__ uint32_t bits[];
    __shared__ DistillShared<TH> s;
    const T *z = static_cast<const T *>(a.z) + (int64_t)blockIdx.x * a.ldz;
    T *dz = static_cast<T *>(a.dz) + (int64_t)blockIdx.x * a.lddz;   // if a.dz
    Row<TH> R;
    if (a.row_weight && a.row_weight[blockIdx.x] == 0.0f) {
        skip_row<GT, TH>(a, blockIdx.x, dz);
        return;
    }
    Resident<GT, TH, NV> x;
    x.load(z, a.vocab);                       // in flight while the slots are read
    read_row<GT, TH>(a, R, s, bits, z);
    float m_in, um;
    slot_maxima(R, s, m_in, um);
    if (x.has_last(R.V) && is_marked(bits, x.last_column())) x.last = -INFINITY;
    float m_out = x.last;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const uint32_t marks = x.at(v) < x.vecs ? marks_of<GT>(bits, x.at(v) * K) : 0u;
        if (marks) {
#pragma unroll
            for (int q = 0; q < K; ++q)
                if (marks >> q & 1) {
                    if constexpr (GT == GT_F32)
                        x.w[v][q] = kNegInf<GT>;
                    else
                        x.w[v][q >> 1] = q & 1 ? (x.w[v][q >> 1] & 0xFFFFu) | kNegInf<GT> << 16
                                               : (x.w[v][q >> 1] & 0xFFFF0000u) |
                                                     (kNegInf<GT> & 0xFFFFu);
                }
        }
        m_out = fmaxf(m_out, max_of<GT>(x.w[v]));
        __builtin_amdgcn_sched_barrier(0);       // keeps the unpacked logits few
    }
    group_put<OpMax>(m_out, s.red[0]);
    group_put<OpMax>(m_in, s.red[1]);
    group_put<OpMax>(um, s.red[2]);
    __syncthreads();
    m_out = group_get<OpMax, NW>(s.red[0]);
    m_in = group_get<OpMax, NW>(s.red[1]);
    um = group_get<OpMax, NW>(s.red[2]);
    // below 2^31, the products of both largest logits (-infinity: none) with both factors
    // are rounded by at most 64, so that an e of the largest is within 2^-64 to 2^64, and
    // its square at tau = 2, where c is half as large, as well
    const float size = fmaxf(m_out == -INFINITY ? 0.0f : fabsf(m_out),
                             m_in == -INFINITY ? 0.0f : fabsf(m_in));
    if (!(size * fmaxf(R.c, kLog2e) < 0x1p31f)) {
        far_row<GT, F, TH>(a, R, s, bits, z, dz);
        return;
    }
    const float c = uniform(R.c), b = uniform(base_of<false>(m_out, c));
    const float b1 = uniform(base_of<false>(fmaxf(m_out, m_in), kLog2e));
    float sum = 0.0f, one = 0.0f;
    add_terms<F>(x.last, c, b, b1, sum, one);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        repack<GT>(x.w[v]);
        if (v * TH < x.vecs) {                   // the same for all threads
#pragma unroll
            for (int q = 0; q < K; ++q)
                add_terms<F>(elem_of<GT>(x.w[v], q), c, b, b1, sum, one);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    const Stats t = statistics<false, F>(a, R, s, m_out, m_in, um, sum, one);
    if (!a.dz) return;
    float f_out, f_one;
    rest_factors<false, F>(t, R.y >= 0, c, f_out, f_one);
    f_out = uniform(f_out);
    f_one = uniform(f_one);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        repack<GT>(x.w[v]);
        if (x.at(v) < x.vecs)
            *reinterpret_cast<u32x4_a2 *>(dz + (int64_t)x.at(v) * K) =
                rest_gradient<GT, false, F>(x.w[v], c, t, f_out, f_one);
        __builtin_amdgcn_sched_barrier(0);
    }
    if (x.has_last(R.V))
        dz[x.last_column()] = narrow<GT>(rest_value<false, F>(x.last, c, t, f_out, f_one));
    slot_gradient<GT, false, F>(R, s, t, f_out, f_one, bits, dz);
}

template <int GT, LabelForm F>
static hipError_t launch_form(const zo_distill &a, hipStream_t st)
{
    const int64_t vecs = a.vocab / Elem<GT>::kVec;
    const uint32_t lds = (uint32_t)((a.vocab + 31) / 32 * 4);
    if (vecs > 1024 * 16)
        return start(k_distill_long<GT, F>, a.rows, 1024, lds, st, a);
    if (vecs > 512 * 16)
        return start(k_distill<GT, F, 1024, 16>, a.rows, 1024, lds, st, a);
    if (vecs > 512 * 8)
        return start(k_distill<GT, F, 512, 16>, a.rows, 512, lds, st, a);
    if (vecs > 256 * 8)
        return start(k_distill<GT, F, 512, 8>, a.rows, 512, lds, st, a);
    if (vecs > 256 * 4)
        return start(k_distill<GT, F, 256, 8>, a.rows, 256, lds, st, a);
    return start(k_distill<GT, F, 256, 4>, a.rows, 256, lds, st, a);
}

static hipError_t launch_rows(const zo_distill &a, hipStream_t st)
{
    const int gt = a.dtype == ZO_DTYPE_F16 ? GT_F16 : a.dtype == ZO_DTYPE_BF16 ? GT_BF16 : GT_F32;
    const bool labels = a.labels && a.ce_weight != 0.0f;
    return with_elem_type(gt, [&](auto g) {
        constexpr int GT = decltype(g)::value;
        if (!labels || a.tau == 1.0f)
            return launch_form<GT, kSame>(a, st);
        if (a.tau == 2.0f) return launch_form<GT, kSquare>(a, st);
        return launch_form<GT, kOwn>(a, st);
    });
}

hipError_t launch_distill(const zo_distill &a, hipStream_t st)
{
    const int64_t size = a.dtype == ZO_DTYPE_F32 ? 4 : 2;
    for (int64_t r = 0; r < a.rows; r += kLaunchRows) {
        zo_distill part = a;
        part.rows = a.rows - r < kLaunchRows ? a.rows - r : kLaunchRows;
        part.z = static_cast<const char *>(a.z) + r * a.ldz * size;
        part.values += r * a.top;
        part.columns += r * a.top;
        if (a.teacher_lse) part.teacher_lse += r;
        if (a.labels) part.labels += r;
        if (a.row_weight) part.row_weight += r;
        if (a.loss) part.loss += r;
        if (a.dz) part.dz = static_cast<char *>(a.dz) + r * a.lddz * size;
        const hipError_t e = launch_rows(part, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace zo
