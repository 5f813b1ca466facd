// zo_logits.hip -- the teacher's top logits, and the distillation loss with the
// gradient of the student's logits.  One workgroup per row.
#include "zo_ops_device.h"

namespace zo {

// Binary32 in the order of unsigned integers: ascending, -0 as +0, NaN last.
__device__ __forceinline__ uint32_t order_key(float v)
{
    uint32_t b = __float_as_uint(v);
    if (v == 0.0f) b = 0;
    const uint32_t k = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
    return v != v ? 0xFFFFFFFFu : k;
}

__device__ __forceinline__ float key_value(uint32_t k)
{
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// Running maximum m of the logits and sum s of 2^(c (z - m)), c = log2(e) / tau.
// The difference is formed before the factor: it is exact or rounded once
// relative to itself, so a term that counts (z near m) keeps its digits however
// large the logits are, and the lowest finite value does not overflow.
struct Run {
    float m, s;
};

__device__ __forceinline__ void run_add(Run &r, float z, float c)
{
    if (z == -INFINITY) return;      // adds nothing; r.m may still be -infinity
    const float m = fmaxf(r.m, z);
    r.s = r.s * exp2_hw((r.m - m) * c) + exp2_hw((z - m) * c);
    r.m = m;
}

// Both sums about the larger maximum.
__device__ __forceinline__ Run run_join(const Run &a, const Run &b, float c)
{
    const float m = fmaxf(a.m, b.m);
    return {m, (a.m == -INFINITY ? a.s : a.s * exp2_hw((a.m - m) * c)) +
                   (b.m == -INFINITY ? b.s : b.s * exp2_hw((b.m - m) * c))};
}

// Over a workgroup of NW waves: every thread gets the joined (m, s).
template <int NW>
__device__ __forceinline__ Run run_join(Run r, float c, float *sh)
{
    const float m = group_max<NW>(r.m, sh);
    const float part = r.m == -INFINITY ? r.s : r.s * exp2_hw((r.m - m) * c);
    return {m, group_sum<NW>(part, sh)};
}

constexpr int kMaxTop = 1024;

template <int GT>
__global__ __launch_bounds__(1024) void k_top(TopArgs a)
{
    using T = typename Elem<GT>::T;
    __shared__ uint32_t hist[256];
    __shared__ uint64_t cand[kMaxTop];
    __shared__ uint32_t sel[4];      // digit, slots left, candidates, equals so far
    __shared__ uint32_t wcount[16];
    __shared__ float red[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = blockIdx.x;
    const T *z = static_cast<const T *>(a.z) + row * a.ld;
    const int64_t V = a.vocab;

    uint32_t prefix = 0, left = (uint32_t)a.top;
    for (int p = 3; p >= 0; --p) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int64_t i = tid; i < V; i += 1024) {
            const uint32_t k = order_key(widen<GT>(z[i]));
            if (p == 3 || k >> (8 * p + 8) == prefix >> (8 * p + 8))
                atomicAdd(&hist[k >> (8 * p) & 255], 1u);
        }
        __syncthreads();
        if (tid == 0) {
            uint32_t n = 0;
            int d = 255;
            while (n + hist[d] < left) n += hist[d--];
            sel[0] = d;
            sel[1] = left - n;
        }
        __syncthreads();
        prefix |= sel[0] << (8 * p);
        left = sel[1];
        __syncthreads();
    }
    // keys above prefix: all; equal ones: the `left` lowest columns
    if (tid == 0) sel[2] = sel[3] = 0;
    __syncthreads();
    Run r = {-INFINITY, 0.0f};
    bool nan = false;
    for (int64_t i0 = 0; i0 < V; i0 += 1024) {
        const int64_t i = i0 + tid;
        const float v = i < V ? widen<GT>(z[i]) : -INFINITY;
        const uint32_t k = i < V ? order_key(v) : 0;
        if (i < V) {
            nan |= v != v;
            run_add(r, v, kLog2e / a.tau);
        }
        if (i < V && k > prefix)
            cand[atomicAdd(&sel[2], 1u)] = (uint64_t)k << 32 | (uint32_t)~(uint32_t)i;
        const bool eq = i < V && k == prefix;
        const uint64_t mask = __ballot(eq);
        if (lane == 0) wcount[wave] = __popcll(mask);
        const uint32_t before = sel[3];
        __syncthreads();
        uint32_t at = before + __popcll(mask & ((1ull << lane) - 1));
        uint32_t all = 0;
        for (int w = 0; w < 16; ++w) {
            if (w < wave) at += wcount[w];
            all += wcount[w];
        }
        if (eq && at < left)
            cand[a.top - left + at] = (uint64_t)k << 32 | (uint32_t)~(uint32_t)i;
        __syncthreads();
        if (tid == 0) sel[3] = before + all;
        __syncthreads();
    }
    if (tid < a.top) {
        const uint64_t mine = cand[tid];
        int rank = 0;
        for (int j = 0; j < a.top; ++j) rank += cand[j] > mine;
        a.values[row * a.top + rank] = key_value((uint32_t)(mine >> 32));
        a.columns[row * a.top + rank] = (int32_t)~(uint32_t)mine;
    }
    if (a.lse) {
        const Run j = run_join<16>(r, kLog2e / a.tau, red);
        const float any = group_max<16>(nan ? 1.0f : 0.0f, red);
        if (tid == 0)
            a.lse[row] = any > 0 ? NAN
                         : j.m == INFINITY || j.m == -INFINITY ? j.m
                                                               : j.m / a.tau + logf(j.s);
    }
}

hipError_t launch_top_logits(const TopArgs &a, int gt, hipStream_t st)
{
    if (a.rows == 0) return hipSuccess;
    return with_elem_type(gt, [&](auto g) {
        k_top<decltype(g)::value><<<dim3((uint32_t)a.rows), 1024, 0, st>>>(a);
        return hipGetLastError();
    });
}

// What 1 - sum p is known to, its terms being rounded exponentials of numbers
// around 10: where the student has nothing outside S, less than this is nothing.
constexpr float kRestRounding = 0x1p-16f;

template <int GT>
__global__ __launch_bounds__(1024) void k_distill(zo_distill a)
{
    using T = typename Elem<GT>::T;
    extern __shared__ uint32_t bits[];           // a bit per column: in S
    __shared__ float sp[kMaxTop], sz[kMaxTop];   // p and z of the slots
    __shared__ int32_t scol[kMaxTop];            // their columns, -1: unused
    __shared__ float red[16];
    __shared__ int dup;
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x, V = a.vocab;
    const T *z = static_cast<const T *>(a.z) + row * a.ldz;
    T *dz = a.dz ? static_cast<T *>(a.dz) + row * a.lddz : nullptr;
    const float w = a.row_weight ? a.row_weight[row] : 1.0f;
    if (w == 0.0f) {
        if (a.loss && tid == 0) a.loss[row] = 0.0f;
        if (dz)
            for (int64_t i = tid; i < V; i += 1024) dz[i] = 0;
        return;
    }
    const bool tail = a.teacher_lse != nullptr;
    const float ct = kLog2e / a.tau;
    // slots: distinct columns inside the vocabulary
    for (int64_t i = tid; i < (V + 31) / 32; i += 1024) bits[i] = 0;
    if (tid == 0) dup = 0;
    __syncthreads();
    int32_t col = -1;
    float u = -INFINITY;
    if (tid < a.top) {
        col = a.columns[row * a.top + tid];
        if (col < 0 || col >= V) col = -1;
        if (col >= 0 && (atomicOr(&bits[col >> 5], 1u << (col & 31)) >> (col & 31) & 1)) dup = 1;
        scol[tid] = col;
    }
    __syncthreads();
    if (dup && tid < a.top && col >= 0)
        for (int j = 0; j < tid; ++j)
            if (scol[j] == col) {
                col = -1;
                break;
            }
    __syncthreads();
    float zs = -INFINITY;
    if (tid < a.top) {
        scol[tid] = col;
        if (col >= 0) {
            u = a.values[row * a.top + tid];
            zs = widen<GT>(z[col]);
        }
        sz[tid] = zs;
    }
    const int32_t y0 = a.labels && a.ce_weight != 0.0f ? a.labels[row] : -1;
    const bool has = y0 >= 0 && y0 < V;
    const float zy = has ? widen<GT>(z[y0]) : 0.0f;
    const int used = (int)group_sum<16>(col >= 0 ? 1.0f : 0.0f, red);
    // the teacher's p and its logarithm
    float p = 0.0f, logp = -INFINITY;
    if (tail) {
        if (col >= 0) logp = u / a.tau - a.teacher_lse[row];
        p = expf(logp);
    } else {
        const float m = group_max<16>(u, red);
        if (col >= 0 && u != -INFINITY) logp = (u - m) / a.tau;
        p = expf(logp);
        const float s = group_sum<16>(p, red);
        p /= s;
        logp -= logf(s);
    }
    if (tid < a.top) sp[tid] = p;
    const float psum = group_sum<16>(p, red);
    // the student's statistics: outside S (everything, without teacher_lse), in S, at tau 1
    Run out = {-INFINITY, 0.0f}, one = out, in = out;
    for (int64_t i = tid; i < V; i += 1024) {
        const float v = widen<GT>(z[i]);
        run_add(one, v, kLog2e);
        if (!(tail && (bits[i >> 5] >> (i & 31) & 1))) run_add(out, v, ct);
    }
    if (tail && col >= 0) run_add(in, zs, ct);
    out = run_join<16>(out, ct, red);
    one = run_join<16>(one, kLog2e, red);
    Run all = out;
    float pr = 0.0f, qr = 0.0f;
    if (tail) {
        all = run_join(out, run_join<16>(in, ct, red), ct);
        if (out.m != -INFINITY) qr = out.s * exp2_hw((out.m - all.m) * ct) / all.s;
        pr = fmaxf(0.0f, 1.0f - psum);
        if (out.m == -INFINITY && out.s == 0.0f && pr < kRestRounding) pr = 0.0f;
    }
    const bool none = all.m == -INFINITY && all.s == 0.0f;
    const bool kd = a.kd_weight != 0.0f && (tail || used > 0);
    const float gk = w * a.kd_weight * a.tau, ge = w * a.ce_weight;
    const float log_all = logf(all.s);
    if (one.m == -INFINITY && one.s == 0.0f) one = {0.0f, INFINITY};   // softmax 0 everywhere
    const float inv_one = 1.0f / one.s;

    // loss, with p log(p / q) - p + q for each outcome: what is added sums to 0
    // over all outcomes, and a term is then small where p is near q
    float q = 0.0f, term = 0.0f;
    if (col >= 0) {
        q = none ? 0.0f : exp2_hw((zs - all.m) * ct) / all.s;
        if (p > 0.0f)
            term = none || zs == -INFINITY
                       ? INFINITY
                       : p * (logp - ((zs - all.m) / a.tau - log_all)) - p + q;
        else
            term = q;
    }
    const float qin = group_sum<16>(q, red);
    float kl = group_sum<16>(term, red);
    if (tail)
        kl += pr > 0.0f ? (qr > 0.0f ? pr * logf(pr / qr) - pr + qr : INFINITY) : qr;
    else
        kl += none ? 0.0f : 1.0f - qin;
    kl += fmaxf(0.0f, psum - 1.0f);
    if (a.loss && tid == 0) {
        float l = 0.0f;
        if (kd) l = a.kd_weight * a.tau * a.tau * kl;
        if (has) l += a.ce_weight * (zy == -INFINITY ? INFINITY : one.m - zy + logf(one.s));
        a.loss[row] = w * l;
    }
    if (!dz) return;
    // outside S every probability is 2^(c (z - out.m)) times one factor
    const float c = !kd || (out.m == -INFINITY && out.s == 0.0f) ? 0.0f
                    : tail ? gk * (qr - pr) / out.s : gk / out.s;
    __syncthreads();
    for (int64_t i = tid; i < V; i += 1024) {
        const float v = widen<GT>(z[i]);
        if (!(bits[i >> 5] >> (i & 31) & 1)) {
            float d = c == 0.0f ? 0.0f : c * exp2_hw((v - out.m) * ct);
            if (has)
                d += ge * (exp2_hw((v - one.m) * kLog2e) * inv_one - (i == y0 ? 1.0f : 0.0f));
            dz[i] = narrow<GT>(d);
        }
    }
    if (col >= 0) {
        float d = kd ? gk * (q - p) : 0.0f;
        if (has)
            d += ge * (exp2_hw((zs - one.m) * kLog2e) * inv_one - (col == y0 ? 1.0f : 0.0f));
        dz[col] = narrow<GT>(d);
    }
}

hipError_t launch_distill(const zo_distill &a, hipStream_t st)
{
    if (a.rows == 0) return hipSuccess;
    const uint32_t lds = (uint32_t)((a.vocab + 31) / 32 * 4);
    const int gt = a.dtype == ZO_DTYPE_F16 ? GT_F16 : a.dtype == ZO_DTYPE_BF16 ? GT_BF16 : GT_F32;
    return with_elem_type(gt, [&](auto g) {
        k_distill<decltype(g)::value><<<dim3((uint32_t)a.rows), 1024, lds, st>>>(a);
        return hipGetLastError();
    });
}

}  // namespace zo
