// zo_top_device.h -- the largest logits of a row: what zo_top.hip and zo_score.hip share
// (the bound below the k-th largest, the candidates' order, the count digit by digit).
#pragma once

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

__device__ __forceinline__ uint64_t full_key(uint32_t key, uint32_t column)
{
    return (uint64_t)key << 32 | (uint32_t)~column;
}

constexpr int kRoom = 2048;      // candidates

template <int TH>
struct TopShared {
    alignas(16) uint64_t cand[kRoom];
    uint32_t hist[256];
    uint32_t sel[4];
    uint32_t wcount[TH / 64];
    float red[4][TH / 64];
};

// The first `top` of the n keys in s.cand, in descending order, n <= kRoom: put(rank, key).
template <int TH, class PUT>
__device__ void sort_out(TopShared<TH> &s, int n, int top, PUT &&put)
{
    const int tid = threadIdx.x;
    if (n <= (TH < 384 ? TH : 384)) {
        // each key's rank is the number of larger keys (all differ): no barriers; about
        // as quick as the 45 steps below at 384 keys (280 keys: 208 us instead of 240
        // for 256 of 4096 x 50257)
        if (tid == 0 && (n & 1)) s.cand[n] = 0;
        __syncthreads();
        if (tid < n) {
            const uint64_t mine = s.cand[tid];
            const ulong2 *p = reinterpret_cast<const ulong2 *>(s.cand);
            int rank = 0;
            for (int j = 0; j < (n + 1) / 2; ++j) {
                const ulong2 o = p[j];
                rank += (o.x > mine) + (o.y > mine);
            }
            if (rank < top) put(rank, mine);
        }
        return;
    }
    // bitonic, descending, over the next power of two
    int size = 512;
    while (size < n) size *= 2;
    for (int i = n + tid; i < size; i += TH) s.cand[i] = 0;
    for (int k = 2; k <= size; k *= 2)
        for (int j = k / 2; j; j /= 2) {
            __syncthreads();
            for (int t = tid; t < size / 2; t += TH) {
                const int i = 2 * t - (t & (j - 1));      // bit j of i is 0
                const uint64_t x = s.cand[i], y = s.cand[i + j];
                if (((i & k) == 0) == (x < y)) {
                    s.cand[i] = y;
                    s.cand[i + j] = x;
                }
            }
        }
    __syncthreads();
    for (int i = tid; i < top; i += TH) put(i, s.cand[i]);
}

// The digit of the `left`-th largest key in s.hist (256 bins): s.sel[0], what is
// then left within it in s.sel[1], and how many are in and above it in s.sel[2].
// By the first wave, four bins a lane.
template <int TH>
__device__ __forceinline__ void find_bin(TopShared<TH> &s, uint32_t left)
{
    const int lane = threadIdx.x;
    if (lane >= 64) return;
    const u32x4 h = *reinterpret_cast<const u32x4 *>(s.hist + 4 * lane);
    const uint32_t own = h[0] + h[1] + h[2] + h[3];
    uint32_t n = own;                                   // of this lane and those above
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const uint32_t up = __shfl_down(n, o, 64);
        if (lane + o < 64) n += up;
    }
    uint32_t above = n - own;
#pragma unroll
    for (int q = 3; q >= 0; --q) {
        if (above < left && above + h[q] >= left) {
            s.sel[0] = 4 * lane + q;
            s.sel[1] = left - above;
            s.sel[2] = above + h[q];
        }
        above += h[q];
    }
}

// Any row z of V logits, from memory: the k-th largest key digit by digit, the keys above it
// and the lowest columns of those equal to it.
template <int GT, int TH, class PUT>
__device__ void select_row(const typename Elem<GT>::T *z, int64_t V, int top, TopShared<TH> &s,
                           PUT &&put)
{
    constexpr int NW = TH / 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint32_t prefix = 0, left = (uint32_t)top;
    for (int p = 24; p >= 0; p -= 8) {
        __syncthreads();
        for (int i = tid; i < 256; i += TH) s.hist[i] = 0;
        __syncthreads();
        for (int64_t i = tid; i < V; i += TH) {
            const uint32_t k = order_key(widen<GT>(z[i]));
            if (((uint64_t)(k ^ prefix) >> (p + 8)) == 0) atomicAdd(&s.hist[k >> p & 255], 1u);
        }
        __syncthreads();
        find_bin<TH>(s, left);
        __syncthreads();
        prefix |= s.sel[0] << p;
        left = s.sel[1];
    }
    __syncthreads();
    if (tid == 0) s.sel[0] = 0;
    uint32_t equal = 0;                                  // so far
    for (int64_t i0 = 0; i0 < V; i0 += TH) {
        const int64_t i = i0 + tid;
        const uint32_t k = i < V ? order_key(widen<GT>(z[i])) : 0;
        const uint64_t mask = __ballot(i < V && k == prefix);
        if (lane == 0) s.wcount[wave] = __popcll(mask);
        __syncthreads();
        if (i < V && k > prefix) s.cand[atomicAdd(&s.sel[0], 1u)] = full_key(k, (uint32_t)i);
        uint32_t at = equal + __popcll(mask & ((1ull << lane) - 1));
        for (int w = 0; w < NW; ++w) {
            if (w < wave) at += s.wcount[w];
            equal += s.wcount[w];
        }
        if (i < V && k == prefix && at < left)
            s.cand[top - left + at] = full_key(k, (uint32_t)i);
        __syncthreads();
    }
    sort_out<TH>(s, top, top, put);
}

// Groups of the vectors of a thread, when more than a quarter as many logits are
// wanted as there are threads.
constexpr int kGroups = 4;

// A thread's part in the bound: its largest logit, those of its groups, and which
// of the groups have logits (bit g).
struct GroupMaxima {
    float all, of[kGroups];
    uint32_t there;
};

// The key of a lower bound of the `top`-th largest logit from the group maxima, the
// largest of which is M.  s.hist is zero.  Synchronises.
template <int TH>
__device__ __forceinline__ uint32_t find_bound(TopShared<TH> &s, uint32_t top, float M,
                                               const GroupMaxima &m)
{
    constexpr int NW = TH / 64;
    const int tid = threadIdx.x;
    const bool by_thread = top <= TH / kGroups;
    float lo = INFINITY;
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
        if (m.there >> g & 1) lo = fminf(lo, m.of[g]);
    if (by_thread) lo = m.there ? m.all : INFINITY;
    group_put<OpMin>(lo, s.red[1]);
    __syncthreads();
    lo = group_get<OpMin, NW>(s.red[1]);
    // bins of key - key(lo), shifted until 256 cover the range; a NaN falls in none
    const uint32_t klo = order_key(lo);
    const int shift = max(0, 24 - __clz((int)(order_key(M) - klo)));
    const int fine = max(0, shift - 8);
    auto count = [&](uint32_t from, int by, uint32_t bins) {
        auto one = [&](float g, bool there) {
            const uint32_t k = (order_key(g) - from) >> by;
            if (there && k < bins) atomicAdd(&s.hist[k], 1u);
        };
        if (by_thread) {
            one(m.all, m.there != 0);
        } else {
#pragma unroll
            for (int g = 0; g < kGroups; ++g) one(m.of[g], m.there >> g & 1);
        }
    };
    count(klo, shift, 256);
    __syncthreads();
    find_bin<TH>(s, top);
    __syncthreads();
    const uint32_t left = s.sel[1];
    uint32_t least = klo + (s.sel[0] << shift);
    if (shift > 0 && s.sel[2] > top + 64) {
        __syncthreads();
        for (int i = tid; i < 256; i += TH) s.hist[i] = 0;
        __syncthreads();
        count(least, fine, 1u << (shift - fine));
        __syncthreads();
        find_bin<TH>(s, left);
        __syncthreads();
        least += s.sel[0] << fine;
    }
    return least;
}

// A logit that reaches the bound joins the candidates, while there is room.
template <int TH>
__device__ __forceinline__ void offer(TopShared<TH> &s, float v, int64_t i)
{
    const uint32_t at = atomicAdd(&s.sel[3], 1u);
    if (at < kRoom) s.cand[at] = full_key(order_key(v), (uint32_t)i);
}

}  // namespace zo
