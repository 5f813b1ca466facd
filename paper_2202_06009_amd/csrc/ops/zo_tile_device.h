// zo_tile_device.h -- what the products of 4-bit and of 8-bit matrices share: the order
// of the workgroups' tiles, and the store of a wave's results (32 x 32 fragments).
#pragma once

#include "zo_ops_device.h"

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
// bytes: 16-byte chunk c of row r is kept at c ^ (r % 8) (% 4 where there are four).  16-bit results: the wave's
// halves swap runs of four, so that a lane holds 8 consecutive columns.  rows, cols: how
// many of them are there; STREAM: past the caches (see streamed).  Straight from the
// registers, 32 bytes of each row: 8192 x 6400 by 128 31 us in 16 bits, 60 in 32; so 27 and 46.
template <int GT, bool STREAM, int NF>
__device__ __forceinline__ void store_rows(typename Elem<GT>::T *out, int64_t ld, int64_t rows,
                                           int64_t cols, const f32x16 (&v)[NF], u32x4 *mine)
{
    constexpr int V = Elem<GT>::kVec, C = 32 * NF / V;     // 16-byte chunks of a row
    constexpr int SWAP = C < 8 ? C - 1 : 7;
    const int lane = threadIdx.x & 63, r = lane & 31, half = lane >> 5;
#pragma unroll
    for (int j = 0; j < NF; ++j) {
        if constexpr (GT == GT_F32) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                mine[r * C + ((j * 8 + q * 2 + half) ^ (r & SWAP))] =
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
                mine[r * C + ((j * 4 + q + half) ^ (r & SWAP))] = w;
            }
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int i = 0; i < C / 2; ++i) {
        const int row = i * (64 / C) + lane / C, c = lane % C;
        const u32x4 w = mine[row * C + (c ^ (row & SWAP))];
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

}  // namespace zo
