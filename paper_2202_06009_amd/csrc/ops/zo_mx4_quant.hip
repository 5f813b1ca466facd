// zo_mx4_quant.hip -- quantisation to microscaled 4-bit floating point along
// rows, columns or both in one read, and the values read back.
//
// A block of 32 elements with largest magnitude a has the scale byte
// b = max(0, exponent field of a (binary32) - 2); 255 when that field is 255
// (a NaN or an infinity).  Magnitudes are compared as the unsigned integers
// that their bits are without the sign.  The conversion instruction divides by
// 2^(b - 127), taken from the exponent field of its scale operand (so b = 0 is
// 2^-127), rounds to nearest even and saturates at 6.
//
// Both forms move far more bytes than they compute on: the bound is HBM.  A
// workgroup takes 64 (binary32) or 128 rows of 128 columns: 16 lanes read a
// row's 128 elements, 8 each, so that four lanes hold a block, and the four
// 16-row passes of a 64-row group make up the dwords in which the scales are
// stored.  For the column form the tile goes through shared memory once.  8192 x 6400
// bfloat16 both ways 34 us (4.7 TB/s), 6400 x 1600 binary32 14.1 us (3.7), 8192 x 1600
// bfloat16 by rows 11.0 us (3.0), 8191 x 4097 binary16 both ways, off the lines, 26.0 us (4.0).
#include "zo_mx4_device.h"

namespace zo {

template <int GT>
constexpr int kTileRows = GT == GT_F32 ? 64 : 128;

// The row forms of a 64-row group of the tile.  w: the 8 elements of each of
// the four passes, pass p holding row 16 p + rr of the group.
template <int GT, int D>
__device__ __forceinline__ void rows_form(const uint32_t (&w)[4][D], const Mx4View &q, int64_t row0,
                                          int64_t ct, int i, int rr)
{
    uint32_t bytes = 0;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        uint32_t a = 0;
#pragma unroll
        for (int d = 0; d < D; ++d) a = mag<GT>(a, w[p][d]);
        if constexpr (GT != GT_F32) a = max(a & 0xFFFFu, a >> 16);
        a = max(a, dpp<0xB1>(a));   // lanes 1 apart, then 2 apart, of the block's four
        a = max(a, dpp<0x4E>(a));
        const uint32_t b = scale_byte<GT>(a);
        const float s = __uint_as_float(b << 23);
        uint32_t c = 0;
        if constexpr (GT == GT_F32) {
            c = convert2<GT, 0>(c, w[p][0], w[p][1], s);
            c = convert2<GT, 1>(c, w[p][2], w[p][3], s);
            c = convert2<GT, 2>(c, w[p][4], w[p][5], s);
            c = convert2<GT, 3>(c, w[p][6], w[p][7], s);
        } else {
            c = convert2<GT, 0>(c, w[p][0], 0, s);
            c = convert2<GT, 1>(c, w[p][1], 0, s);
            c = convert2<GT, 2>(c, w[p][2], 0, s);
            c = convert2<GT, 3>(c, w[p][3], 0, s);
        }
        if (b == 255) c = 0;
        bytes |= b << (8 * p);
        if (row0 + 16 * p + rr < q.rows) {
            const int64_t tile = (row0 / 16 + p) * q.kt + ct;
            *reinterpret_cast<uint32_t *>(q.codes + tile * 1024 + ((i >> 2) * 16 + rr) * 16 +
                                          (i & 3) * 4) = c;
        }
    }
    if ((i & 3) == 0 && row0 + rr < q.rows)
        *reinterpret_cast<uint32_t *>(
            q.scales + ((row0 / 64 * q.kt + ct) * 64 + (i >> 2) * 16 + rr) * 4) = bytes;
}

template <int GT, bool ROWS, bool COLS>
__global__ __launch_bounds__(256) void k_mx4_quantize(const typename Elem<GT>::T *__restrict__ x,
                                                      int64_t rows, int64_t cols, int64_t ld,
                                                      uint32_t col_tiles, Mx4View q, Mx4View qt)
{
    using T = typename Elem<GT>::T;
    constexpr int D = GT == GT_F32 ? 8 : 4;     // dwords of a lane's 8 elements
    constexpr int TR = kTileRows<GT>;
    constexpr int LW = GT == GT_F32 ? 128 : 64; // dwords of a tile's row
    __shared__ uint32_t tile[COLS ? TR * LW : 1];
    __shared__ uint8_t cscale[COLS ? 4 * 128 : 1];
    const int tid = threadIdx.x, i = tid & 15, rr = tid >> 4;
    const int64_t rt = blockIdx.x / col_tiles, ct = blockIdx.x % col_tiles;
    const int64_t col = ct * 128 + i * 8;

#pragma unroll
    for (int h = 0; h < TR / 64; ++h) {
        const int64_t row0 = rt * TR + h * 64;
        if (!COLS && row0 >= rows) break;
        uint32_t w[4][D];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const int64_t row = row0 + p * 16 + rr;
            const int64_t nv = row < rows ? cols - col : 0;
            const T *at = x + row * ld + col;
            const u32x4 lo = load16<GT>(at, nv);
#pragma unroll
            for (int d = 0; d < 4; ++d) w[p][d] = lo[d];
            if constexpr (GT == GT_F32) {
                const u32x4 hi = load16<GT>(at + 4, nv - 4);
#pragma unroll
                for (int d = 0; d < 4; ++d) w[p][4 + d] = hi[d];
            }
        }
        if constexpr (COLS) {
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                u32x4 *at = reinterpret_cast<u32x4 *>(tile + (h * 64 + p * 16 + rr) * LW + i * D);
                at[0] = u32x4{w[p][0], w[p][1], w[p][2], w[p][3]};
                if constexpr (GT == GT_F32) at[1] = u32x4{w[p][4], w[p][5], w[p][6], w[p][7]};
            }
        }
        if constexpr (ROWS) rows_form<GT, D>(w, q, row0, ct, i, rr);
    }

    if constexpr (COLS) {
        __syncthreads();
        const int64_t kt = rt * TR / 128;       // the transpose's tile along its rows
        const int g0 = TR == 64 ? (int)(rt & 1) * 2 : 0;
        if constexpr (GT == GT_F32) {
            // one column, 32 rows
            const int c = tid & 127, g = tid >> 7;
            uint32_t a = 0, v[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                v[j] = tile[(g * 32 + j) * LW + c];
                a = mag<GT>(a, v[j]);
            }
            const uint32_t b = scale_byte<GT>(a);
            const float s = __uint_as_float(b << 23);
            u32x4 o;
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                uint32_t r = 0;
                r = convert2<GT, 0>(r, v[8 * d], v[8 * d + 1], s);
                r = convert2<GT, 1>(r, v[8 * d + 2], v[8 * d + 3], s);
                r = convert2<GT, 2>(r, v[8 * d + 4], v[8 * d + 5], s);
                r = convert2<GT, 3>(r, v[8 * d + 6], v[8 * d + 7], s);
                o[d] = b == 255 ? 0 : r;
            }
            cscale[g * 128 + c] = (uint8_t)b;
            const int64_t cc = ct * 128 + c;
            if (cc < cols)
                *reinterpret_cast<u32x4 *>(qt.codes + (cc / 16 * qt.kt + kt) * 1024 +
                                           ((g0 + g) * 16 + cc % 16) * 16) = o;
        } else {
            // two adjacent columns, 32 rows
            const int c = (tid & 63) * 2, g = tid >> 6;
            uint32_t a = 0, v[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                v[j] = tile[(g * 32 + j) * LW + (tid & 63)];
                a = mag<GT>(a, v[j]);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t b = scale_byte<GT>(e ? a >> 16 : a & 0xFFFFu);
                const float s = __uint_as_float(b << 23);
                u32x4 o;
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    uint32_t r = 0, m[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        m[j] = __builtin_amdgcn_perm(v[8 * d + 2 * j + 1], v[8 * d + 2 * j],
                                                     e ? 0x07060302u : 0x05040100u);
                    r = convert2<GT, 0>(r, m[0], 0, s);
                    r = convert2<GT, 1>(r, m[1], 0, s);
                    r = convert2<GT, 2>(r, m[2], 0, s);
                    r = convert2<GT, 3>(r, m[3], 0, s);
                    o[d] = b == 255 ? 0 : r;
                }
                cscale[g * 128 + c + e] = (uint8_t)b;
                const int64_t cc = ct * 128 + c + e;
                if (cc < cols)
                    *reinterpret_cast<u32x4 *>(qt.codes + (cc / 16 * qt.kt + kt) * 1024 +
                                               (g * 16 + cc % 16) * 16) = o;
            }
        }
        __syncthreads();
        // dword: the bytes of columns c, c + 16, c + 32, c + 48 of a 64-column group
        constexpr int G = TR / 32;
        if (tid < 2 * G * 16) {
            const int c = tid & 15, g = (tid >> 4) % G, half = tid / (16 * G);
            uint32_t bytes = 0;
#pragma unroll
            for (int p = 0; p < 4; ++p)
                bytes |= (uint32_t)cscale[g * 128 + half * 64 + p * 16 + c] << (8 * p);
            const int64_t c0 = ct * 128 + half * 64;
            if (c0 < cols)
                *reinterpret_cast<uint32_t *>(qt.scales + ((c0 / 64 * qt.kt + kt) * 64 +
                                                           (g0 + g) * 16 + c) * 4) = bytes;
        }
    }
}

// Row tiles of the launch; the column form covers whole tiles of 128 rows (its padding
// columns).
static int64_t quantize_row_tiles(int64_t rows, bool transposed, int tile)
{
    return ((transposed ? (rows + 127) / 128 * 128 : rows) + tile - 1) / tile;
}

bool mx4_quantize_fits(int gt, int64_t rows, int64_t cols, bool transposed)
{
    const int tile = gt == GT_F32 ? kTileRows<GT_F32> : kTileRows<GT_BF16>;
    return fits_a_launch(quantize_row_tiles(rows, transposed, tile) * ((cols + 127) / 128), 256);
}

bool mx4_dequantize_fits(int64_t rows, int64_t cols)
{
    return fits_a_launch((rows + 63) / 64 * ((cols + 127) / 128), 256);
}

hipError_t launch_mx4_quantize(const void *x, int gt, int64_t rows, int64_t cols, int64_t ld,
                               const Mx4View *q, const Mx4View *qt, hipStream_t st)
{
    if (rows == 0 || cols == 0) return hipSuccess;
    return with_elem_type(gt, [&](auto g) {
        constexpr int GT = decltype(g)::value;
        const int64_t ct = (cols + 127) / 128;
        const int64_t tiles = quantize_row_tiles(rows, qt != nullptr, kTileRows<GT>) * ct;
        const auto *p = static_cast<const typename Elem<GT>::T *>(x);
        const Mx4View none{};
        const auto kernel = q && qt ? k_mx4_quantize<GT, true, true>
                            : q     ? k_mx4_quantize<GT, true, false>
                                    : k_mx4_quantize<GT, false, true>;
        return start(kernel, tiles, 256, 0, st, p, rows, cols, ld, (uint32_t)ct, q ? *q : none,
                     qt ? *qt : none);
    });
}

template <int GT, bool NT>
__device__ __forceinline__ void put16(typename Elem<GT>::T *p, const u32x4 &w, int64_t nv)
{
    if (NT && nv >= Elem<GT>::kVec)
        __builtin_nontemporal_store(w, reinterpret_cast<u32x4 *>(p));
    else
        store16<GT>(p, w, nv);
}

// 16 lanes per row of a 128-column tile and 16 bytes of results at a time (8 elements, or
// 4 of each half of the tile), so that a store writes 256 contiguous bytes of a row;
// four rows a thread.  The conversion to binary32 is exact; its upper half is the bfloat16.
//
// NT: nontemporal stores, for rows on lines of 128 bytes, which are then written once:
// 16384 x 8192 bfloat16 61 -> 51 us (6.6 TB/s), 8191 x 4096 binary32 29.9 -> 26.1 us (5.8 TB/s).
// Off the lines a store touches parts of some: 8191 x 4104 binary16 26.3 us, 31.6 us
// nontemporal; 8191 x 4097 30.9 us (2.7 TB/s; outputs in turn, past the caches' size).
// Eight elements of a lane side by side, in binary32 two stores of every other 16 bytes,
// took 72 us for 8191 x 4096 where this took 24.6.
template <int GT, bool NT>
__global__ __launch_bounds__(256) void k_mx4_dequantize(Mx4View q,
                                                        typename Elem<GT>::T *__restrict__ out,
                                                        int64_t ld, uint32_t col_tiles)
{
    constexpr int V = Elem<GT>::kVec, G = 8 / V, PER = 32 / V;   // lanes of a block of 32
    using Codes = std::conditional_t<GT == GT_F32, uint16_t, uint32_t>;
    const int tid = threadIdx.x, i = tid & 15, rr = tid >> 4;
    const int64_t rt = blockIdx.x / col_tiles, ct = blockIdx.x % col_tiles;
    const int64_t col = ct * 128 + i * V;
    uint32_t bytes[G], c[G][4];
#pragma unroll
    for (int g = 0; g < G; ++g) {
        const int at = (g * 2 + i / PER) * 16 + rr;              // block and row
        bytes[g] =
            *reinterpret_cast<const uint32_t *>(q.scales + ((rt * q.kt + ct) * 64 + at) * 4);
#pragma unroll
        for (int p = 0; p < 4; ++p)      // rows beyond the matrix are stored as well
            c[g][p] = *reinterpret_cast<const Codes *>(
                q.codes + ((rt * 4 + p) * q.kt + ct) * 1024 + at * 16 + i % PER * (V / 2));
    }
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int64_t row = rt * 64 + p * 16 + rr;
        if (row >= q.rows) return;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int64_t nv = q.cols - col - g * 64;
            if (nv <= 0) break;
            const uint32_t b = bytes[g] >> (8 * p) & 255u;
            const float s = __uint_as_float(b << 23);
            typedef float f32x2 __attribute__((ext_vector_type(2)));
            u32x4 w;
            if constexpr (GT == GT_F32) {
                const f32x2 v[2] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[g][p], s, 0),
                                    __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[g][p], s, 1)};
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    w[j] = b == 255 ? 0x7FC00000u : __float_as_uint(v[j >> 1][j & 1]);
            } else {
                const f32x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[g][p], s, 0),
                                    __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[g][p], s, 1),
                                    __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[g][p], s, 2),
                                    __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[g][p], s, 3)};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (GT == GT_BF16)
                        w[j] = __builtin_amdgcn_perm(__float_as_uint(v[j][1]),
                                                     __float_as_uint(v[j][0]), 0x07060302u);
                    else
                        w[j] = (uint32_t)narrow<GT>(v[j][0]) | (uint32_t)narrow<GT>(v[j][1]) << 16;
                    if (b == 255) w[j] = GT == GT_BF16 ? 0x7FC07FC0u : 0x7E007E00u;
                }
            }
            put16<GT, NT>(out + row * ld + col + g * 64, w, nv);
        }
    }
}

hipError_t launch_mx4_dequantize(const Mx4View &q, void *out, int gt, int64_t ld, hipStream_t st)
{
    if (q.rows == 0 || q.cols == 0) return hipSuccess;
    const int64_t tiles = (q.rows + 63) / 64 * q.kt;
    return with_elem_type(gt, [&](auto g) {
        constexpr int GT = decltype(g)::value;
        auto *p = static_cast<typename Elem<GT>::T *>(out);
        const bool lines = (uintptr_t)p % 128 == 0 && ld * sizeof(*p) % 128 == 0;
        return start(lines ? k_mx4_dequantize<GT, true> : k_mx4_dequantize<GT, false>, tiles, 256,
                     0, st, q, p, ld, (uint32_t)q.kt);
    });
}

}  // namespace zo
