// zo_i8_quant.hip -- matrices into 8-bit integers with a scale for each row, along their
// rows, their columns or both, and back.
//
// Bound by memory: by rows a read and half a write of 16-bit elements (8192 x 6400 bfloat16
// 31 us, 5.1 TB/s).  A column's largest magnitude is known only after the whole of it, so the
// columns take a second read: the first pass leaves the maxima of blocks of rows, beside the
// codes of the rows where these are wanted too, a small kernel joins them, and the second pass
// makes the transposed codes (both ways 81 us: 44, 5 and 29).
#include "zo_i8_device.h"

namespace zo {

template <int N>
using Int = std::integral_constant<int, N>;

// Rows of a workgroup where the columns' maxima are wanted too.  One set of partial maxima
// for that many rows goes to memory: 4 bytes for 16 or more elements.
static int64_t rows_a_block(int64_t rows)
{
    const int64_t least = (rows + 511) / 512;
    return least < 16 ? 16 : least;
}

int64_t i8_blocks(int64_t rows)
{
    const int64_t per = rows_a_block(rows);
    return (rows + per - 1) / per;
}

// Rows [blockIdx.x * per, + per), by TEAMS teams of TH threads that hold a row in NV vectors
// a thread, the next row on its way.  q.codes: NULL, or the rows' codes.  COLS: the columns'
// largest magnitudes over these rows into work[blockIdx.x][cols].
template <int GT, int TH, int NV, int TEAMS, bool COLS>
__global__ __launch_bounds__(TH *TEAMS, COLS && NV <= 2 ? 8 : 4) void k_i8_rows(
    const typename Elem<GT>::T *__restrict__ x, int64_t rows, int cols, int64_t ld, I8View q,
    uint32_t *__restrict__ work, int per)
{
    constexpr int K = Elem<GT>::kVec, NW = TH / 64;
    __shared__ uint32_t red[2][TEAMS][NW];
    __shared__ u32x4 joined[COLS && TEAMS > 1 ? (TEAMS - 1) * TH * NV : 1];
    const int t = threadIdx.x % TH, team = threadIdx.x / TH;
    const int64_t from = (int64_t)blockIdx.x * per, to = min(rows, from + per);
    const int turns = (int)(to - from + TEAMS - 1) / TEAMS;
    u32x4 most[COLS ? NV : 1] = {}, w[NV];
    // a team without a row takes the last one again, and stores no codes of it
    auto fetch = [&](int turn) {
        load_row<GT, TH>(w, x + min(from + turn * TEAMS + team, to - 1) * ld, cols, t);
    };
    fetch(0);
    for (int turn = 0; turn < turns; ++turn) {
        const int64_t r = from + turn * TEAMS + team;
        u32x4 m = {};
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                m[i] = packed_max<GT>(m[i], w[v][i]);
                if constexpr (COLS) most[v][i] = packed_max<GT>(most[v][i], w[v][i]);
            }
        if (!q.codes) {                          // the same for all
            if (turn + 1 < turns) fetch(turn + 1);
            continue;
        }
        uint32_t top = wave_max(max_in<GT>(m));
        if constexpr (TH > 64) {
            uint32_t *s = red[turn & 1][team];
            if ((t & 63) == 0) s[t >> 6] = top;
            __syncthreads();
            top = s[0];
#pragma unroll
            for (int i = 1; i < NW; ++i) top = max(top, s[i]);
        }
        const Step s = step_of(top);
        if (t == 0 && r < to) q.scales[r] = s.s;
        int8_t *codes = q.codes + r * q.wide;
        const int wide = r < to ? (int)q.wide : 0;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * TH + t) * K;
            float e[K];
            repack<GT>(w[v]);
#pragma unroll
            for (int i = 0; i < K; ++i) e[i] = elem_of<GT>(w[v], i);
            if (c < wide) store_codes<K>(codes + c, e, s);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (turn + 1 < turns) fetch(turn + 1);
    }
    if constexpr (COLS) {
        if constexpr (TEAMS > 1) {
            if (team > 0)
#pragma unroll
                for (int v = 0; v < NV; ++v) joined[((team - 1) * NV + v) * TH + t] = most[v];
            __syncthreads();
            if (team > 0) return;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
#pragma unroll 1
                for (int k = 0; k < TEAMS - 1; ++k) {
                    const u32x4 o = joined[(k * NV + v) * TH + t];
#pragma unroll
                    for (int i = 0; i < 4; ++i) most[v][i] = packed_max<GT>(most[v][i], o[i]);
                }
            }
        }
        uint32_t *to_work = work + (int64_t)blockIdx.x * cols;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * TH + t) * K;
#pragma unroll
            for (int i = 0; i < K; ++i)
                if (c + i < cols) to_work[c + i] = mag_bits(elem_of<GT>(most[v], i));
        }
    }
}

// Rows that do not fit a workgroup's registers: two reads.
template <int GT>
__global__ __launch_bounds__(1024) void k_i8_rows_long(const typename Elem<GT>::T *__restrict__ x,
                                                       int64_t cols, int64_t ld, I8View q)
{
    constexpr int TH = 1024, K = Elem<GT>::kVec;
    __shared__ uint32_t red[TH / 64];
    const int64_t r = blockIdx.x;
    const typename Elem<GT>::T *p = x + r * ld;
    u32x4 m = {};
    for (int64_t c = (int64_t)threadIdx.x * K; c < cols; c += TH * K) {
        const u32x4 w = load16<GT>(p + c, cols - c);
#pragma unroll
        for (int i = 0; i < 4; ++i) m[i] = packed_max<GT>(m[i], w[i]);
    }
    const Step s = step_of(row_max<TH>(max_in<GT>(m), red));
    if (threadIdx.x == 0) q.scales[r] = s.s;
    for (int64_t c = (int64_t)threadIdx.x * K; c < q.wide; c += TH * K) {
        u32x4 w = {0, 0, 0, 0};
        if (c < cols) w = load16<GT>(p + c, cols - c);
        float e[K];
#pragma unroll
        for (int i = 0; i < K; ++i) e[i] = elem_of<GT>(w, i);
        store_codes<K>(q.codes + r * q.wide + c, e, s);
    }
}

// Columns' largest magnitudes of such rows: workgroup (row block, every runs-th run of 256
// vectors).
template <int GT>
__global__ __launch_bounds__(256) void k_i8_colmax(const typename Elem<GT>::T *__restrict__ x,
                                                   int64_t rows, int64_t cols, int64_t ld,
                                                   uint32_t *__restrict__ work, int64_t per,
                                                   uint32_t runs)
{
    constexpr int K = Elem<GT>::kVec;
    const int64_t block = blockIdx.x / runs, from = block * per, to = min(rows, from + per);
    for (int64_t c = ((int64_t)(blockIdx.x % runs) * 256 + threadIdx.x) * K; c < cols;
         c += (int64_t)runs * 256 * K) {
        u32x4 m = {};
        for (int64_t r = from; r < to; ++r) {
            const u32x4 w = load16<GT>(x + r * ld + c, cols - c);
#pragma unroll
            for (int i = 0; i < 4; ++i) m[i] = packed_max<GT>(m[i], w[i]);
        }
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (c + i < cols) work[block * cols + c + i] = mag_bits(elem_of<GT>(m, i));
    }
}

// The columns' scales from the partial maxima: 32 columns a workgroup, the blocks in 32
// slices.
__global__ __launch_bounds__(1024) void k_i8_colscale(const uint32_t *__restrict__ work,
                                                      int64_t blocks, int64_t stride,
                                                      int64_t cols, float *__restrict__ scales)
{
    __shared__ uint32_t s[32][32];
    const int i = threadIdx.x & 31, slice = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + i;
    uint32_t m = 0;
    if (c < cols)
#pragma unroll 8
        for (int64_t b = slice; b < blocks; b += 32) m = max(m, work[b * stride + c]);
    s[slice][i] = m;
    __syncthreads();
    if (slice == 0 && c < cols) {
#pragma unroll
        for (int k = 1; k < 32; ++k) m = max(m, s[k][i]);
        scales[c] = step_of(m).s;
    }
}

// The transposed codes of a tile of 128 rows x 64 columns: a thread takes four rows of a
// vector of columns at a time, makes a dword of four codes of each column, and the tile
// goes through shared memory so that 128 bytes of a row of qt are stored together.
template <int GT>
__global__ __launch_bounds__(256) void k_i8_cols(const typename Elem<GT>::T *__restrict__ x,
                                                 int64_t rows, int64_t cols, int64_t ld, I8View qt,
                                                 uint32_t strips)
{
    constexpr int K = Elem<GT>::kVec, LANES = 64 / K, GROUPS = 256 / LANES;
    __shared__ uint32_t tile[64][33];
    const int64_t r0 = (int64_t)(blockIdx.x / strips) * 128, c0 = (int64_t)(blockIdx.x % strips) * 64;
    const int j = threadIdx.x % LANES, g = threadIdx.x / LANES;
    const int64_t c = c0 + j * K;
    Step s[K];
#pragma unroll
    for (int q = 0; q < K; ++q) s[q] = step_from(c + q < cols ? qt.scales[c + q] : 0.0f);
#pragma unroll
    for (int n = 0; n < 32 / GROUPS; ++n) {
        const int quad = n * GROUPS + g;
        u32x4 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t r = r0 + quad * 4 + i;
            w[i] = u32x4{0, 0, 0, 0};
            if (r < rows && c < cols) w[i] = load16<GT>(x + r * ld + c, cols - c);
        }
#pragma unroll
        for (int q = 0; q < K; ++q)
            tile[j * K + q][quad] = codes4(elem_of<GT>(w[0], q), elem_of<GT>(w[1], q),
                                           elem_of<GT>(w[2], q), elem_of<GT>(w[3], q), s[q]);
    }
    __syncthreads();
    // whole lines, past the caches (8192 x 6400 bfloat16 both ways 83.6 us, 82.6 so)
    const int i = threadIdx.x & 31;
#pragma unroll
    for (int n = 0; n < 8; ++n) {
        const int k = n * 8 + (threadIdx.x >> 5);
        if (c0 + k < cols)
            __builtin_nontemporal_store(
                tile[k][i], reinterpret_cast<uint32_t *>(qt.codes + (c0 + k) * qt.wide + r0 + i * 4));
    }
}

// Eight codes a thread, 64 threads along a row, four rows a workgroup.
template <int GT>
__global__ __launch_bounds__(256) void k_i8_dequantize(I8View q,
                                                       typename Elem<GT>::T *__restrict__ out,
                                                       int64_t ld, uint32_t runs)
{
    constexpr int K = Elem<GT>::kVec;
    const int64_t r = (int64_t)(blockIdx.x / runs) * 4 + (threadIdx.x >> 6);
    const int64_t c = ((int64_t)(blockIdx.x % runs) * 64 + (threadIdx.x & 63)) * 8;
    if (r >= q.rows || c >= q.cols) return;
    const u32x2 w = *reinterpret_cast<const u32x2 *>(q.codes + r * q.wide + c);
    const float s = q.scales[r];
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = as_binary32<GT>(s * (float)(int8_t)(w[i / 4] >> (8 * (i % 4))));
#pragma unroll
    for (int h = 0; h < 8 / K; ++h) {
        float e[K];
#pragma unroll
        for (int i = 0; i < K; ++i) e[i] = v[h * K + i];
        if (c + h * K < q.cols)
            store16<GT>(out + r * ld + c + h * K, pack16<GT>(e), q.cols - c - h * K);
    }
}

// Columns that a workgroup's registers hold, and with the columns' maxima.
template <int GT, bool COLS>
constexpr int64_t kResident = 1024 * (COLS ? 4 : 8) * Elem<GT>::kVec;

static int64_t runs_of(int64_t cols, int64_t run) { return (cols + run - 1) / run; }

// Only the transposed tiles need one launch of all; the others go into as many as they take.
bool i8_quantize_fits(int64_t rows, int64_t cols, bool transposed)
{
    return !transposed || fits_a_launch(runs_of(rows, 128) * runs_of(cols, 64), 256);
}

template <int GT, bool COLS>
static hipError_t launch_rows(const typename Elem<GT>::T *x, int64_t rows, int64_t cols,
                              int64_t ld, const I8View &q, uint32_t *work, hipStream_t st)
{
    const int64_t vecs = (cols + 127) / 128 * (128 / Elem<GT>::kVec);
    // threads of a row, their vectors, and rows at a time: where the columns are wanted, as
    // many as a workgroup takes
    auto go = [&](auto th, auto nv, auto teams) {
        constexpr int TH = decltype(th)::value, NV = decltype(nv)::value;
        constexpr int TEAMS = COLS ? decltype(teams)::value : TH == 64 ? 4 : 1;
        const auto kernel = k_i8_rows<GT, TH, NV, TEAMS, COLS>;
        if constexpr (COLS) {
            return start(kernel, i8_blocks(rows), TH * TEAMS, 0, st, x, rows, (int)cols, ld, q,
                         work, (int)rows_a_block(rows));
        } else {
            hipError_t e = hipSuccess;
            for (int64_t r = 0; r < rows && e == hipSuccess; r += kLaunchRows) {
                const int64_t part = rows - r < kLaunchRows ? rows - r : kLaunchRows;
                I8View to = q;
                to.codes += r * q.wide;
                to.scales += r;
                e = start(kernel, runs_of(part, TEAMS), TH * TEAMS, 0, st, x + r * ld, part,
                          (int)cols, ld, to, nullptr, TEAMS);
            }
            return e;
        }
    };
    if (vecs <= 64) return go(Int<64>{}, Int<1>{}, Int<16>{});
    if (!COLS && vecs > 512 && vecs <= 1024) return go(Int<256>{}, Int<4>{}, Int<8>{});
    if (vecs <= 256) return go(Int<128>{}, Int<2>{}, Int<8>{});
    if (vecs <= 512) return go(Int<256>{}, Int<2>{}, Int<4>{});
    if (vecs <= 1024) return go(Int<512>{}, Int<2>{}, Int<2>{});
    if (vecs <= 2048) return go(Int<1024>{}, Int<2>{}, Int<1>{});
    if (vecs <= 4096) return go(Int<1024>{}, Int<4>{}, Int<1>{});
    if constexpr (COLS)
        return hipErrorInvalidValue;            // the caller takes the long form
    else
        return go(Int<1024>{}, Int<8>{}, Int<1>{});
}

hipError_t launch_i8_quantize(const void *px, int gt, int64_t rows, int64_t cols, int64_t ld,
                              const I8View *q, const I8View *qt, uint32_t *work, hipStream_t st)
{
    if (rows == 0 || cols == 0) return hipSuccess;
    return with_elem_type(gt, [&](auto g) {
        constexpr int GT = decltype(g)::value, K = Elem<GT>::kVec;
        const auto *x = static_cast<const typename Elem<GT>::T *>(px);
        const I8View none = {};
        hipError_t e = hipSuccess;
        const bool joint = qt && cols <= kResident<GT, true>;
        if (joint) {
            e = launch_rows<GT, true>(x, rows, cols, ld, q ? *q : none, work, st);
        } else {
            if (q && cols <= kResident<GT, false>)
                e = launch_rows<GT, false>(x, rows, cols, ld, *q, nullptr, st);
            else
                for (int64_t r = 0; q && r < rows && e == hipSuccess; r += kLaunchRows) {
                    I8View to = *q;
                    to.codes += r * q->wide;
                    to.scales += r;
                    e = start(k_i8_rows_long<GT>, rows - r < kLaunchRows ? rows - r : kLaunchRows,
                              1024, 0, st, x + r * ld, cols, ld, to);
                }
            if (qt && e == hipSuccess) {
                const int64_t all = runs_of(cols, 256 * K), runs = all < 1024 ? all : 1024;
                e = start(k_i8_colmax<GT>, i8_blocks(rows) * runs, 256, 0, st, x, rows, cols, ld,
                          work, rows_a_block(rows), (uint32_t)runs);
            }
        }
        if (!qt || e != hipSuccess) return e;
        for (int64_t c = 0; c < cols && e == hipSuccess; c += 32 * kLaunchRows)
            e = start(k_i8_colscale, runs_of(cols - c < 32 * kLaunchRows ? cols - c : 32 * kLaunchRows, 32),
                      1024, 0, st, work + c, i8_blocks(rows), cols, cols - c, qt->scales + c);
        if (e != hipSuccess) return e;
        const int64_t strips = runs_of(cols, 64);
        return start(k_i8_cols<GT>, runs_of(rows, 128) * strips, 256, 0, st, x, rows, cols, ld, *qt,
                     (uint32_t)strips);
    });
}

hipError_t launch_i8_dequantize(const I8View &q, void *out, int gt, int64_t ld, hipStream_t st)
{
    if (q.rows == 0 || q.cols == 0) return hipSuccess;
    return with_elem_type(gt, [&](auto g) {
        constexpr int GT = decltype(g)::value;
        const int64_t runs = runs_of(q.cols, 512), most = ((1 << 22) / runs) * 4;
        hipError_t e = hipSuccess;
        for (int64_t r = 0; r < q.rows && e == hipSuccess; r += most) {
            const int64_t part = q.rows - r < most ? q.rows - r : most;
            const I8View from = {q.codes + r * q.wide, q.scales + r, part, q.cols, q.wide};
            e = start(k_i8_dequantize<GT>, runs_of(part, 4) * runs, 256, 0, st, from,
                      static_cast<typename Elem<GT>::T *>(out) + r * ld, ld, (uint32_t)runs);
        }
        return e;
    });
}

}  // namespace zo
