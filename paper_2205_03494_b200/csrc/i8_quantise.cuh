// Quantisation to 8-bit integers (i8_format.cuh) along the rows and / or the columns of what a source gives: a matrix in memory, or
// gradients computed from several (omc_gated.cu).
//
// Along the rows alone one kernel reads the values once: a row in the registers of 32 .. 512 threads, sixteen-byte pieces a thread; its largest
// magnitude by shuffles (and a barrier of the row's own threads), then its codes.
// A column's scale follows from the whole column, so its values are needed twice.  A first kernel only takes maxima: a warp walks down a window
// of columns, keeps the largest magnitudes of its columns in registers (a CTA leaves one set in the workspace) and leaves the largest magnitude of
// each row's piece of the window.  A second kernel joins these for a strip of 64 or 128 columns and its rows, and makes the codes along both axes
// from one more read: four rows of a piece a thread; along the rows they go out as they are, along the columns the codes of four rows make a word that
// goes to shared memory, and from there 64 or 128 bytes of a column at a time to memory.  It starts with the rows that the first kernel read last,
// which the L2 cache still holds.
// Whole rows along both axes: the first kernel is the one of the rows alone, which has each row's codes on the way, and leaves the columns' maxima.
// Magnitudes are compared as bit patterns, two 16-bit values in one instruction: their order is that of the values, Inf and NaN on top.
//
// Along the rows memory bounds it: 16384 x 8192 BF16 61.5 us, 6.55 TB/s of values and codes, the rate of a copy.  Along both axes (8192 x 8192 BF16 70.7 us,
// 8192 x 2048 FP32 29.8) the values are read twice and each kernel falls short of the memory's rate, 36 us each: the first issues 60 % of what it could, the second
// waits for loads, its two tiles in shared memory leaving five CTAs of four warps an SM.  (With the rows' codes made in the second: 83 us instead of 71.)  Rows off
// the 16-byte boundaries: 8192 x 8191 BF16 48.6 us along the rows, 130 along both axes (two aligned loads for a piece, shifted together; 109 and 124 registers).
#pragma once
#include <type_traits>

#include "element.cuh"
#include "i8_format.cuh"
#include "mx_encode.cuh"
#include "omc_internal.h"

namespace omc {
namespace i8 {

using el::Word;
using mx::fp32_bits;
using mx::max_magnitude;

template <typename T> constexpr int PIECE = 16 / (int)sizeof(T);               // values of a piece: 8 or 4
template <typename T> constexpr uint32_t MAGNITUDE = sizeof(T) == 4 ? 0x7FFFFFFFu : 0x7FFF7FFFu;
constexpr int ROW_THREADS = 512;                                               // of the widest group that shares a row
constexpr int MAXIMA_WARPS = 8, MAXIMA_CTAS = DEFAULT_SMS * 3;                 // of the first kernel: warps of a CTA, CTAs
constexpr int STRIP_THREADS = 128;                                             // of the second kernel

// Pieces of a warp's window of columns in the first kernel, and CTAs that share a window's rows: their sets of maxima.
template <int OUT> constexpr int WINDOW_PIECES = OUT == 1 ? 4 : 2;
inline uint64_t shares_of(uint64_t rows, uint64_t windows)
{
    // (every CTA of the second kernel reads all sets: of narrow matrices there are as many as SMs and no more)
    uint64_t most = windows < (uint64_t)MAXIMA_CTAS ? MAXIMA_CTAS / windows : 1;
    if (most > DEFAULT_SMS) most = DEFAULT_SMS;
    const uint64_t all = (rows + MAXIMA_WARPS - 1) / MAXIMA_WARPS;
    return all < most ? all : most;
}
// Bytes of the sets of `cols` columns' maxima and of the rows' maxima in the windows, of any type: most sets, widest words, most windows.
inline uint64_t maxima_bytes(uint64_t rows, uint64_t cols, int out)
{
    const uint64_t sets = rows < DEFAULT_SMS ? rows : DEFAULT_SMS, windows = (cols + 255) / 256;
    return sets * out * ((cols + 7) / 8 * 8) * 4 + windows * ((rows + 3) / 4 * 4) * 4;
}

// A piece value by value, `left` of them at most, zeros behind: out of line, since the code of the usual path has to fit the instruction cache.
template <typename T>
__device__ __noinline__ uint4 piece_by_value(const T *at, uint32_t left)
{
    uint32_t w[4];
    mx::load<T, false, PIECE<T>>(at, 0, left, w);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// A piece on its way.  WHOLE, rows on 16-byte boundaries and a multiple of 16 bytes wide: its four words.  Else, of a piece that is `inside`, the two aligned
// sixteens that hold it, which `words` shifts; the others `words` reads value by value.  (Loads are predicated, never one side of a branch: where registers
// meet after a branch the compiler copies them, which waits for the load.  8192 x 8192 BF16, first kernel, 44 us with a branch, 31 us without.)
template <typename T, bool WHOLE>
struct Piece {
    static constexpr int E = PIECE<T>;
    uint4 a, b;
    __device__ __forceinline__ void load(const T *at, bool inside)
    {
        if constexpr (WHOLE) {
            a = *reinterpret_cast<const uint4 *>(at);
        } else if (inside) {
            const uint4 *low = reinterpret_cast<const uint4 *>(reinterpret_cast<uintptr_t>(at) & ~(uintptr_t)15);
            a = low[0];
            b = low[1];
        }
    }
    __device__ __forceinline__ void words(const T *at, uint32_t left, bool inside, uint32_t *out) const
    {
        if constexpr (WHOLE) {
            out[0] = a.x, out[1] = a.y, out[2] = a.z, out[3] = a.w;
        } else {
            const uint32_t skip = (uint32_t)reinterpret_cast<uintptr_t>(at), w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
            uint32_t v[6], u[5];
#pragma unroll
            for (int i = 0; i < 6; ++i) v[i] = skip & 8 ? w[i + 2] : w[i];
#pragma unroll
            for (int i = 0; i < 5; ++i) u[i] = skip & 4 ? v[i + 1] : v[i];
#pragma unroll
            for (int i = 0; i < 4; ++i) out[i] = sizeof(T) == 4 ? u[i] : __funnelshift_r(u[i], u[i + 1], (skip & 2) * 8);
            if (!inside) {
                const uint4 q = piece_by_value<T>(at, left);
                out[0] = q.x, out[1] = q.y, out[2] = q.z, out[3] = q.w;
            } else if (left < (uint32_t)E) {              // zeros behind the row's end
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t n = left > (uint32_t)(i * E / 4) ? left - i * E / 4 : 0u;
                    out[i] &= n >= (uint32_t)(E / 4) ? 0xFFFFFFFFu : n ? 0xFFFFu : 0u;
                }
            }
        }
    }
};
// Whether the two aligned sixteens around a piece lie inside its matrix: in any row but the first and the last, of rows of 32 bytes at least (the first
// begins in the row before it at the earliest, the second ends in the row behind it at the latest).
template <typename T>
__device__ __forceinline__ bool inside(uint32_t row, uint32_t rows, uint32_t cols)
{
    return row - 1u < rows - 2u && rows > 2u && cols >= 2 * PIECE<T>;
}

// Four rows from `row` on, each taken to the nearest one whose pieces may be loaded without a check: the first of them, and whether there is another row
// to go on to behind row i.
template <bool WHOLE>
struct Nearest {
    uint32_t low, high, row;
    __device__ __forceinline__ Nearest(uint32_t r, uint32_t rows) : low(WHOLE ? 0u : 1u), high(WHOLE ? rows - 1 : rows - 2), row(r) {}
    __device__ __forceinline__ uint32_t first() const { return min(max(row, low), high); }
    __device__ __forceinline__ bool on(int i) const { return row + i >= low && row + i < high; }
};

// A matrix in memory.
template <typename T_, bool WHOLE>
struct Matrix {
    using T = T_;
    static constexpr int OUT = 1, HEAVY = WHOLE ? 0 : 1;           // pieces made at a place; whether loads take more registers than those of whole rows
    static constexpr bool WHOLE_ROWS = WHOLE;
    const T *x;
    uint64_t ld;
    uint32_t rows;
    struct Raw {
        Piece<T, WHOLE> x;
    };
    __device__ __forceinline__ void fetch(uint32_t row, uint32_t col, uint32_t cols, Raw &raw) const
    {
        raw.x.load(x + row * ld + col, inside<T>(row, rows, cols));
    }
    // Four rows' pieces, all inside, or (EDGE) from the rows nearest to them; not for matrices whose pieces are all read value by value (see inside).
    template <bool EDGE>
    __device__ __forceinline__ void fetch4(uint32_t row, uint32_t col, Raw *raw) const
    {
        const Nearest<WHOLE> near(row, rows);
        const T *p = x + (EDGE ? near.first() : row) * ld + col;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            raw[i].x.load(p, true);
            if (!EDGE || near.on(i)) p += ld;
        }
    }
    // Of a place that was fetched.
    __device__ __forceinline__ void make(uint32_t row, uint32_t col, uint32_t cols, const Raw &raw, uint32_t (*out)[4]) const
    {
        raw.x.words(x + row * ld + col, cols - col, WHOLE || inside<T>(row, rows, cols), out[0]);
    }
    __device__ __forceinline__ void emit(uint32_t, uint32_t, uint32_t, const uint32_t (*)[4]) const {}
};

// Largest of the two 16-bit magnitudes of a word, or the one 32-bit one, as FP32 bits.
template <typename T>
__device__ __forceinline__ uint32_t top_bits(uint32_t m)
{
    if constexpr (sizeof(T) == 2) m = max(m >> 16, m & 0xFFFFu);
    return fp32_bits<T>(m);
}

// Codes of a piece with one factor.
template <typename T>
__device__ __forceinline__ void encode_piece(const uint32_t *w, float r, bool nan, uint32_t *codes)
{
    constexpr int E = PIECE<T>, N = Word<T>::N;
    float v[E];
#pragma unroll
    for (int i = 0; i < 4; ++i) Word<T>::unpack(w[i], v + N * i);
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = __fmaf_rn(v[i], r, TO_INTEGER);
#pragma unroll
    for (int i = 0; i < E / 4; ++i) codes[i] = nan ? 0u : bytes4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
}

template <int E>
__device__ __forceinline__ void store_whole(int8_t *at, const uint32_t *codes)
{
    if constexpr (E == 8) *reinterpret_cast<uint2 *>(at) = make_uint2(codes[0], codes[1]);
    else *reinterpret_cast<uint32_t *>(at) = codes[0];
}
// A piece's codes into a row of codes from byte `at` on, `n` of them.
template <int E>
__device__ __forceinline__ void store_codes(int8_t *row, uint64_t at, uint32_t n, const uint32_t *codes)
{
    if (n >= (uint32_t)E && at % E == 0) {
        store_whole<E>(row + at, codes);
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if ((uint32_t)i < n) row[at + i] = (int8_t)(codes[i / 4] >> (8 * (i & 3)));
    }
}

// A piece of half o of a row of codes.  One half: zeros behind the last column up to the row's end belong to the pieces there; two: the second
// half starts where the first one ends, and pad_row writes the zeros.
template <int E, int OUT>
__device__ __forceinline__ void store_row_piece(int8_t *row, int o, uint32_t col, uint32_t cols, uint64_t pitch, const uint32_t *codes)
{
    if (OUT == 1 && col < pitch) store_codes<E>(row, col, E, codes);
    if (OUT > 1 && col < cols) store_codes<E>(row, (uint64_t)o * cols + col, cols - col, codes);
}
__device__ __forceinline__ void pad_row(int8_t *row, uint64_t from, uint64_t pitch)
{
    for (uint64_t c = from; c < pitch; ++c) row[c] = 0;
}

struct RowsOut {
    int8_t *codes;            // rows of `pitch` bytes, OUT * cols codes
    float *scales;
    uint64_t pitch;
};

// A CTA's window of columns and share of the rows: blockIdx.x counts the shares of the first window, then those of the next.
struct Place {
    uint32_t shares;
    __device__ __forceinline__ uint32_t window() const { return blockIdx.x / shares; }
    __device__ __forceinline__ uint32_t share() const { return blockIdx.x % shares; }
};

// What the first kernel leaves for the second.
struct Maxima {
    uint4 *cols;              // [set][OUT][pieces of a row] magnitudes
    uint32_t *rows;           // [window][row] magnitudes as FP32 bits
    uint32_t sets, windows;
};

// CTAs on an SM, as the registers allow.
template <typename SRC, int P, int THREADS> constexpr int ROWS_CTAS = THREADS > 256 ? 1 : SRC::HEAVY ? 2 : P > 2 ? 3 : 4;

// The largest magnitudes of a CTA's threads that have the same columns (thread t of every group of them), and a set of them to the workspace.
template <typename T, int P, int OUT, typename F>
__device__ __forceinline__ void leave_maxima(uint32_t (*most)[OUT][4], uint4 *joined, uint32_t groups, uint32_t group, uint32_t set, uint32_t cols, uint4 *out, F column)
{
    constexpr int E = PIECE<T>;
    const uint32_t pieces = (cols + E - 1) / E, tid = threadIdx.x;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int o = 0; o < OUT; ++o) {
            uint32_t *m = most[p][o];
            __syncthreads();
            joined[tid] = make_uint4(m[0], m[1], m[2], m[3]);
            __syncthreads();
            if (tid < group) {
                for (uint32_t i = 1; i < groups; ++i) {
                    const uint4 q = joined[i * group + tid];
                    m[0] = max_magnitude<T>(m[0], q.x), m[1] = max_magnitude<T>(m[1], q.y);
                    m[2] = max_magnitude<T>(m[2], q.z), m[3] = max_magnitude<T>(m[3], q.w);
                }
                if (column(p) < cols) out[((uint64_t)set * OUT + o) * pieces + column(p) / E] = make_uint4(m[0], m[1], m[2], m[3]);
            }
        }
}

// Along the rows.  A row's threads: 2^group_log of them, P pieces each, piece p of thread t at column (p 2^group_log + t) E.  While a row is worked
// on the next AHEAD ones are on their way.  Without ROWS only what the source emits, window by window.  With COLS the columns' maxima too, for codes_kernel.
template <typename SRC, int P, int THREADS, bool ROWS, bool COLS>
__global__ void __launch_bounds__(THREADS, ROWS_CTAS<SRC, P, THREADS>) rows_kernel(SRC src, uint32_t rows, uint32_t cols, uint32_t group_log, Place place, RowsOut out,
                                                                                  Maxima maxima)
{
    using T = typename SRC::T;
    constexpr int E = PIECE<T>, OUT = SRC::OUT, AHEAD = SRC::HEAVY ? 1 : 2;
    __shared__ uint32_t slots[2][THREADS / 32];
    __shared__ uint4 joined[COLS ? THREADS : 1];
    const uint32_t tid = threadIdx.x, group = 1u << group_log, t = tid & (group - 1), g = tid >> group_log, together = THREADS >> group_log;
    const uint32_t window = ROWS ? 0u : place.window() * (group * P * E);
    const uint32_t first_warp = g << (group_log - 5);
    el::enter_stream_order();
    typename SRC::Raw raw[AHEAD][P];
    uint32_t most[COLS ? P : 1][OUT][4];
    if constexpr (COLS) {
#pragma unroll
        for (int i = 0; i < P * OUT * 4; ++i) most[i / (OUT * 4)][i / 4 % OUT][i % 4] = 0u;
    }
    auto column = [&](int p) { return window + (((uint32_t)p << group_log) + t) * E; };
    auto fetch = [&](uint32_t row, typename SRC::Raw *r) {
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (row < rows && column(p) < cols) src.fetch(row, column(p), cols, r[p]);
    };
    const uint32_t step = place.shares * together;
    uint32_t base = place.share() * together, turn = 0;
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) fetch(base + a * step + g, raw[a]);
    while (base < rows) {
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            if (base >= rows) break;
            const uint32_t row = base + g;
            uint32_t w[P][OUT][4];
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if (row < rows && column(p) < cols) {
                    src.make(row, column(p), cols, raw[a][p], w[p]);
                    src.emit(row, column(p), cols, w[p]);
                } else {
#pragma unroll
                    for (int i = 0; i < OUT * 4; ++i) w[p][i / 4][i % 4] = 0u;
                }
            }
            fetch(row + AHEAD * step, raw[a]);
            if constexpr (ROWS) {
                uint32_t top = 0u;
#pragma unroll
                for (int i = 0; i < P * OUT * 4; ++i) {
                    const uint32_t m = w[i / (OUT * 4)][i / 4 % OUT][i % 4] & MAGNITUDE<T>;
                    top = max_magnitude<T>(top, m);
                    if constexpr (COLS) most[i / (OUT * 4)][i / 4 % OUT][i % 4] = max_magnitude<T>(most[i / (OUT * 4)][i / 4 % OUT][i % 4], m);
                }
                top = __reduce_max_sync(0xFFFFFFFFu, top_bits<T>(top));
                if (group_log > 5) {                  // a barrier of the row's own threads
                    if ((tid & 31) == 0) slots[turn][tid >> 5] = top;
                    asm volatile("bar.sync %0, %1;" ::"r"(g + 1), "r"(group) : "memory");
                    for (uint32_t i = 0; i < group >> 5; ++i) top = max(top, slots[turn][first_warp + i]);
                    turn ^= 1u;
                }
                if (row < rows) {
                    const Scale s = scale_of(top);
                    int8_t *to = out.codes + row * out.pitch;
#pragma unroll
                    for (int p = 0; p < P; ++p)
#pragma unroll
                        for (int o = 0; o < OUT; ++o) {
                            uint32_t c[E / 4];
                            encode_piece<T>(w[p][o], s.r, s.nan(), c);
                            store_row_piece<E, OUT>(to, o, column(p), cols, out.pitch, c);
                        }
                    if (OUT > 1 && t == 0) pad_row(to, (uint64_t)OUT * cols, out.pitch);
                    if (t == 0) out.scales[row] = s.s;
                }
            }
            base += step;
        }
    }
    if constexpr (COLS) leave_maxima<T, P, OUT>(most, joined, together, group, place.share(), cols, maxima.cols, column);
}

// Rows too wide for the registers, along the rows only: read for the magnitude and again for the codes.
constexpr int WIDE_THREADS = 512;
template <typename SRC>
__global__ void __launch_bounds__(WIDE_THREADS) wide_rows_kernel(SRC src, uint32_t rows, uint32_t cols, RowsOut out)
{
    using T = typename SRC::T;
    constexpr int E = PIECE<T>, OUT = SRC::OUT;
    __shared__ uint32_t slots[WIDE_THREADS / 32];
    el::enter_stream_order();
    for (uint32_t row = blockIdx.x; row < rows; row += gridDim.x) {
        typename SRC::Raw raw;
        uint32_t w[OUT][4], top = 0u;
        for (uint32_t col = threadIdx.x * E; col < cols; col += WIDE_THREADS * E) {
            src.fetch(row, col, cols, raw);
            src.make(row, col, cols, raw, w);
            src.emit(row, col, cols, w);
#pragma unroll
            for (int i = 0; i < OUT * 4; ++i) top = max_magnitude<T>(top, w[i / 4][i % 4] & MAGNITUDE<T>);
        }
        top = __reduce_max_sync(0xFFFFFFFFu, top_bits<T>(top));
        if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = top;
        __syncthreads();
        for (int i = 0; i < WIDE_THREADS / 32; ++i) top = max(top, slots[i]);
        const Scale s = scale_of(top);
        int8_t *to = out.codes + row * out.pitch;
        for (uint32_t col = threadIdx.x * E; col < cols; col += WIDE_THREADS * E) {
            src.fetch(row, col, cols, raw);
            src.make(row, col, cols, raw, w);
#pragma unroll
            for (int o = 0; o < OUT; ++o) {
                uint32_t c[E / 4];
                encode_piece<T>(w[o], s.r, s.nan(), c);
                store_codes<E>(to, (uint64_t)o * cols + col, cols - col, c);
            }
        }
        if (threadIdx.x == 0) {
            pad_row(to, (uint64_t)OUT * cols, out.pitch);
            out.scales[row] = s.s;
        }
        __syncthreads();
    }
}

// First kernel.
template <typename SRC, bool ROWS>
__global__ void __launch_bounds__(32 * MAXIMA_WARPS, SRC::HEAVY ? 2 : 3) maxima_kernel(SRC src, uint32_t rows, uint32_t cols, Place place, Maxima out)
{
    using T = typename SRC::T;
    constexpr int E = PIECE<T>, OUT = SRC::OUT, P = WINDOW_PIECES<OUT>, AHEAD = SRC::WHOLE_ROWS ? 2 : 1;
    __shared__ uint4 joined[32 * MAXIMA_WARPS];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, window = place.window() * (32 * P * E);
    el::enter_stream_order();
    typename SRC::Raw raw[AHEAD][P];
    uint32_t most[P][OUT][4];
    auto column = [&](int p) { return window + (p * 32 + lane) * E; };
    auto fetch = [&](uint32_t row, typename SRC::Raw *r) {
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (row < rows && column(p) < cols) src.fetch(row, column(p), cols, r[p]);
    };
#pragma unroll
    for (int i = 0; i < P * OUT * 4; ++i) most[i / (OUT * 4)][i / 4 % OUT][i % 4] = 0u;
    const uint32_t step = place.shares * MAXIMA_WARPS;
    uint32_t row = place.share() * MAXIMA_WARPS + warp;
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) fetch(row + a * step, raw[a]);
    while (row < rows) {
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            if (row >= rows) break;
            uint32_t top = 0u;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if (column(p) < cols) {
                    uint32_t w[OUT][4];
                    src.make(row, column(p), cols, raw[a][p], w);
                    src.emit(row, column(p), cols, w);
#pragma unroll
                    for (int i = 0; i < OUT * 4; ++i) {
                        const uint32_t m = w[i / 4][i % 4] & MAGNITUDE<T>;
                        if constexpr (ROWS) top = max_magnitude<T>(top, m);
                        most[p][i / 4][i % 4] = max_magnitude<T>(most[p][i / 4][i % 4], m);
                    }
                }
            }
            fetch(row + AHEAD * step, raw[a]);
            if constexpr (ROWS) {
                top = __reduce_max_sync(0xFFFFFFFFu, top_bits<T>(top));
                if (lane == 0) out.rows[(uint64_t)place.window() * rows + row] = top;
            }
            row += step;
        }
    }
    // (leave_maxima written out: called here, the compiler's loop above took 126 instead of 77 us for the gated layer's gradients at 8192 x 8192 BF16, before the tails of the gates were made exact)
    const uint32_t pieces = (cols + E - 1) / E;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int o = 0; o < OUT; ++o) {
            uint32_t *m = most[p][o];
            __syncthreads();
            joined[threadIdx.x] = make_uint4(m[0], m[1], m[2], m[3]);
            __syncthreads();
            if (warp == 0) {
                for (uint32_t i = 1; i < MAXIMA_WARPS; ++i) {
                    const uint4 q = joined[i * 32 + lane];
                    m[0] = max_magnitude<T>(m[0], q.x), m[1] = max_magnitude<T>(m[1], q.y);
                    m[2] = max_magnitude<T>(m[2], q.z), m[3] = max_magnitude<T>(m[3], q.w);
                }
                if (column(p) < cols) out.cols[((uint64_t)place.share() * OUT + o) * pieces + column(p) / E] = make_uint4(m[0], m[1], m[2], m[3]);
            }
        }
}

struct ColsOut {
    int8_t *codes;            // OUT * cols rows of `pitch` bytes, `rows` codes
    float *scales;
    uint64_t pitch;
};

// A truth value that the compiler knows, and one that it does not.
template <bool V>
struct Known {
    static constexpr bool value = V;
};
struct Asked {
    bool value;
};

// Second kernel: blockIdx.x is a strip of sixteen pieces of columns and a share of the row tiles, the last ones first.  A thread takes four rows of a
// piece at a time, a CTA a sweep of 32 rows; the loads of the next sweeps are on their way.
template <typename SRC>
struct Strip {
    static constexpr int E = PIECE<typename SRC::T>, COLS = 16 * E, SWEEPS = SRC::OUT == 1 ? 4 : 2;     // 128 or 64 columns; sweeps of a tile
    static constexpr int AHEAD = SRC::OUT == 1 && !SRC::HEAVY ? 2 : 1;
    static constexpr int ROWS = 32 * SWEEPS, WORDS = ROWS / 4;                                         // of a tile; of a column of its codes
    static constexpr int CTAS = SRC::OUT == 1 ? (SRC::HEAVY ? 4 : 5) : 3;        // on an SM, as the registers allow
    static constexpr int WORDS_ALL = SRC::OUT * COLS * WORDS;
    // Column e of piece p is column e 16 + p of the tile in shared memory.  Its words are turned by the piece (an even number), so that a warp's
    // stores, sixteen pieces of two words each, fall into different banks.
    static __device__ __forceinline__ uint32_t turned(uint32_t piece) { return WORDS == 32 ? piece * 2 : (piece >> 1) * 2; }
};
template <typename SRC, bool ROWS>
__global__ void __launch_bounds__(STRIP_THREADS, Strip<SRC>::CTAS) codes_kernel(SRC src, uint32_t rows, uint32_t cols, uint32_t strips, uint32_t tiles_each, Maxima in,
                                                                               RowsOut out_r, ColsOut out)
{
    using T = typename SRC::T;
    using S = Strip<SRC>;
    constexpr int E = S::E, OUT = SRC::OUT, COLS = S::COLS, WORDS = S::WORDS, SWEEPS = S::SWEEPS, AHEAD = S::AHEAD, DOWN = STRIP_THREADS / 16;
    static_assert(DOWN * 4 == 32 && S::ROWS <= STRIP_THREADS, "");
    __shared__ __align__(16) uint32_t tiles_smem[2 * S::WORDS_ALL];            // two tiles, in turn: one barrier a tile
    __shared__ __align__(16) float factor[OUT * COLS], row_factor[2][ROWS ? S::ROWS : 4];
    __shared__ uint32_t any_nan, nan_rows[2];
    const uint32_t tid = threadIdx.x, piece = tid % 16, down = tid / 16;
    const uint32_t strip = blockIdx.x % strips, share = blockIdx.x / strips, tiles = (rows + S::ROWS - 1) / S::ROWS;
    const uint32_t end = tiles - share * tiles_each, begin = end > tiles_each ? end - tiles_each : 0u;
    const uint32_t col = strip * COLS + piece * E;
    if (tid == 0) any_nan = nan_rows[0] = nan_rows[1] = 0u;
    __syncthreads();
    el::enter_stream_order();
    typename SRC::Raw raw[AHEAD][4];
    auto row_of = [&](uint32_t t, int k) { return t * S::ROWS + k * 32 + down * 4; };      // the first of four, in sweep k of tile t
    const bool here = col < cols;
    const bool loads = here && (SRC::WHOLE_ROWS || (rows > 2 && cols >= 2 * E));      // (else every piece is read value by value)
    // whether all of a tile's rows are there and inside
    auto full = [&](uint32_t t) { return SRC::WHOLE_ROWS ? (t + 1) * S::ROWS <= rows : t > 0 && (t + 1) * S::ROWS < rows; };
    auto fetch = [&](uint32_t t, int k, typename SRC::Raw *r) {
        if (!loads) return;
        if (full(t)) src.template fetch4<false>(row_of(t, k), col, r);
        else src.template fetch4<true>(row_of(t, k), col, r);
    };
    auto rows_of = [&](uint32_t t) {                               // a tile's rows' factors, a row a thread; the first strip stores the scales
        if constexpr (ROWS) {
            const uint32_t row = t * S::ROWS + tid;
            if (tid < S::ROWS && row < rows) {
                uint32_t top = 0u;
                for (uint32_t i = 0; i < in.windows; ++i) top = max(top, in.rows[(uint64_t)i * rows + row]);
                const Scale s = scale_of(top);
                row_factor[t & 1u][tid] = s.r;
                if (s.nan()) nan_rows[t & 1u] = t + 1;             // (no other tile's number)
                if (strip == 0) out_r.scales[row] = s.s;
            }
        }
    };
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) fetch(end - 1, k, raw[k]);
    rows_of(end - 1);
    // the strip's magnitudes: eight threads share the sets of a piece, and join what they found in shared memory
    const uint32_t pieces = (cols + E - 1) / E;
    uint4 *const found = reinterpret_cast<uint4 *>(tiles_smem);    // [OUT][8][16]
    static_assert(OUT * STRIP_THREADS * 4 <= 2 * S::WORDS_ALL, "");
    auto join = [](uint4 &m, const uint4 &q) {
        m.x = max_magnitude<T>(m.x, q.x), m.y = max_magnitude<T>(m.y, q.y);
        m.z = max_magnitude<T>(m.z, q.z), m.w = max_magnitude<T>(m.w, q.w);
    };
    uint4 m[OUT];
#pragma unroll
    for (int o = 0; o < OUT; ++o) m[o] = make_uint4(0u, 0u, 0u, 0u);
    if (here) {
        constexpr int BATCH = 8;                                   // sets on their way
        const uint4 *from = in.cols + (uint64_t)down * OUT * pieces + col / E;
        for (uint32_t i = down; i < in.sets; i += DOWN * BATCH) {
            uint4 q[BATCH][OUT];
#pragma unroll
            for (int j = 0; j < BATCH; ++j, from += (uint64_t)DOWN * OUT * pieces)
#pragma unroll
                for (int o = 0; o < OUT; ++o) q[j][o] = i + j * DOWN < in.sets ? from[(uint64_t)o * pieces] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int j = 0; j < BATCH * OUT; ++j) join(m[j % OUT], q[j / OUT][j % OUT]);
        }
    }
#pragma unroll
    for (int o = 0; o < OUT; ++o) found[o * STRIP_THREADS + tid] = m[o];
    __syncthreads();
    if (down < OUT) {                                              // sixteen threads finish a half
        const uint32_t o = down;
        uint4 all = found[o * STRIP_THREADS + piece];
        for (int i = 1; i < DOWN; ++i) join(all, found[o * STRIP_THREADS + i * 16 + piece]);
        const uint32_t w[4] = {all.x, all.y, all.z, all.w};
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint32_t bits = fp32_bits<T>(sizeof(T) == 4 ? w[e % 4] : w[e / 2] >> (16 * (e & 1)) & 0xFFFFu);
            const Scale s = scale_of(bits);
            factor[o * COLS + piece * E + e] = s.r;
            if (s.nan()) any_nan = 1u;
            if (begin == 0 && col + e < cols) out.scales[(uint64_t)o * cols + col + e] = s.s;
        }
    }
    __syncthreads();
    const bool masked = any_nan != 0u;
    // what a thread brings from the tile to memory: chunk `chunk` of columns STEP places apart, which are STEP / 16 columns of its piece p apart
    constexpr int CHUNKS = WORDS / 4, STEP = STRIP_THREADS / CHUNKS;
    const uint32_t chunk = tid % CHUNKS, slot = tid / CHUNKS, p_out = slot % 16, turned = S::turned(p_out), first_col = strip * COLS + p_out * E + slot / 16;
    int8_t *const to_cols = out.codes + (uint64_t)first_col * out.pitch + chunk * 16;

    for (uint32_t t = end; t-- > begin;) {
        uint32_t *const tile = tiles_smem + (t & 1u) * S::WORDS_ALL;
        const bool masked_rows = ROWS && nan_rows[t & 1u] == t + 1, all_there = (strip + 1) * COLS <= cols && (t + 1) * S::ROWS <= rows;
        auto work = [&](auto all) {
            const bool all_there = all.value;
#pragma unroll 1
            for (int k0 = 0; k0 < SWEEPS; k0 += AHEAD)
#pragma unroll
            for (int kk = 0; kk < AHEAD; ++kk) {
                constexpr int N = Word<T>::N;
                const int k = k0 + kk;
                const uint32_t row0 = row_of(t, k);
                uint32_t w[4][OUT][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool there = here && row0 + i < rows;
                    if (SRC::WHOLE_ROWS || there) src.make(row0 + i, col, cols, raw[kk][i], w[i]);
                    if (!all_there)
#pragma unroll
                        for (int j = 0; j < OUT * 4; ++j) w[i][j / 4][j % 4] = there ? w[i][j / 4][j % 4] : 0u;
                }
                if (k + AHEAD < SWEEPS) fetch(t, k + AHEAD, raw[kk]);
                else if (t > begin) fetch(t - 1, k + AHEAD - SWEEPS, raw[kk]);
                if constexpr (ROWS) {
                    int8_t *to = out_r.codes + (uint64_t)row0 * out_r.pitch;
                    const float4 r4 = *reinterpret_cast<const float4 *>(&row_factor[t & 1u][k * 32 + down * 4]);
                    const float rs[4] = {r4.x, r4.y, r4.z, r4.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i, to += out_r.pitch) {
                        if (!all_there && row0 + i >= rows) break;
#pragma unroll
                        for (int o = 0; o < OUT; ++o) {
                            uint32_t c[E / 4];
                            encode_piece<T>(w[i][o], rs[i], false, c);
                            if (masked_rows && rs[i] == 0.f)
#pragma unroll
                                for (int j = 0; j < E / 4; ++j) c[j] = 0u;
                            store_row_piece<E, OUT>(to, o, col, cols, out_r.pitch, c);
                        }
                        if (OUT > 1 && strip == strips - 1 && piece == 0) pad_row(to, (uint64_t)OUT * cols, out_r.pitch);
                    }
                }
                const uint32_t place = (k * DOWN + down) ^ S::turned(piece);
#pragma unroll
                for (int o = 0; o < OUT; ++o)
#pragma unroll
                    for (int e = 0; e < E; e += 2) {
                        const float2 r = *reinterpret_cast<const float2 *>(factor + o * COLS + piece * E + e);
                        float p[4], q[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float v[2];
                            if constexpr (N == 2) Word<T>::unpack(w[i][o][e / 2], v);
                            else v[0] = __uint_as_float(w[i][o][e % 4]), v[1] = __uint_as_float(w[i][o][(e + 1) % 4]);
                            p[i] = __fmaf_rn(v[0], r.x, TO_INTEGER);
                            q[i] = __fmaf_rn(v[1], r.y, TO_INTEGER);
                        }
                        uint32_t a = bytes4(p[0], p[1], p[2], p[3]), b = bytes4(q[0], q[1], q[2], q[3]);
                        if (masked) {
                            if (r.x == 0.f) a = 0u;
                            if (r.y == 0.f) b = 0u;
                        }
                        tile[(o * COLS + e * 16 + piece) * WORDS + place] = a;
                        tile[(o * COLS + e * 16 + 16 + piece) * WORDS + place] = b;
                    }
            }
        };
        // compiled with and without the checks where that is faster (gated layer, 8192 x 8192 BF16, before the tails of the gates were made exact: 141 and 154 us; else the code is better short)
        if constexpr (OUT > 1 && SRC::WHOLE_ROWS) {
            if (all_there) work(Known<true>());
            else work(Known<false>());
        } else {
            work(Asked{all_there});
        }
        if (t > begin) rows_of(t - 1);
        __syncthreads();
        const uint32_t *const from = tile + slot * WORDS + ((chunk ^ (turned >> 2)) * 4);
        int8_t *const at = to_cols + (uint64_t)t * S::ROWS;
        const bool inside = (uint64_t)t * S::ROWS + chunk * 16 < out.pitch;
#pragma unroll
        for (int i = 0; i < OUT * COLS / STEP; ++i) {
            constexpr int PER = COLS / STEP;               // steps in a half
            const uint32_t more = i % PER * (STEP / 16);
            if (inside && first_col + more < cols) {
                uint4 q = *reinterpret_cast<const uint4 *>(from + i * STEP * WORDS);
                if (turned & 2) q = make_uint4(q.z, q.w, q.x, q.y);
                *reinterpret_cast<uint4 *>(at + ((uint64_t)(i / PER) * cols + more) * out.pitch) = q;
            }
        }
    }
}

// Threads that share a row (32 or a power of two from 128 on) and pieces a thread.
struct Group {
    uint32_t log, pieces;
    bool fits;
};
// A warp a row while a thread then has MOST_P pieces at most, more threads beyond that.
template <typename T, int MOST_P>
Group group_of(uint64_t cols)
{
    const uint64_t pieces = (cols + PIECE<T> - 1) / PIECE<T>;
    Group g = {5, 1, true};
    while ((int)g.pieces < MOST_P && pieces > 32u * g.pieces) g.pieces *= 2;
    if (pieces > 32u * g.pieces) {
        g.log = 7;
        if (pieces <= 256) g.pieces = 2;
    }
    while ((1u << g.log) < (uint32_t)ROW_THREADS && pieces > ((uint64_t)g.pieces << g.log)) ++g.log;
    g.fits = pieces <= ((uint64_t)g.pieces << g.log);
    return g;
}

template <typename SRC, int P, int THREADS, bool ROWS, bool COLS>
int launch_rows(const SRC &src, uint32_t rows, uint32_t cols, uint32_t group_log, const RowsOut &out, Maxima &maxima, void *stream)
{
    const uint32_t together = THREADS >> group_log, most = (uint32_t)DEFAULT_SMS * ROWS_CTAS<SRC, P, THREADS>;
    const uint64_t window = (uint64_t)(P * PIECE<typename SRC::T>) << group_log;
    const uint32_t windows = ROWS ? 1u : (uint32_t)((cols + window - 1) / window);
    uint32_t ctas = (rows + together - 1) / together;
    if (ctas > most) ctas = most;
    maxima.sets = ctas;
    return note_cuda(el::launch(rows_kernel<SRC, P, THREADS, ROWS, COLS>, dim3(ctas * windows), THREADS, 0, 1, stream, src, rows, cols, group_log, Place{ctas}, out, maxima));
}

// CTAs of 256 threads, or of a whole wider group.
template <typename SRC, int MOST_P, bool ROWS>
int launch_rows_by_width(const SRC &src, uint32_t rows, uint32_t cols, const Group &g, const RowsOut &out, void *stream)
{
    Maxima none = {};
    if ((1 << g.log) == ROW_THREADS) return launch_rows<SRC, MOST_P, ROW_THREADS, ROWS, false>(src, rows, cols, g.log, out, none, stream);
    if constexpr (MOST_P > 2)
        if (g.pieces > 2) return launch_rows<SRC, MOST_P, 256, ROWS, false>(src, rows, cols, g.log, out, none, stream);
    if (g.pieces == 2) return launch_rows<SRC, 2, 256, ROWS, false>(src, rows, cols, g.log, out, none, stream);
    return launch_rows<SRC, 1, 256, ROWS, false>(src, rows, cols, g.log, out, none, stream);
}
// One CTA on an SM where it leaves a set of maxima, so that there are few of these.
template <typename SRC>
int launch_rows_and_maxima(const SRC &src, uint32_t rows, uint32_t cols, const Group &g, const RowsOut &out, Maxima &maxima, void *stream)
{
    if (g.pieces > 2) return launch_rows<SRC, 4, 512, true, true>(src, rows, cols, g.log, out, maxima, stream);
    if (g.pieces == 2) return launch_rows<SRC, 2, 1024, true, true>(src, rows, cols, g.log, out, maxima, stream);
    return launch_rows<SRC, 1, 1024, true, true>(src, rows, cols, g.log, out, maxima, stream);
}

template <typename SRC, bool ROWS>
int launch_codes(const SRC &src, uint32_t rows, uint32_t cols, const Maxima &m, const RowsOut &ro, const ColsOut &co, void *stream)
{
    using S = Strip<SRC>;
    const uint32_t strips = (cols + S::COLS - 1) / S::COLS, tiles = (rows + S::ROWS - 1) / S::ROWS, resident = DEFAULT_SMS * S::CTAS;
    uint32_t shares = strips < resident ? resident / strips : 1u;          // all CTAs at once
    if (shares > tiles) shares = tiles;
    const uint32_t each = (tiles + shares - 1) / shares;
    shares = (tiles + each - 1) / each;
    return note_cuda(el::launch(codes_kernel<SRC, ROWS>, dim3(strips * shares), STRIP_THREADS, 0, 1, stream, src, rows, cols, strips, each, m, ro, co));
}

template <typename SRC, bool ROWS>
int launch_both(const SRC &src, uint32_t rows, uint32_t cols, const RowsOut &ro, const ColsOut &co, void *workspace, void *stream)
{
    const uint32_t window = 32 * WINDOW_PIECES<SRC::OUT> * PIECE<typename SRC::T>, windows = (uint32_t)(((uint64_t)cols + window - 1) / window), sets = (uint32_t)shares_of(rows, windows);
    const uint64_t pieces = ((uint64_t)cols + PIECE<typename SRC::T> - 1) / PIECE<typename SRC::T>;
    uint4 *const maxima = static_cast<uint4 *>(workspace);
    const Maxima m = {maxima, reinterpret_cast<uint32_t *>(maxima + sets * SRC::OUT * pieces), sets, windows};
    if (const int rc = note_cuda(el::launch(maxima_kernel<SRC, ROWS>, dim3(sets * windows), 32 * MAXIMA_WARPS, 0, 1, stream, src, rows, cols, Place{sets}, m))) return rc;
    return launch_codes<SRC, ROWS>(src, rows, cols, m, ro, co, stream);
}

// Along the rows (codes) and / or the columns (codes_t) of a source; with neither, what the source emits alone.
template <int MOST_P, typename SRC>
int quantise(const SRC &src, uint32_t rows, uint32_t cols, int8_t *codes, float *scales, int8_t *codes_t, float *scales_t, void *workspace, void *stream)
{
    const RowsOut ro = {codes, scales, row_bytes((uint64_t)SRC::OUT * cols)};
    const ColsOut co = {codes_t, scales_t, row_bytes(rows)};
    const Group g = group_of<typename SRC::T, MOST_P>(cols);
    if (codes && codes_t) {
        // a matrix of whole rows: the first kernel makes the codes along the rows (8192 x 8192 BF16 71 us; along both axes by the second one, 83 us)
        if constexpr (SRC::OUT == 1 && SRC::WHOLE_ROWS) {
            if (g.fits) {
                Maxima m = {static_cast<uint4 *>(workspace), nullptr, 0, 0};
                if (const int rc = launch_rows_and_maxima(src, rows, cols, g, ro, m, stream)) return rc;
                return launch_codes<SRC, false>(src, rows, cols, m, ro, co, stream);
            }
        }
        return launch_both<SRC, true>(src, rows, cols, ro, co, workspace, stream);
    }
    if (codes_t) return launch_both<SRC, false>(src, rows, cols, ro, co, workspace, stream);
    if (!codes) {
        if constexpr (SRC::OUT > 1) return launch_rows_by_width<SRC, MOST_P, false>(src, rows, cols, g, ro, stream);
        return OMC_OK;
    }
    if (g.fits) return launch_rows_by_width<SRC, MOST_P, true>(src, rows, cols, g, ro, stream);
    const uint32_t most = DEFAULT_SMS * 4;
    return note_cuda(el::launch(wide_rows_kernel<SRC>, dim3(rows < most ? rows : most), WIDE_THREADS, 0, 1, stream, src, rows, cols, ro));
}

}  // namespace i8
}  // namespace omc
