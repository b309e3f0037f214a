// Quantisation to 8-bit integers (i8_format.cuh) along the rows and / or the columns of what a source gives: a matrix in memory, or
// gradients computed from several (omc_gated.cu).
//
// A row's scale follows from the whole row, a column's from the whole column, so at least one of the two needs the values twice.
// First kernel: a row in the registers of 32 .. 512 threads, sixteen-byte pieces a thread; its largest magnitude by shuffles (and
// one barrier), its codes at once; each thread keeps the largest magnitudes of its own columns over all rows that it sees, which it
// leaves in the workspace, one set a CTA.  Second kernel: a CTA joins these sets for a strip of 128 columns and takes the strip's
// rows, 128 at a time: four rows of a piece a thread, whose codes of one column make a word that goes to shared memory, and from there
// 128 bytes of a column at a time to memory.  It starts with the rows that the first kernel read last, which the L2 cache still holds.
// Magnitudes are compared as bit patterns, two 16-bit values in one instruction: their order is that of the values, Inf and NaN on top.
#pragma once
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
constexpr uint32_t MOST_PARTS = 296;                                           // sets of column maxima: two CTAs on each of 148 SMs
constexpr int ROW_THREADS = 512;                                               // of the widest group that shares a row
constexpr int STRIP = 128, STRIP_ROWS = 128, STRIP_THREADS = 256;              // tile of the second kernel

// Bytes of the sets of `values` columns' maxima (as FP32 magnitudes, the widest).
inline uint64_t parts_bytes(uint64_t rows, uint64_t values)
{
    return (rows < MOST_PARTS ? rows : MOST_PARTS) * ((values + 7) / 8 * 8) * 4;
}

// A matrix in memory.
template <typename T_, bool VECTOR>
struct Matrix {
    using T = T_;
    static constexpr int IN = 1, OUT = 1;         // pieces read and made at a place
    const T *x;
    uint64_t ld;
    __device__ __forceinline__ void fetch(uint32_t row, uint32_t col, uint32_t cols, uint32_t (*raw)[4]) const
    {
        mx::load<T, VECTOR, PIECE<T>>(x + row * ld, col, cols, raw[0]);
    }
    __device__ __forceinline__ void make(const uint32_t (*raw)[4], uint32_t (*out)[4]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) out[0][i] = raw[0][i];
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
    for (int i = 0; i < E; i += 2) {
        const float2 q = el::fma2(make_float2(v[i], v[i + 1]), el::twice(r), el::twice(TO_INTEGER));
        v[i] = q.x;
        v[i + 1] = q.y;
    }
#pragma unroll
    for (int i = 0; i < E / 4; ++i) codes[i] = nan ? 0u : bytes4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
}

// A piece's codes into a row of codes from byte `at` on, `n` of them.
template <int E>
__device__ __forceinline__ void store_codes(int8_t *row, uint64_t at, uint32_t n, const uint32_t *codes)
{
    if (n >= (uint32_t)E && at % E == 0) {
        if constexpr (E == 8) *reinterpret_cast<uint2 *>(row + at) = make_uint2(codes[0], codes[1]);
        else *reinterpret_cast<uint32_t *>(row + at) = codes[0];
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if ((uint32_t)i < n) row[at + i] = (int8_t)(codes[i / 4] >> (8 * (i & 3)));
    }
}

struct RowsOut {
    int8_t *codes;            // rows of `pitch` bytes, OUT * cols codes
    float *scales;
    uint64_t pitch;
    uint4 *parts;             // [CTA][OUT][pieces of a row] magnitudes
};

// First kernel.  A row's threads: 2^group_log of them, P pieces each, piece p of thread t at column (p 2^group_log + t) E.  Without ROWS
// a row is not needed whole: blockIdx.y is a window of it.
template <typename SRC, int P, int THREADS, bool ROWS, bool COLS>
__global__ void __launch_bounds__(THREADS) rows_kernel(SRC src, uint32_t rows, uint32_t cols, uint32_t group_log, RowsOut out)
{
    using T = typename SRC::T;
    constexpr int E = PIECE<T>, IN = SRC::IN, OUT = SRC::OUT;
    __shared__ uint32_t slots[2][THREADS / 32];
    __shared__ uint4 joined[COLS ? THREADS : 1];
    const uint32_t tid = threadIdx.x, group = 1u << group_log, t = tid & (group - 1), g = tid >> group_log, together = THREADS >> group_log;
    const uint32_t window = ROWS ? 0u : blockIdx.y * (group * P * E);
    const uint32_t first_warp = g << (group_log - 5);
    el::enter_stream_order();
    uint32_t raw[P][IN][4], most[COLS ? P : 1][COLS ? OUT : 1][4];
    auto column = [&](int p) { return window + (((uint32_t)p << group_log) + t) * E; };
    auto fetch = [&](uint32_t row) {
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (row < rows && column(p) < cols) src.fetch(row, column(p), cols, raw[p]);
    };
#pragma unroll
    for (int p = 0; p < P; ++p) {
#pragma unroll
        for (int i = 0; i < IN * 4; ++i) raw[p][i / 4][i % 4] = 0u;
        if constexpr (COLS) {
#pragma unroll
            for (int i = 0; i < OUT * 4; ++i) most[p][i / 4][i % 4] = 0u;
        }
    }
    const uint32_t step = gridDim.x * together;
    uint32_t base = blockIdx.x * together, turn = 0;
    fetch(base + g);
    for (; base < rows; base += step, turn ^= 1u) {
        const uint32_t row = base + g;
        uint32_t w[P][OUT][4], top = 0u;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            src.make(raw[p], w[p]);
            if (row < rows && column(p) < cols) src.emit(row, column(p), cols, w[p]);
        }
        fetch(row + step);
        if constexpr (ROWS || COLS) {
            const bool here = row < rows;             // (behind the last row the pieces are those of a row before it)
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < OUT * 4; ++i) {
                    const uint32_t m = w[p][i / 4][i % 4] & MAGNITUDE<T>;
                    if constexpr (ROWS) top = max_magnitude<T>(top, m);
                    if constexpr (COLS) most[p][i / 4][i % 4] = here ? max_magnitude<T>(most[p][i / 4][i % 4], m) : most[p][i / 4][i % 4];
                }
        }
        if constexpr (ROWS) {
            top = __reduce_max_sync(0xFFFFFFFFu, top_bits<T>(top));
            if (group_log > 5) {                      // the same for all threads
                if ((tid & 31) == 0) slots[turn][tid >> 5] = top;
                __syncthreads();
                for (uint32_t i = 0; i < group >> 5; ++i) top = max(top, slots[turn][first_warp + i]);
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
                        // one piece a place: zeros behind the last column up to the row's end; two: the second half starts where the first one ends
                        if (OUT == 1 && column(p) < out.pitch) store_codes<E>(to, column(p), E, c);
                        if (OUT > 1 && column(p) < cols) store_codes<E>(to, (uint64_t)o * cols + column(p), cols - column(p), c);
                    }
                if (OUT > 1)
                    for (uint64_t c = (uint64_t)OUT * cols + t; c < out.pitch; c += group) to[c] = 0;
                if (t == 0) out.scales[row] = s.s;
            }
        }
    }
    if constexpr (COLS) {
        const uint32_t pieces = (cols + E - 1) / E;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int o = 0; o < OUT; ++o) {
                uint32_t *m = most[p][o];
                if (together > 1) {
                    __syncthreads();
                    joined[tid] = make_uint4(m[0], m[1], m[2], m[3]);
                    __syncthreads();
                    if (g == 0)
                        for (uint32_t i = 1; i < together; ++i) {
                            const uint4 q = joined[i * group + t];
                            m[0] = max_magnitude<T>(m[0], q.x), m[1] = max_magnitude<T>(m[1], q.y);
                            m[2] = max_magnitude<T>(m[2], q.z), m[3] = max_magnitude<T>(m[3], q.w);
                        }
                }
                if (g == 0 && column(p) < cols)
                    out.parts[((uint64_t)blockIdx.x * OUT + o) * pieces + column(p) / E] = make_uint4(m[0], m[1], m[2], m[3]);
            }
    }
}

// Rows too wide for the registers, along the rows only: read for the magnitude and again for the codes.
constexpr int WIDE_THREADS = 512;
template <typename SRC>
__global__ void __launch_bounds__(WIDE_THREADS) wide_rows_kernel(SRC src, uint32_t rows, uint32_t cols, RowsOut out)
{
    using T = typename SRC::T;
    constexpr int E = PIECE<T>, IN = SRC::IN, OUT = SRC::OUT;
    __shared__ uint32_t slots[WIDE_THREADS / 32];
    el::enter_stream_order();
    for (uint32_t row = blockIdx.x; row < rows; row += gridDim.x) {
        uint32_t raw[IN][4], w[OUT][4], top = 0u;
        for (uint32_t col = threadIdx.x * E; col < cols; col += WIDE_THREADS * E) {
            src.fetch(row, col, cols, raw);
            src.make(raw, w);
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
            src.make(raw, w);
#pragma unroll
            for (int o = 0; o < OUT; ++o) {
                uint32_t c[E / 4];
                encode_piece<T>(w[o], s.r, s.nan(), c);
                store_codes<E>(to, (uint64_t)o * cols + col, cols - col, c);
            }
        }
        for (uint64_t c = (uint64_t)OUT * cols + threadIdx.x; c < out.pitch; c += WIDE_THREADS) to[c] = 0;
        if (threadIdx.x == 0) out.scales[row] = s.s;
        __syncthreads();
    }
}

struct ColsOut {
    const uint4 *parts;
    uint32_t n_parts;
    int8_t *codes;            // OUT * cols rows of `pitch` bytes, `rows` codes
    float *scales;
    uint64_t pitch;
};

// Second kernel: blockIdx.x is a strip of 128 columns and a share of the row tiles, the last ones first.
template <typename SRC>
__global__ void __launch_bounds__(STRIP_THREADS, 2) cols_kernel(SRC src, uint32_t rows, uint32_t cols, uint32_t strips, uint32_t tiles_each, ColsOut out)
{
    using T = typename SRC::T;
    constexpr int E = PIECE<T>, IN = SRC::IN, OUT = SRC::OUT, ACROSS = STRIP / E, DOWN = STRIP_THREADS / ACROSS, SWEEP = DOWN * 4;
    constexpr int TOGETHER = IN == 1 ? 2 : 1;                      // sweeps whose loads are on their way at a time
    __shared__ __align__(16) uint32_t tile[OUT * STRIP * STRIP_ROWS / 4];
    __shared__ float factor[OUT * STRIP];
    __shared__ uint32_t any_nan;
    const uint32_t tid = threadIdx.x, piece = tid % ACROSS, down = tid / ACROSS;
    const uint32_t strip = blockIdx.x % strips, share = blockIdx.x / strips, tiles = (rows + STRIP_ROWS - 1) / STRIP_ROWS;
    const uint32_t end = tiles - share * tiles_each, begin = end > tiles_each ? end - tiles_each : 0u;
    const uint32_t col = strip * STRIP + piece * E;
    if (tid == 0) any_nan = 0u;
    el::enter_stream_order();
    // the strip's magnitudes: DOWN threads share the sets of a piece, and join what they found in shared memory
    const uint32_t pieces = (cols + E - 1) / E;
    uint4 *const found = reinterpret_cast<uint4 *>(tile);          // [DOWN][ACROSS]
#pragma unroll
    for (int o = 0; o < OUT; ++o) {
        uint4 m = make_uint4(0u, 0u, 0u, 0u);
        auto join = [&](const uint4 &q) {
            m.x = max_magnitude<T>(m.x, q.x), m.y = max_magnitude<T>(m.y, q.y);
            m.z = max_magnitude<T>(m.z, q.z), m.w = max_magnitude<T>(m.w, q.w);
        };
        if (col < cols)
#pragma unroll 4
            for (uint32_t i = down; i < out.n_parts; i += DOWN) join(out.parts[((uint64_t)i * OUT + o) * pieces + col / E]);
        __syncthreads();
        found[tid] = m;
        __syncthreads();
        if (down == 0) {
            for (int i = 1; i < DOWN; ++i) join(found[i * ACROSS + piece]);
            const uint32_t w[4] = {m.x, m.y, m.z, m.w};
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const uint32_t bits = fp32_bits<T>(sizeof(T) == 4 ? w[e % 4] : w[e / 2] >> (16 * (e & 1)) & 0xFFFFu);
                const Scale s = scale_of(bits);
                factor[o * STRIP + piece * E + e] = s.r;
                if (s.nan()) any_nan = 1u;
                if (begin == 0 && col + e < cols) out.scales[(uint64_t)o * cols + col + e] = s.s;
            }
        }
    }
    __syncthreads();
    float r[OUT][E];
#pragma unroll
    for (int i = 0; i < OUT * E; ++i) r[i / E][i % E] = factor[i / E * STRIP + piece * E + i % E];
    const bool masked = any_nan != 0u;

    for (uint32_t t = end; t-- > begin;) {
        const uint32_t r0 = t * STRIP_ROWS;
#pragma unroll 1
        for (int sweep0 = 0; sweep0 < STRIP_ROWS / SWEEP; sweep0 += TOGETHER) {
            uint32_t raw[TOGETHER][4][IN][4];
#pragma unroll
            for (int k = 0; k < TOGETHER * 4; ++k) {
                const uint32_t row = r0 + ((sweep0 + k / 4) * DOWN + down) * 4 + k % 4;
#pragma unroll
                for (int j = 0; j < IN * 4; ++j) raw[k / 4][k % 4][j / 4][j % 4] = 0u;
                if (row < rows && col < cols) src.fetch(row, col, cols, raw[k / 4][k % 4]);
            }
#pragma unroll
            for (int k = 0; k < TOGETHER; ++k) {
                const uint32_t four = (sweep0 + k) * DOWN + down;
                float v[OUT][4][E];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t w[OUT][4];
                    src.make(raw[k][i], w);
#pragma unroll
                    for (int j = 0; j < OUT * 4; ++j) Word<T>::unpack(w[j / 4][j % 4], &v[j / 4][i][j % 4 * Word<T>::N]);
                }
                // word `four` of a column, turned by the piece so that a warp's stores fall into different banks
                const uint32_t place = four ^ (piece * (32 / ACROSS));
#pragma unroll
                for (int o = 0; o < OUT; ++o)
#pragma unroll
                    for (int e = 0; e < E; e += 2) {
                        float2 q[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            q[i] = el::fma2(make_float2(v[o][i][e], v[o][i][e + 1]), make_float2(r[o][e], r[o][e + 1]), el::twice(TO_INTEGER));
                        uint32_t a = bytes4(q[0].x, q[1].x, q[2].x, q[3].x), b = bytes4(q[0].y, q[1].y, q[2].y, q[3].y);
                        if (masked) {
                            if (r[o][e] == 0.f) a = 0u;
                            if (r[o][e + 1] == 0.f) b = 0u;
                        }
                        tile[(o * STRIP + piece * E + e) * 32 + place] = a;
                        tile[(o * STRIP + piece * E + e + 1) * 32 + place] = b;
                    }
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < OUT * STRIP * 8 / STRIP_THREADS; ++i) {
            const uint32_t n = i * STRIP_THREADS + tid, c = n >> 3, chunk = n & 7, in_strip = c % STRIP;
            const uint32_t at = strip * STRIP + in_strip, first = r0 + chunk * 16;
            if (at < cols && first < out.pitch) {
                const uint32_t turned = in_strip / E * (32 / ACROSS);
                uint4 q = *reinterpret_cast<const uint4 *>(tile + c * 32 + ((chunk ^ (turned >> 2)) * 4));
                if (turned & 1) q = make_uint4(q.y, q.x, q.w, q.z);
                if (turned & 2) q = make_uint4(q.z, q.w, q.x, q.y);
                *reinterpret_cast<uint4 *>(out.codes + ((uint64_t)(c / STRIP) * cols + at) * out.pitch + first) = q;
            }
        }
        __syncthreads();
    }
}

// Threads that share a row (a power of two, 32 at least) and pieces a thread.
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
    while ((1u << g.log) < (uint32_t)ROW_THREADS && pieces > ((uint64_t)g.pieces << g.log)) ++g.log;
    g.fits = pieces <= ((uint64_t)g.pieces << g.log);
    return g;
}

template <typename SRC, int P, int THREADS, bool ROWS, bool COLS>
int launch_rows(const SRC &src, uint32_t rows, uint32_t cols, uint32_t group_log, const RowsOut &out, uint32_t &parts, void *stream)
{
    const uint32_t together = THREADS >> group_log;
    const uint64_t window = (uint64_t)(P * PIECE<typename SRC::T>) << group_log;
    const uint32_t windows = ROWS ? 1u : (uint32_t)((cols + window - 1) / window);
    const uint32_t most = COLS ? MOST_PARTS : (uint32_t)DEFAULT_SMS * (THREADS > 256 ? 2u : 4u);
    uint32_t ctas = (rows + together - 1) / together;
    if (ctas > most) ctas = most;
    parts = ctas;
    return note_cuda(el::launch(rows_kernel<SRC, P, THREADS, ROWS, COLS>, dim3(ctas, windows), THREADS, 0, 1, stream, src, rows, cols, group_log, out));
}

template <typename SRC, int MOST_P, bool ROWS, bool COLS>
int launch_rows_by_width(const SRC &src, uint32_t rows, uint32_t cols, const Group &g, const RowsOut &out, uint32_t &parts, void *stream)
{
    if ((1u << g.log) == (uint32_t)ROW_THREADS) return launch_rows<SRC, MOST_P, ROW_THREADS, ROWS, COLS>(src, rows, cols, g.log, out, parts, stream);
    if constexpr (MOST_P > 2)
        if (g.pieces > 2) return launch_rows<SRC, MOST_P, 256, ROWS, COLS>(src, rows, cols, g.log, out, parts, stream);
    if (g.pieces == 2) return launch_rows<SRC, 2, 256, ROWS, COLS>(src, rows, cols, g.log, out, parts, stream);
    return launch_rows<SRC, 1, 256, ROWS, COLS>(src, rows, cols, g.log, out, parts, stream);
}

// Along the rows (codes) and / or the columns (codes_t) of a source; with neither, what the source emits alone.
template <int MOST_P, typename SRC>
int quantise(const SRC &src, uint32_t rows, uint32_t cols, int8_t *codes, float *scales, int8_t *codes_t, float *scales_t, void *workspace, void *stream)
{
    using T = typename SRC::T;
    const Group g = group_of<T, MOST_P>(cols);
    const RowsOut ro = {codes, scales, row_bytes((uint64_t)SRC::OUT * cols), static_cast<uint4 *>(workspace)};
    uint32_t parts = 0;
    int rc = OMC_OK;
    const bool wide = codes && !g.fits;
    if (wide) {
        const uint32_t most = DEFAULT_SMS * 4;
        rc = note_cuda(el::launch(wide_rows_kernel<SRC>, dim3(rows < most ? rows : most), WIDE_THREADS, 0, 1, stream, src, rows, cols, ro));
        if (rc || !codes_t) return rc;
    }
    if (codes && !wide)
        rc = codes_t ? launch_rows_by_width<SRC, MOST_P, true, true>(src, rows, cols, g, ro, parts, stream)
                     : launch_rows_by_width<SRC, MOST_P, true, false>(src, rows, cols, g, ro, parts, stream);
    else if (codes_t)
        rc = launch_rows_by_width<SRC, MOST_P, false, true>(src, rows, cols, g, ro, parts, stream);
    else if constexpr (SRC::OUT > 1)
        rc = launch_rows_by_width<SRC, MOST_P, false, false>(src, rows, cols, g, ro, parts, stream);
    if (rc || !codes_t) return rc;
    const uint32_t strips = (cols + STRIP - 1) / STRIP, tiles = (rows + STRIP_ROWS - 1) / STRIP_ROWS;
    uint32_t shares = (DEFAULT_SMS * 3 + strips - 1) / strips;
    if (shares > tiles) shares = tiles;
    const uint32_t each = (tiles + shares - 1) / shares;
    shares = (tiles + each - 1) / each;
    const ColsOut co = {ro.parts, parts, codes_t, scales_t, row_bytes(rows)};
    return note_cuda(el::launch(cols_kernel<SRC>, dim3(strips * shares), STRIP_THREADS, 0, 1, stream, src, rows, cols, strips, each, co));
}

}  // namespace i8
}  // namespace omc
