// omc_layer_norm / omc_layer_norm_backward: normalisation over the last dimension, its gradient, and the
// gradients of its gain and bias.
//
//     y = xhat gamma + beta,  xhat = (x - mean) rstd,  rstd = (var + eps)^(-1/2), var the mean squared deviation
//     dx = rstd (g - mean(g) - xhat mean(g xhat)),  g = dy gamma;   dgamma = sum_rows dy xhat,  dbeta = sum_rows dy
//
// One pass over memory: a row stays on the chip between its moments and its results, and the column sums of the
// backward pass stay in registers over all rows of a group.  Rows of up to 8192 values; longer ones are read again, value by value, three
// times forward and (with a kernel for the column sums) three times backward: 4000 x 9000 BF16 78 and 160 us, 3.5 and 4.8 times what their
// bytes need, bound by instructions (two thirds of the issue slots).
// Measured (BF16, 32768 x 2048): forward 44 us, 6.1 TB/s, bound by memory; backward 75 us, 5.4 TB/s, bound by
// instructions (about 20 per value) at the sixteen warps that its sums leave room for.  Rows off the 4-byte boundaries take twice as
// long (16000 x 2047: 45 and 61 us): every value is read from shared memory and stored on its own.
#include <cuda_runtime.h>

#include <type_traits>

#include "element.cuh"
#include "omc_internal.h"
#include "row_copy.h"

namespace {

using namespace omc;
using el::add2;
using el::fma2;
using el::mul2;
using el::twice;

constexpr int THREADS = 256;

// The CTA's sum of v, known to all its threads; `room` holds a float per warp.
__device__ __forceinline__ float cta_sum(float v, float *room)
{
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) room[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.f;
    for (uint32_t w = 0; w < blockDim.x / 32; ++w) s += room[w];
    return s;
}

// The mean of the deviations from a first mean corrects it, unless that mean is not finite (Inf stays Inf, NaN NaN) or the
// deviations overflowed.
__device__ __forceinline__ float finite_or_0(float v) { return isfinite(v) ? v : 0.f; }
// Variance from the mean squared deviation `around` a mean that is `off` from the right one.  Not below zero after rounding,
// but a NaN stays one (fmaxf would make it 0); where the squares overflowed it is Inf, since off is finite.
__device__ __forceinline__ float variance(float around, float off)
{
    float v;
    asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(v) : "f"(__fmaf_rn(-off, off, around)));
    return v;
}

// Any width: a CTA per row, three passes over it.
template <typename T>
__global__ void __launch_bounds__(THREADS)
norm_wide_kernel(const T *x, uint32_t cols, uint64_t ld, const float *gamma, const float *beta,
                 float eps, T *y, uint64_t ldy, float *__restrict__ mean_out, float *__restrict__ rstd_out)
{
    el::enter_stream_order();
    __shared__ float room[THREADS / 32];
    const uint64_t row = blockIdx.x;
    const T *xr = x + row * ld;
    T *yr = y + row * ldy;
    float s = 0.f;
    for (uint32_t c = threadIdx.x; c < cols; c += THREADS) s += el::to_float(xr[c]);
    const float near = cta_sum(s, room) / (float)cols;
    s = 0.f;
    float s1 = 0.f;
    for (uint32_t c = threadIdx.x; c < cols; c += THREADS) {
        const float d = el::to_float(xr[c]) - near;
        s1 += d;
        s = __fmaf_rn(d, d, s);
    }
    const float off = finite_or_0(cta_sum(s1, room) / (float)cols), mean = near + off;
    const float rstd = __frsqrt_rn(variance(cta_sum(s, room) / (float)cols, off) + eps);
    for (uint32_t c = threadIdx.x; c < cols; c += THREADS)
        yr[c] = el::from_float<T>(__fmaf_rn((el::to_float(xr[c]) - near - off) * rstd, gamma[c], beta[c]));
    if (threadIdx.x == 0) {
        if (mean_out) mean_out[row] = mean;
        if (rstd_out) rstd_out[row] = rstd;
    }
}

template <typename T>
__global__ void __launch_bounds__(THREADS)
norm_backward_wide_kernel(const T *dy, uint64_t ld_dy, const T *x, uint64_t ld_x, uint32_t cols,
                          const float *gamma, const float *mean_in, const float *rstd_in,
                          T *dx, uint64_t ld_dx)
{
    el::enter_stream_order();
    __shared__ float room[THREADS / 32];
    const uint64_t row = blockIdx.x;
    const T *xr = x + row * ld_x, *gr = dy + row * ld_dy;
    T *dr = dx + row * ld_dx;
    const float mean = mean_in[row], rstd = rstd_in[row];
    float s1 = 0.f, s2 = 0.f;
    for (uint32_t c = threadIdx.x; c < cols; c += THREADS) {
        const float g = el::to_float(gr[c]) * gamma[c], h = (el::to_float(xr[c]) - mean) * rstd;
        s1 += g;
        s2 = __fmaf_rn(g, h, s2);
    }
    const float m1 = cta_sum(s1, room) / (float)cols, m2 = cta_sum(s2, room) / (float)cols;
    for (uint32_t c = threadIdx.x; c < cols; c += THREADS) {
        const float g = el::to_float(gr[c]) * gamma[c], h = (el::to_float(xr[c]) - mean) * rstd;
        dr[c] = el::from_float<T>((g - m1 - h * m2) * rstd);
    }
}

// Column sums of part of the rows: a thread per column, blockIdx.y the part.
template <typename T>
__global__ void __launch_bounds__(THREADS)
norm_columns_kernel(const T *dy, uint64_t ld_dy, const T *x, uint64_t ld_x, uint32_t rows, uint32_t cols,
                    const float *mean_in, const float *rstd_in, float *__restrict__ part)
{
    el::enter_stream_order();
    const uint32_t c = blockIdx.x * THREADS + threadIdx.x;
    if (c >= cols) return;
    float sg = 0.f, sb = 0.f;
    for (uint64_t r = blockIdx.y; r < rows; r += gridDim.y) {
        const float g = el::to_float(dy[r * ld_dy + c]), h = (el::to_float(x[r * ld_x + c]) - mean_in[r]) * rstd_in[r];
        sg = __fmaf_rn(g, h, sg);
        sb += g;
    }
    part[(uint64_t)blockIdx.y * 2 * cols + c] = sg;
    part[(uint64_t)blockIdx.y * 2 * cols + cols + c] = sb;
}

// ---- rows that fit in registers ------------------------------------------------------------------
// A row is held by a group of G threads, E values each: 8 or 16 lanes of a warp (narrow rows: the warp works on four or
// two rows at a time), a warp, or several warps.  Each group walks over rows of its own.  The rows ahead are on their
// way into a ring of row images in shared memory (cp.async), so that what is in flight takes no registers.
//   ALIGN  bytes on whose multiples every row begins and that divide its length: 16, 4 or that of one value.  A row's units,
//          ALIGN bytes each, are dealt out to the threads.  With 16 a thread copies and reads its own units: no barrier.  Otherwise the
//          image starts at the 16-byte boundary below the row (never below the matrix), and the group meets
//          between copying and reading.
template <typename T, int ALIGN, int E, int L>
struct Row {
    static constexpr uint32_t SIZE = sizeof(T), PER = ALIGN / SIZE;   // values of a unit
    static constexpr int UNITS = E / PER;                             // of a thread
    static_assert(UNITS >= 1 && E % PER == 0, "");

    // unit i of thread t, without i L: a warp's units lie together, so that the others are at constant distances
    static __device__ __forceinline__ uint32_t first(uint32_t t) { return L == 32 ? (t & ~31u) * UNITS + (t & 31u) : t; }

    static __host__ __device__ constexpr uint32_t image_bytes(uint32_t G) { return G * E * SIZE + (ALIGN == 16 ? 0 : 16); }

    static __device__ __forceinline__ void copy16(uint32_t dst, const void *src, uint32_t bytes)      // the rest of the 16 becomes 0
    {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
    }
    static __device__ __forceinline__ void fetch(uint8_t *image, const T *row, bool from_below, uint32_t cols, uint32_t t, uint32_t G)
    {
        const uint32_t dst = (uint32_t)__cvta_generic_to_shared(image);
        if constexpr (ALIGN == 16) {
            const uint32_t u = first(t);
#pragma unroll
            for (int i = 0; i < UNITS; ++i)
                if ((u + i * L) * PER < cols) copy16(dst + u * 16 + i * L * 16, row + u * PER + i * L * PER, 16);
        } else {
            const uint32_t skip = row_skip(reinterpret_cast<uintptr_t>(row)), total = skip + cols * SIZE;
            const uint8_t *src = reinterpret_cast<const uint8_t *>(row) - skip;
            constexpr int CHUNKS = (E * SIZE + 15) / 16;
#pragma unroll
            for (int i = 0; i <= CHUNKS; ++i) {
                const uint32_t k = i * G + t;
                if (k * 16 >= total) break;
                if (by_value(k, from_below)) {              // nothing before the matrix is read
                    for (uint32_t j = skip; j < 16 && j < total; j += SIZE)
                        *reinterpret_cast<T *>(image + j) = *reinterpret_cast<const T *>(src + j);
                } else {
                    copy16(dst + k * 16, src + k * 16, min(16u, total - k * 16));
                }
            }
        }
    }
    static __device__ __forceinline__ void values(const uint8_t *image, const T *row, uint32_t t, float *v)
    {
        constexpr int N = el::Word<T>::N;
        const uint8_t *p = image + (ALIGN == 16 ? 0 : row_skip(reinterpret_cast<uintptr_t>(row))) + first(t) * ALIGN;      // (behind the row: never used)
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            if constexpr (ALIGN == 16) {
                const uint4 w = *reinterpret_cast<const uint4 *>(p + i * L * 16);
                el::Word<T>::unpack(w.x, v + i * PER);
                el::Word<T>::unpack(w.y, v + i * PER + N);
                el::Word<T>::unpack(w.z, v + i * PER + 2 * N);
                el::Word<T>::unpack(w.w, v + i * PER + 3 * N);
            } else if constexpr (ALIGN == 4) {
                el::Word<T>::unpack(*reinterpret_cast<const uint32_t *>(p + i * L * 4), v + i * PER);
            } else {
                v[i] = el::to_float(*reinterpret_cast<const T *>(p + i * L * SIZE));
            }
        }
    }
    static __device__ __forceinline__ void store(T *row, uint32_t cols, uint32_t t, const float *v)
    {
        constexpr int N = el::Word<T>::N;
        const uint32_t c0 = first(t) * PER;
        row += c0;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            constexpr uint32_t D = L * PER;
            const float *p = v + i * PER;
            if (c0 + i * D >= cols) continue;
            if constexpr (ALIGN == 16)
                *reinterpret_cast<uint4 *>(row + i * D) = make_uint4(el::Word<T>::pack(p), el::Word<T>::pack(p + N), el::Word<T>::pack(p + 2 * N),
                                                                 el::Word<T>::pack(p + 3 * N));
            else if constexpr (ALIGN == 4)
                *reinterpret_cast<uint32_t *>(row + i * D) = el::Word<T>::pack(p);
            else
                row[i * D] = el::from_float<T>(*p);
        }
    }
    // The thread's values of an FP32 vector of the row's length; 0 behind its end.
    static __device__ __forceinline__ void vector(const float *p, uint32_t cols, uint32_t t, float *v)
    {
        const uint32_t u = first(t);
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const uint32_t c = (u + i * L) * PER;
            if constexpr (PER % 4 == 0) {
#pragma unroll
                for (uint32_t j = 0; j < PER; j += 4) {
                    const float4 f = c < cols ? *reinterpret_cast<const float4 *>(p + c + j) : make_float4(0.f, 0.f, 0.f, 0.f);
                    v[i * PER + j] = f.x;
                    v[i * PER + j + 1] = f.y;
                    v[i * PER + j + 2] = f.z;
                    v[i * PER + j + 3] = f.w;
                }
            } else if constexpr (PER == 2) {
                const float2 f = c < cols ? *reinterpret_cast<const float2 *>(p + c) : make_float2(0.f, 0.f);
                v[i * 2] = f.x;
                v[i * 2 + 1] = f.y;
            } else {
                v[i] = c < cols ? p[c] : 0.f;
            }
        }
    }
    // Sets the values behind the row's end.
    static __device__ __forceinline__ void fill(uint32_t cols, uint32_t t, float *v, float to)
    {
        const uint32_t u = first(t);
#pragma unroll
        for (int i = 0; i < UNITS; ++i)
            if ((u + i * L) * PER >= cols) {
#pragma unroll
                for (uint32_t j = 0; j < PER; ++j) v[i * PER + j] = to;
            }
    }
    // Calls f(index of the value in v, column) for the values inside the row.
    template <typename F>
    static __device__ __forceinline__ void each(uint32_t cols, uint32_t t, F f)
    {
        const uint32_t u = first(t);
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const uint32_t c = (u + i * L) * PER;
            if (c < cols) {
#pragma unroll
                for (uint32_t j = 0; j < PER; ++j) f(i * PER + j, c + j);
            }
        }
    }
};
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// Sums over a group, known to all its threads.  Groups of several warps (L = 32): consecutive calls use the two halves of
// `room` in turn, so that one barrier per call is enough: who writes a half again has passed the barrier of the call between.
template <int L>
struct Group {
    uint32_t warps, index, thread;
    float *room;        // [2][32] of this group
    uint32_t turn;

    __device__ __forceinline__ Group(uint32_t warps_, float *rooms)
        : warps(warps_), index(threadIdx.x / (L * warps_)), thread(threadIdx.x - index * L * warps_), room(rooms + index * 64), turn(0) {}

    __device__ __forceinline__ void meet()
    {
        if (L == 32 && warps > 1) asm volatile("bar.sync %0, %1;" ::"r"(index + 1), "r"(warps * 32) : "memory");
        else __syncwarp();
    }
    // One value: every lane ends with the total.
    __device__ __forceinline__ float sum(float v)
    {
#pragma unroll
        for (int d = L / 2; d >= 1; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
        if (L == 32 && warps > 1) {
            float *half = room + 32 * (turn & 1);
            ++turn;
            const uint32_t lane = threadIdx.x & 31;
            if (lane == 0) half[thread >> 5] = v;
            meet();
            v = (lane & 15) < warps ? half[lane & 15] : 0.f;
#pragma unroll
            for (int d = 8; d >= 1; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
        }
        return v;
    }
    // Two values: the lower half of the lanes adds up the first, the upper half the second.
    __device__ __forceinline__ float2 sum2(float a, float b)
    {
        const uint32_t lane = threadIdx.x & 31;
        const bool upper = (lane & (L / 2)) != 0;
        float v = (upper ? b : a) + __shfl_xor_sync(0xFFFFFFFFu, upper ? a : b, L / 2);
#pragma unroll
        for (int d = L / 4; d >= 1; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
        if (L == 32 && warps > 1) {
            float *half = room + 32 * (turn & 1);
            ++turn;
            if ((lane & 15) == 0) half[(thread >> 5) + (upper ? 16 : 0)] = v;
            meet();
            v = (lane & 15) < warps ? half[lane] : 0.f;
#pragma unroll
            for (int d = 8; d >= 1; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
        }
        const float other = __shfl_xor_sync(0xFFFFFFFFu, v, L / 2);
        return upper ? make_float2(other, v) : make_float2(v, other);
    }
};

constexpr int MAX_GROUPS = 15;      // of several warps: named barriers 1 .. 15

constexpr int STAGES = 3;      // row images of a group: two ahead of the one in work

// Registers a thread of the forward kernel gets: what lets 1024, 768 or 512 threads share an SM.
template <int ALIGN, int E> constexpr int forward_registers = E == 8 ? 64 : E == 16 && ALIGN == 16 ? 80 : 128;

template <typename T, int ALIGN, int E, int L>
__global__ void __maxnreg__((forward_registers<ALIGN, E>))
norm_kernel(const T *x, uint32_t rows, uint32_t cols, uint64_t ld, const float *gamma, const float *beta, float eps,
            T *y, uint64_t ldy, float *__restrict__ mean_out, float *__restrict__ rstd_out, uint32_t warps,
            uint32_t below)
{
    using R = Row<T, ALIGN, E, L>;
    constexpr int S = STAGES;
    __shared__ float room[L == 32 ? 16 * 64 : 1];
    extern __shared__ __align__(16) uint8_t images[];
    Group<L> g(warps, room);
    const uint32_t G = warps * L, groups = blockDim.x / G, t = g.thread, bytes = R::image_bytes(G);
    uint8_t *ring = images + g.index * S * bytes;
    const float inv = 1.f / (float)cols;
    el::enter_stream_order();
    const uint32_t step = gridDim.x * groups, first = blockIdx.x * groups + g.index;
    const bool whole = cols == G * E;                      // no thread holds anything behind a row's end
    const T *src = x + (uint64_t)first * ld, *row_x = src;
    T *row_y = y + (uint64_t)first * ldy;
    uint32_t coming = first;                               // the row to fetch next (no overflow: rows < 2^31, step < 2^14)
    auto fetch = [&](uint32_t s) {
        if (coming < rows) R::fetch(ring + s * bytes, src, coming < below, cols, t, G);
        commit_copies();
        coming += step;
        src += step * ld;
    };
#pragma unroll
    for (int s = 0; s < S - 1; ++s) fetch(s);
    float ga[E], be[E];
    R::vector(gamma, cols, t, ga);
    R::vector(beta, cols, t, be);
    uint32_t now = 0, ahead = S - 1;
    const uint32_t neighbour = L < 32 ? g.index % (32 / L) : 0u;      // a warp's groups go on as long as the first has a row
    for (uint32_t row = first; row - neighbour < rows; row += step) {
        fetch(ahead);                                      // where the row before was: its group has met since
        wait_copies<S - 1>();
        if (ALIGN != 16) g.meet();
        float v[E];
        R::values(ring + now * bytes, row_x, t, v);
        now = now + 1 == S ? 0 : now + 1;
        ahead = ahead + 1 == S ? 0 : ahead + 1;
        if (!whole) R::fill(cols, t, v, 0.f);
        float2 *p = reinterpret_cast<float2 *>(v);
        float2 s = twice(0.f);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) s = add2(s, p[i]);
        // the mean of the deviations from the first mean corrects it: a row of equal values leaves zeros, not the
        // rounding of the sum times 1 / sqrt(eps)
        const float near = g.sum(s.x + s.y) * inv;
#pragma unroll
        for (int i = 0; i < E / 2; ++i) p[i] = add2(p[i], twice(-near));
        if (!whole) R::fill(cols, t, v, 0.f);              // (not the mean before: Inf - Inf)
        s = twice(0.f);
        float2 s1 = twice(0.f);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            s1 = add2(s1, p[i]);
            s = fma2(p[i], p[i], s);
        }
        const float2 m = g.sum2(s1.x + s1.y, s.x + s.y);
        const float off = finite_or_0(m.x * inv), mean = near + off, rstd = __frsqrt_rn(variance(m.y * inv, off) + eps);
#pragma unroll
        for (int i = 0; i < E / 2; ++i)
            p[i] = fma2(mul2(add2(p[i], twice(-off)), twice(rstd)), make_float2(ga[2 * i], ga[2 * i + 1]), make_float2(be[2 * i], be[2 * i + 1]));
        if (L < 32 && row >= rows) break;                  // the neighbours' last row
        R::store(row_y, cols, t, v);
        if (t == 0) {
            if (mean_out) mean_out[row] = mean;
            if (rstd_out) rstd_out[row] = rstd;
        }
        if (ALIGN != 16) row_x += step * ld;
        row_y += step * ldy;
    }
}

// dx, and this CTA's part of the column sums: each thread adds up its own columns over its group's rows in registers.
template <typename T, int ALIGN, int E, int L>
__global__ void __launch_bounds__(E == 8 ? 384 : 512, E == 8 ? 2 : 1)
norm_backward_kernel(const T *dy, uint64_t ld_dy, const T *x, uint64_t ld_x, uint32_t rows, uint32_t cols, const float *gamma,
                     const float *mean_in, const float *rstd_in, T *dx, uint64_t ld_dx, float *__restrict__ part,
                     uint32_t warps, uint32_t below_x, uint32_t below_d)
{
    using R = Row<T, ALIGN, E, L>;
    constexpr int S = STAGES;
    __shared__ float room[L == 32 ? 16 * 64 : 1];
    extern __shared__ __align__(16) uint8_t images[];
    Group<L> g(warps, room);
    const uint32_t G = warps * L, groups = blockDim.x / G, t = g.thread, bytes = R::image_bytes(G);
    uint8_t *ring = images + g.index * S * 2 * bytes;      // x and dy
    const float inv = 1.f / (float)cols;
    el::enter_stream_order();
    const uint32_t step = gridDim.x * groups, first = blockIdx.x * groups + g.index;
    const bool whole = cols == G * E;                      // no thread holds anything behind a row's end
    const T *src_x = x + (uint64_t)first * ld_x, *src_d = dy + (uint64_t)first * ld_dy, *row_x = src_x, *row_d = src_d;
    T *row_dx = dx + (uint64_t)first * ld_dx;
    uint32_t coming = first;                               // the row to fetch next (no overflow: rows < 2^31, step < 2^14)
    auto fetch = [&](uint32_t s) {
        if (coming < rows) {
            R::fetch(ring + s * 2 * bytes, src_x, coming < below_x, cols, t, G);
            R::fetch(ring + s * 2 * bytes + bytes, src_d, coming < below_d, cols, t, G);
        }
        commit_copies();
        coming += step;
        src_x += step * ld_x;
        src_d += step * ld_dy;
    };
#pragma unroll
    for (int s = 0; s < S - 1; ++s) fetch(s);
    float2 sg[E / 2], sb[E / 2];
#pragma unroll
    for (int i = 0; i < E / 2; ++i) sg[i] = sb[i] = twice(0.f);
    float mean = 0.f, rstd = 0.f;
    if (first < rows) {
        mean = mean_in[first];
        rstd = rstd_in[first];
    }
    uint32_t now = 0, ahead = S - 1;
    const uint32_t neighbour = L < 32 ? g.index % (32 / L) : 0u;      // a warp's groups go on as long as the first has a row
    for (uint32_t row = first; row - neighbour < rows; row += step) {
        fetch(ahead);                                      // where the row before was: its group has met since
        float mu = mean, rs = rstd;
        if (row + step < rows) {
            mean = mean_in[row + step];
            rstd = rstd_in[row + step];
        }
        wait_copies<S - 1>();
        if (ALIGN != 16) g.meet();
        float h[E], d[E];
        R::values(ring + now * 2 * bytes, row_x, t, h);
        R::values(ring + now * 2 * bytes + bytes, row_d, t, d);
        now = now + 1 == S ? 0 : now + 1;
        ahead = ahead + 1 == S ? 0 : ahead + 1;
        if (!whole) {
            R::fill(cols, t, h, mu);
            R::fill(cols, t, d, 0.f);
        }
        if (L < 32 && row >= rows) {                       // no row of its own: nothing to add to the columns
#pragma unroll
            for (int i = 0; i < E; ++i) h[i] = d[i] = 0.f;
            mu = rs = 0.f;
        }
        float ga[E];                                       // from L1 each time: registers are short here
        R::vector(gamma, cols, t, ga);
        float2 *ph = reinterpret_cast<float2 *>(h), *pd = reinterpret_cast<float2 *>(d);
        float2 s1 = twice(0.f), s2 = twice(0.f);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            ph[i] = mul2(add2(ph[i], twice(-mu)), twice(rs));
            sg[i] = fma2(pd[i], ph[i], sg[i]);
            sb[i] = add2(sb[i], pd[i]);
            pd[i] = mul2(pd[i], make_float2(ga[2 * i], ga[2 * i + 1]));
            s1 = add2(s1, pd[i]);
            s2 = fma2(pd[i], ph[i], s2);
        }
        const float2 m = g.sum2(s1.x + s1.y, s2.x + s2.y);
        const float2 m1 = twice(-(m.x * inv)), m2 = twice(-(m.y * inv));
#pragma unroll
        for (int i = 0; i < E / 2; ++i) pd[i] = mul2(fma2(ph[i], m2, add2(pd[i], m1)), twice(rs));
        if (L < 32 && row >= rows) break;                  // the neighbours' last row
        R::store(row_dx, cols, t, d);
        if (ALIGN != 16) {
            row_x += step * ld_x;
            row_d += step * ld_dy;
        }
        row_dx += step * ld_dx;
    }
    // the groups' sums side by side where the images were (2 x cols each), added in the groups' order
    __syncthreads();
    float *columns = reinterpret_cast<float *>(images);
    R::each(cols, t, [&](int i, uint32_t c) {
        columns[g.index * 2 * cols + c] = i & 1 ? sg[i / 2].y : sg[i / 2].x;
        columns[(g.index * 2 + 1) * cols + c] = i & 1 ? sb[i / 2].y : sb[i / 2].x;
    });
    __syncthreads();
    float *out = part + (uint64_t)blockIdx.x * 2 * cols;
    for (uint32_t c = threadIdx.x; c < 2 * cols; c += blockDim.x) {
        float sum = columns[c];
        for (uint32_t k = 1; k < groups; ++k) sum += columns[k * 2 * cols + c];
        out[c] = sum;
    }
}

// Sums of the parts: 32 columns per CTA, 32 warps that take every 32nd part, then one that adds their sums.
constexpr int FINISH_WARPS = 32;
__global__ void __launch_bounds__(32 * FINISH_WARPS)
norm_finish_kernel(const float *part, uint32_t parts, uint32_t cols, float *__restrict__ dgamma, float *__restrict__ dbeta)
{
    el::enter_stream_order();
    __shared__ float room[FINISH_WARPS][33];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (c < 2 * cols)
        for (uint32_t p = warp; p < parts; p += FINISH_WARPS) s += part[(uint64_t)p * 2 * cols + c];
    room[warp][lane] = s;
    __syncthreads();
    // warp w adds up column w's sums, lane l holding warp l's
    s = room[lane][warp];
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    const uint32_t k = blockIdx.x * 32 + warp;
    if (lane == 0 && k < 2 * cols) {
        if (k < cols) dgamma[k] = s;
        else dbeta[k - cols] = s;
    }
}

// Parts of the column sums: two CTAs on each of the 148 SMs that the kernels are laid out for.  (Not taken from the device:
// the order of the additions follows from the shape alone.)
constexpr uint32_t MAX_PARTS = 2 * DEFAULT_SMS;
uint32_t parts_of(uint64_t rows) { return (uint32_t)(rows < MAX_PARTS ? rows : MAX_PARTS); }

bool shape_ok(uint64_t rows, uint64_t cols) { return cols >= 1 && rows < (1ull << 31) && cols < (1ull << 30); }

// Bytes on whose multiples the matrix's rows begin and end: 16, 4 or the size of a value.
template <typename T>
int align_of(const void *p, uint64_t ld, uint64_t cols)
{
    const uint64_t all = reinterpret_cast<uintptr_t>(p) | (ld * sizeof(T)) | (cols * sizeof(T));
    return all % 16 == 0 ? 16 : all % 4 == 0 ? 4 : (int)sizeof(T);
}

constexpr uint32_t REGISTER_COLS = 8192;      // 16 warps of 16 values a thread

// Calls f.operator()<ALIGN, E, L>() with the instantiation for rows of this width: narrow rows several to a warp, up to 256 values a
// warp with eight a thread, longer ones with sixteen (per thread and row about 200 instructions do not depend on the number
// of values: 32768 x 2048 BF16 backward 104 us with eight, 83 us with sixteen).
template <int ALIGN, typename F>
int with_width(uint32_t cols, F f)
{
    if (cols <= 64) return f.template operator()<ALIGN, 8, 8>();
    if (cols <= 128) return f.template operator()<ALIGN, 8, 16>();
    if (cols <= 256) return f.template operator()<ALIGN, 8, 32>();
    return f.template operator()<ALIGN, 16, 32>();
}
template <typename T, typename F>
int with_rows(int align, uint32_t cols, F f)
{
    if (align == 16) return with_width<16>(cols, f);
    if constexpr (sizeof(T) == 2) {
        if (align == 2) return with_width<2>(cols, f);
    }
    return with_width<4>(cols, f);
}

template <typename T>
struct Forward {
    const void *x;
    uint32_t rows, cols;
    uint64_t ld;
    const float *gamma, *beta;
    float eps;
    void *y;
    uint64_t ldy;
    float *mean, *rstd;
    void *stream;

    template <int ALIGN, int E, int L>
    int operator()() const
    {
        // Without sums to keep over the rows there is room for 32 values a thread (8000 x 8192 BF16 61 us with 16, 45 us with 32;
        // 32768 x 2048 46.5 and 44 us); off the 16-byte boundaries they spill.
        if constexpr (ALIGN == 16 && E == 16) {
            if (cols > 512) return this->template operator()<16, 32, 32>();
        }
        const uint32_t warps = (cols + L * E - 1) / (L * E), G = warps * L, groups = G >= 256 ? 1 : 256 / G;
        const uint32_t ctas = (rows + groups - 1) / groups, threads = groups * G;
        const uint32_t smem = groups * STAGES * Row<T, ALIGN, E, L>::image_bytes(G);
        // as many CTAs as are resident
        const uint32_t by_regs = 65536 / (threads * forward_registers<ALIGN, E>), by_smem = 220 * 1024 / (smem + 5 * 1024);
        const uint32_t most = DEFAULT_SMS * (by_regs < by_smem ? by_regs : by_smem);
        if (const int rc = el::allow_smem<norm_kernel<T, ALIGN, E, L>>(smem)) return rc;
        return note_cuda(el::launch(norm_kernel<T, ALIGN, E, L>, dim3(ctas < most ? ctas : most), threads, smem, 1, stream,
                                    static_cast<const T *>(x), rows, cols, ld, gamma, beta, eps, static_cast<T *>(y), ldy, mean, rstd, warps,
                                    rows_from_below(reinterpret_cast<uintptr_t>(x), ld * sizeof(T))));
    }
};

template <typename T>
int forward(const void *x, uint64_t rows, uint64_t cols, uint64_t ld, const float *gamma, const float *beta, float eps, void *y,
            uint64_t ldy, float *mean, float *rstd, void *stream)
{
    if (cols > REGISTER_COLS)
        return note_cuda(el::launch(norm_wide_kernel<T>, dim3((uint32_t)rows), THREADS, 0, 1, stream, static_cast<const T *>(x),
                                    (uint32_t)cols, ld, gamma, beta, eps, static_cast<T *>(y), ldy, mean, rstd));
    const int ax = align_of<T>(x, ld, cols), ay = align_of<T>(y, ldy, cols);
    return with_rows<T>(ax < ay ? ax : ay, (uint32_t)cols,
                        Forward<T>{x, (uint32_t)rows, (uint32_t)cols, ld, gamma, beta, eps, y, ldy, mean, rstd, stream});
}

template <typename T>
struct Backward {
    const void *dy;
    uint64_t ld_dy;
    const void *x;
    uint64_t ld_x;
    uint32_t rows, cols;
    const float *gamma, *mean, *rstd;
    void *dx;
    uint64_t ld_dx;
    float *part;
    uint32_t *parts;
    void *stream;

    template <int ALIGN, int E, int L>
    int operator()() const
    {
        const uint32_t warps = (cols + L * E - 1) / (L * E), G = warps * L;
        const uint32_t room = E == 8 ? 384 : 512, groups = G >= room ? 1 : warps == 1 || room / G < MAX_GROUPS ? room / G : MAX_GROUPS;
        const uint32_t ctas = (rows + groups - 1) / groups;
        const uint32_t ring = groups * STAGES * 2 * Row<T, ALIGN, E, L>::image_bytes(G);
        const uint32_t joined = groups * 8 * cols, smem = ring > joined ? ring : joined;
        const uint32_t most = E == 8 ? MAX_PARTS : MAX_PARTS / 2;      // as many CTAs as are resident
        *parts = ctas < most ? ctas : most;
        if (const int rc = el::allow_smem<norm_backward_kernel<T, ALIGN, E, L>>(smem)) return rc;
        return note_cuda(el::launch(norm_backward_kernel<T, ALIGN, E, L>, dim3(*parts), groups * G, smem, 1, stream, static_cast<const T *>(dy),
                                    ld_dy, static_cast<const T *>(x), ld_x, rows, cols, gamma, mean, rstd, static_cast<T *>(dx), ld_dx, part, warps,
                                    rows_from_below(reinterpret_cast<uintptr_t>(x), ld_x * sizeof(T)), rows_from_below(reinterpret_cast<uintptr_t>(dy), ld_dy * sizeof(T))));
    }
};

template <typename T>
int backward(const void *dy, uint64_t ld_dy, const void *x, uint64_t ld_x, uint64_t rows, uint64_t cols, const float *gamma,
             const float *mean, const float *rstd, void *dx, uint64_t ld_dx, float *dgamma, float *dbeta, float *part, void *stream)
{
    const uint32_t c = (uint32_t)cols;
    uint32_t parts = parts_of(rows);
    int rc = 0;
    if (rows && cols <= REGISTER_COLS) {
        const int ad = align_of<T>(dy, ld_dy, cols), ax = align_of<T>(x, ld_x, cols), ao = align_of<T>(dx, ld_dx, cols);
        const int align = ad < ax ? (ad < ao ? ad : ao) : (ax < ao ? ax : ao);
        rc = with_rows<T>(align, c, Backward<T>{dy, ld_dy, x, ld_x, (uint32_t)rows, c, gamma, mean, rstd, dx, ld_dx, part, &parts, stream});
    } else if (rows) {
        // the column sums first: dx may overwrite dy or x
        rc = note_cuda(el::launch(norm_columns_kernel<T>, dim3((c + THREADS - 1) / THREADS, parts), THREADS, 0, 1, stream,
                                  static_cast<const T *>(dy), ld_dy, static_cast<const T *>(x), ld_x, (uint32_t)rows, c, mean, rstd, part));
        if (!rc)
            rc = note_cuda(el::launch(norm_backward_wide_kernel<T>, dim3((uint32_t)rows), THREADS, 0, 1, stream, static_cast<const T *>(dy),
                                      ld_dy, static_cast<const T *>(x), ld_x, c, gamma, mean, rstd, static_cast<T *>(dx), ld_dx));
    }
    if (!rc)
        rc = note_cuda(el::launch(norm_finish_kernel, dim3((2 * c + 31) / 32), 32 * FINISH_WARPS, 0, 1, stream, static_cast<const float *>(part), parts, c,
                                  dgamma, dbeta));
    return rc;
}

}  // namespace

extern "C" int omc_layer_norm(const void *x, int type, uint64_t rows, uint64_t cols, uint64_t ld, const float *gamma, const float *beta,
                              float eps, void *y, uint64_t ldy, float *mean, float *rstd, void *stream)
{
    if (!el::type_ok(type)) return OMC_ERR_INVALID_ARG;
    if (!shape_ok(rows, cols) || ld < cols || ldy < cols || !(eps >= 0.f)) return OMC_ERR_INVALID_ARG;
    if (rows == 0) return OMC_OK;
    if (!x || !gamma || !beta || !y) return OMC_ERR_NULL_PTR;
    if (reinterpret_cast<uintptr_t>(x) % el::size_of(type) || reinterpret_cast<uintptr_t>(y) % el::size_of(type) ||
        !el::aligned16(gamma) || !el::aligned16(beta) || reinterpret_cast<uintptr_t>(mean) % 4 || reinterpret_cast<uintptr_t>(rstd) % 4)
        return OMC_ERR_MISALIGNED;
#define OMC_CALL(T) forward<T>(x, rows, cols, ld, gamma, beta, eps, y, ldy, mean, rstd, stream)
    return type == OMC_TYPE_F32 ? OMC_CALL(float) : type == OMC_TYPE_F16 ? OMC_CALL(__half) : OMC_CALL(__nv_bfloat16);
#undef OMC_CALL
}

extern "C" int omc_layer_norm_workspace(uint64_t rows, uint64_t cols, uint64_t *bytes)
{
    if (!shape_ok(rows, cols)) return OMC_ERR_INVALID_ARG;
    if (!bytes) return OMC_ERR_NULL_PTR;
    *bytes = (uint64_t)(parts_of(rows) ? parts_of(rows) : 1) * 2 * cols * sizeof(float);
    return OMC_OK;
}

extern "C" int omc_layer_norm_backward(const void *dy, uint64_t ld_dy, const void *x, uint64_t ld_x, int type, uint64_t rows, uint64_t cols,
                                       const float *gamma, const float *mean, const float *rstd, void *dx, uint64_t ld_dx, float *dgamma,
                                       float *dbeta, void *workspace, void *stream)
{
    if (!el::type_ok(type)) return OMC_ERR_INVALID_ARG;
    if (!shape_ok(rows, cols) || ld_dy < cols || ld_x < cols || ld_dx < cols) return OMC_ERR_INVALID_ARG;
    if (!gamma || !dgamma || !dbeta || !workspace) return OMC_ERR_NULL_PTR;
    if (rows && (!dy || !x || !mean || !rstd || !dx)) return OMC_ERR_NULL_PTR;
    const uintptr_t odd = reinterpret_cast<uintptr_t>(dy) | reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(dx);
    if (odd % el::size_of(type) || (reinterpret_cast<uintptr_t>(mean) | reinterpret_cast<uintptr_t>(rstd)) % 4 || !el::aligned16(gamma) ||
        !el::aligned16(dgamma) || !el::aligned16(dbeta) || !el::aligned16(workspace))
        return OMC_ERR_MISALIGNED;
#define OMC_CALL(T) \
    backward<T>(dy, ld_dy, x, ld_x, rows, cols, gamma, mean, rstd, dx, ld_dx, dgamma, dbeta, static_cast<float *>(workspace), stream)
    return type == OMC_TYPE_F32 ? OMC_CALL(float) : type == OMC_TYPE_F16 ? OMC_CALL(__half) : OMC_CALL(__nv_bfloat16);
#undef OMC_CALL
}
