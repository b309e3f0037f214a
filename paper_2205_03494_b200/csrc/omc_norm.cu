// omc_layer_norm / omc_layer_norm_backward: normalisation over the last dimension, its gradient, and the
// gradients of its gain and bias.
//
//     y = xhat gamma + beta,  xhat = (x - mean) rstd,  rstd = (var + eps)^(-1/2), var the mean squared deviation
//     dx = rstd (g - mean(g) - xhat mean(g xhat)),  g = dy gamma;   dgamma = sum_rows dy xhat,  dbeta = sum_rows dy
#include <cuda_runtime.h>

#include "element.cuh"
#include "omc_internal.h"

namespace omc {
int note_cuda(cudaError_t e);
}

namespace {

using namespace omc;

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

// Any width: a CTA per row, three passes over it.  (y may be x, dx may be dy or x: no __restrict__ on them.)
template <typename T>
__global__ void __launch_bounds__(THREADS)
norm_wide_kernel(const T *x, uint32_t cols, uint64_t ld, const float *__restrict__ gamma, const float *__restrict__ beta,
                 float eps, T *y, uint64_t ldy, float *__restrict__ mean_out, float *__restrict__ rstd_out)
{
    el::enter_stream_order();
    __shared__ float room[THREADS / 32];
    const uint64_t row = blockIdx.x;
    const T *xr = x + row * ld;
    T *yr = y + row * ldy;
    float s = 0.f;
    for (uint32_t c = threadIdx.x; c < cols; c += THREADS) s += el::to_float(xr[c]);
    const float mean = cta_sum(s, room) / (float)cols;
    s = 0.f;
    for (uint32_t c = threadIdx.x; c < cols; c += THREADS) {
        const float d = el::to_float(xr[c]) - mean;
        s = __fmaf_rn(d, d, s);
    }
    const float rstd = 1.f / sqrtf(cta_sum(s, room) / (float)cols + eps);
    for (uint32_t c = threadIdx.x; c < cols; c += THREADS)
        yr[c] = el::from_float<T>(__fmaf_rn((el::to_float(xr[c]) - mean) * rstd, gamma[c], beta[c]));
    if (threadIdx.x == 0) {
        if (mean_out) mean_out[row] = mean;
        if (rstd_out) rstd_out[row] = rstd;
    }
}

template <typename T>
__global__ void __launch_bounds__(THREADS)
norm_backward_wide_kernel(const T *dy, uint64_t ld_dy, const T *x, uint64_t ld_x, uint32_t cols,
                          const float *__restrict__ gamma, const float *__restrict__ mean_in, const float *__restrict__ rstd_in,
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
norm_columns_kernel(const T *__restrict__ dy, uint64_t ld_dy, const T *__restrict__ x, uint64_t ld_x, uint32_t rows, uint32_t cols,
                    const float *__restrict__ mean_in, const float *__restrict__ rstd_in, float *__restrict__ part)
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

__global__ void __launch_bounds__(THREADS)
norm_finish_kernel(const float *__restrict__ part, uint32_t parts, uint32_t cols, float *__restrict__ dgamma, float *__restrict__ dbeta)
{
    el::enter_stream_order();
    const uint32_t c = blockIdx.x * THREADS + threadIdx.x;
    if (c >= 2 * cols) return;
    float s = 0.f;
    for (uint32_t p = 0; p < parts; ++p) s += part[(uint64_t)p * 2 * cols + c];
    if (c < cols) dgamma[c] = s;
    else dbeta[c - cols] = s;
}

// Partial column sums: one per SM of the device the kernels are laid out for.
uint32_t parts_of(uint64_t rows) { return (uint32_t)(rows < DEFAULT_SMS ? rows : DEFAULT_SMS); }

bool shape_ok(uint64_t rows, uint64_t cols) { return cols >= 1 && rows < (1ull << 31) && cols < (1ull << 30); }

template <typename T>
int forward(const void *x, uint64_t rows, uint64_t cols, uint64_t ld, const float *gamma, const float *beta, float eps, void *y,
            uint64_t ldy, float *mean, float *rstd, void *stream)
{
    return note_cuda(el::launch(norm_wide_kernel<T>, dim3((uint32_t)rows), THREADS, 0, 1, stream, static_cast<const T *>(x), (uint32_t)cols,
                                ld, gamma, beta, eps, static_cast<T *>(y), ldy, mean, rstd));
}

template <typename T>
int backward(const void *dy, uint64_t ld_dy, const void *x, uint64_t ld_x, uint64_t rows, uint64_t cols, const float *gamma,
             const float *mean, const float *rstd, void *dx, uint64_t ld_dx, float *dgamma, float *dbeta, float *part, void *stream)
{
    const uint32_t c = (uint32_t)cols, parts = parts_of(rows);
    int rc = 0;
    if (rows) {
        // the column sums first: dx may overwrite dy or x
        rc = note_cuda(el::launch(norm_columns_kernel<T>, dim3((c + THREADS - 1) / THREADS, parts), THREADS, 0, 1, stream,
                                  static_cast<const T *>(dy), ld_dy, static_cast<const T *>(x), ld_x, (uint32_t)rows, c, mean, rstd, part));
        if (!rc)
            rc = note_cuda(el::launch(norm_backward_wide_kernel<T>, dim3((uint32_t)rows), THREADS, 0, 1, stream, static_cast<const T *>(dy),
                                      ld_dy, static_cast<const T *>(x), ld_x, c, gamma, mean, rstd, static_cast<T *>(dx), ld_dx));
    }
    if (!rc)
        rc = note_cuda(el::launch(norm_finish_kernel, dim3((2 * c + THREADS - 1) / THREADS), THREADS, 0, 1, stream,
                                  static_cast<const float *>(part), parts, c, dgamma, dbeta));
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
