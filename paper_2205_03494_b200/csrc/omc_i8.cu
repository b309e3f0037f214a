// omc_byte_quantise / omc_byte_dequantise: 8-bit integers with a scale for each row (i8_format.cuh, i8_quantise.cuh).
#include <cuda_runtime.h>

#include "element.cuh"
#include "i8_format.cuh"
#include "i8_quantise.cuh"
#include "omc_internal.h"

namespace omc {
bool i8_shape_ok(uint64_t rows, uint64_t cols)
{
    return rows >= 1 && cols >= 1 && rows < (1ull << 31) && cols < (1ull << 31);
}
}  // namespace omc

namespace {

using namespace omc;
using el::Word;

// Values back: a thread takes sixteen codes.
template <typename T, bool VECTOR>
__global__ void __launch_bounds__(256) dequantise_kernel(const int8_t *codes, const float *scales, uint32_t rows, uint32_t cols, T *__restrict__ out, uint64_t ld)
{
    constexpr int N = Word<T>::N;
    el::enter_stream_order();
    const uint32_t chunks = (cols + 15) / 16;
    const uint64_t all = (uint64_t)rows * chunks, step = (uint64_t)gridDim.x * 256;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += step) {
        const uint32_t row = (uint32_t)(i / chunks), col = (uint32_t)(i - (uint64_t)row * chunks) * 16;
        const uint4 q = *reinterpret_cast<const uint4 *>(codes + i * 16);
        const float s = scales[row];
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
        float v[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = (float)(int8_t)(w[j / 4] >> (8 * (j & 3))) * s;
        T *to = out + row * ld + col;
        if (VECTOR && col + 16 <= cols) {
#pragma unroll
            for (int j = 0; j < 16 / N; j += 4)
                *reinterpret_cast<uint4 *>(to + j * N) = make_uint4(Word<T>::pack(v + j * N), Word<T>::pack(v + (j + 1) * N), Word<T>::pack(v + (j + 2) * N), Word<T>::pack(v + (j + 3) * N));
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (col + j < cols) to[j] = el::from_float<T>(v[j]);
        }
    }
}

template <typename T, bool VECTOR>
int dequantise(const int8_t *codes, const float *scales, uint32_t rows, uint32_t cols, void *out, uint64_t ld, void *stream)
{
    const uint64_t ctas = ((uint64_t)rows * ((cols + 15) / 16) + 255) / 256, most = DEFAULT_SMS * 8;
    return note_cuda(el::launch(dequantise_kernel<T, VECTOR>, dim3((uint32_t)(ctas < most ? ctas : most)), 256, 0, 1, stream, codes, scales, rows, cols,
                                static_cast<T *>(out), ld));
}

template <typename T, bool VECTOR>
int quantise(const void *x, uint64_t ld, uint32_t rows, uint32_t cols, int8_t *codes, float *scales, int8_t *codes_t, float *scales_t, void *workspace,
             void *stream)
{
    const i8::Matrix<T, VECTOR> src = {static_cast<const T *>(x), ld};
    return i8::quantise<4>(src, rows, cols, codes, scales, codes_t, scales_t, workspace, stream);
}

bool vector_rows(const void *p, uint64_t ld, int type) { return el::aligned16(p) && ld * el::size_of(type) % 16 == 0; }
bool aligned4(const void *p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

}  // namespace

extern "C" int omc_byte_sizes(uint64_t rows, uint64_t cols, uint64_t *codes_bytes, uint64_t *scales_bytes)
{
    if (!i8_shape_ok(rows, cols)) return OMC_ERR_INVALID_ARG;
    if (codes_bytes) *codes_bytes = rows * i8::row_bytes(cols);
    if (scales_bytes) *scales_bytes = (rows * 4 + 15) / 16 * 16;
    return OMC_OK;
}

extern "C" int omc_byte_quantise_workspace(uint64_t rows, uint64_t cols, uint64_t *bytes)
{
    if (!bytes) return OMC_ERR_NULL_PTR;
    if (!i8_shape_ok(rows, cols)) return OMC_ERR_INVALID_ARG;
    *bytes = i8::parts_bytes(rows, cols);
    return OMC_OK;
}

extern "C" int omc_byte_quantise(const void *x, int type, uint64_t rows, uint64_t cols, uint64_t ld, int8_t *codes, float *scales, int8_t *codes_t,
                               float *scales_t, void *workspace, void *stream)
{
    if (!el::type_ok(type)) return OMC_ERR_INVALID_ARG;
    if (!x || (!codes && !codes_t) || !codes != !scales || !codes_t != !scales_t || (codes_t && !workspace)) return OMC_ERR_NULL_PTR;
    if (!i8_shape_ok(rows, cols) || ld < cols) return OMC_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(x) % el::size_of(type) || !el::aligned16(codes) || !aligned4(scales) || !el::aligned16(codes_t) ||
        !aligned4(scales_t) || !el::aligned16(workspace))
        return OMC_ERR_MISALIGNED;
    const bool vec = vector_rows(x, ld, type);
    const uint32_t r = (uint32_t)rows, c = (uint32_t)cols;
#define OMC_CALL(T) (vec ? quantise<T, true>(x, ld, r, c, codes, scales, codes_t, scales_t, workspace, stream) \
                         : quantise<T, false>(x, ld, r, c, codes, scales, codes_t, scales_t, workspace, stream))
    return type == OMC_TYPE_F32 ? OMC_CALL(float) : type == OMC_TYPE_F16 ? OMC_CALL(__half) : OMC_CALL(__nv_bfloat16);
#undef OMC_CALL
}

extern "C" int omc_byte_dequantise(const int8_t *codes, const float *scales, uint64_t rows, uint64_t cols, void *out, int type, uint64_t ld, void *stream)
{
    if (!el::type_ok(type)) return OMC_ERR_INVALID_ARG;
    if (!codes || !scales || !out) return OMC_ERR_NULL_PTR;
    if (!i8_shape_ok(rows, cols) || ld < cols) return OMC_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(out) % el::size_of(type) || !el::aligned16(codes) || !aligned4(scales)) return OMC_ERR_MISALIGNED;
    const bool vec = vector_rows(out, ld, type);
    const uint32_t r = (uint32_t)rows, c = (uint32_t)cols;
#define OMC_CALL(T) (vec ? dequantise<T, true>(codes, scales, r, c, out, ld, stream) : dequantise<T, false>(codes, scales, r, c, out, ld, stream))
    return type == OMC_TYPE_F32 ? OMC_CALL(float) : type == OMC_TYPE_F16 ? OMC_CALL(__half) : OMC_CALL(__nv_bfloat16);
#undef OMC_CALL
}
