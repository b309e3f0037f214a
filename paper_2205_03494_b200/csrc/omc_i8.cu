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

// Values back.  Rows on 32-byte boundaries: a thread makes 32 bytes, 8 or 16 values, with one store.
template <typename T>
__global__ void __launch_bounds__(256) dequantise_kernel(const int8_t *codes, const float *scales, uint32_t rows, uint32_t cols, T *__restrict__ out, uint64_t ld)
{
    constexpr int N = Word<T>::N, E = 8 * N;
    el::enter_stream_order();
    const uint32_t chunks = (cols + E - 1) / E;
    const uint64_t all = (uint64_t)rows * chunks, step = (uint64_t)gridDim.x * 256, pitch = i8::row_bytes(cols);
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += step) {
        const uint32_t row = (uint32_t)(i / chunks), col = (uint32_t)(i - (uint64_t)row * chunks) * E;
        const int8_t *from = codes + row * pitch + col;
        uint32_t w[E / 4];
        if constexpr (E == 16) {
            const uint4 q = *reinterpret_cast<const uint4 *>(from);
            w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
        } else {
            const uint2 q = *reinterpret_cast<const uint2 *>(from);
            w[0] = q.x, w[1] = q.y;
        }
        const float s = scales[row];
        float v[E];
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = (float)(int8_t)(w[j / 4] >> (8 * (j & 3))) * s;
        T *to = out + row * ld + col;
        if (col + E <= cols) {
            uint32_t o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = Word<T>::pack(v + j * N);
            el::store32(to, o);
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (col + j < cols) to[j] = el::from_float<T>(v[j]);
        }
    }
}
// Other rows: neighbouring lanes make neighbouring words (of 16-bit types two values from the word's boundary on, whose halves at the row's ends
// are stored alone), four of them a thread, 32 apart; a warp a piece of 128 words of a row.
template <typename T>
__global__ void __launch_bounds__(256) dequantise_words_kernel(const int8_t *codes, const float *scales, uint32_t rows, uint32_t cols, T *__restrict__ out, uint64_t ld)
{
    constexpr uint32_t N = Word<T>::N;
    el::enter_stream_order();
    const uint32_t lane = threadIdx.x & 31, pieces = (cols / N + 1 + 127) / 128;
    const uint64_t all = (uint64_t)rows * pieces, step = (uint64_t)gridDim.x * 8, pitch = i8::row_bytes(cols);
    for (uint64_t i = (uint64_t)blockIdx.x * 8 + (threadIdx.x >> 5); i < all; i += step) {
        const uint32_t row = (uint32_t)(i / pieces), word = (uint32_t)(i - (uint64_t)row * pieces) * 128 + lane;
        T *const to = out + row * ld;
        const uint32_t odd = N == 2 ? (uint32_t)(reinterpret_cast<uintptr_t>(to) >> 1) & 1u : 0u;
        const int8_t *const from = codes + row * pitch;
        const float s = scales[row];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t place = (word + 32 * j) * N;        // value place - odd is the word's first one
            float v[2] = {0.f, 0.f};
            const bool before = N == 2 && odd > place, first = !before && place - odd < cols, second = N == 2 && place + 1 - odd < cols;
            if (first) v[0] = (float)from[place - odd] * s;
            if (second) v[1] = (float)from[place + 1 - odd] * s;
            T *const p = to + place - odd;
            if (N == 1 ? first : first && second) *reinterpret_cast<uint32_t *>(p) = Word<T>::pack(v);
            else if (first) p[0] = el::from_float<T>(v[0]);
            else if (second) p[1] = el::from_float<T>(v[1]);
        }
    }
}

template <typename T>
int dequantise(const int8_t *codes, const float *scales, uint32_t rows, uint32_t cols, void *out, uint64_t ld, void *stream)
{
    constexpr uint64_t N = Word<T>::N;
    const bool whole = reinterpret_cast<uintptr_t>(out) % 32 == 0 && ld * sizeof(T) % 32 == 0;
    const uint64_t threads = whole ? (uint64_t)rows * ((cols + 8 * N - 1) / (8 * N)) : (uint64_t)rows * ((cols / N + 1 + 127) / 128) * 32;
    const uint64_t ctas = (threads + 255) / 256, most = DEFAULT_SMS * 8;
    return note_cuda(el::launch(whole ? dequantise_kernel<T> : dequantise_words_kernel<T>, dim3((uint32_t)(ctas < most ? ctas : most)), 256, 0, 1, stream, codes,
                                scales, rows, cols, static_cast<T *>(out), ld));
}

template <typename T, bool WHOLE>
int quantise(const void *x, uint64_t ld, uint32_t rows, uint32_t cols, int8_t *codes, float *scales, int8_t *codes_t, float *scales_t, void *workspace,
             void *stream)
{
    const T *const m = static_cast<const T *>(x);
    const i8::Matrix<T, WHOLE> src = {m, ld, rows};
    return i8::quantise<4>(src, rows, cols, codes, scales, codes_t, scales_t, workspace, stream);
}

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
    *bytes = i8::maxima_bytes(rows, cols, 1);
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
    const bool whole = el::aligned16(x) && ld * el::size_of(type) % 16 == 0 && cols * el::size_of(type) % 16 == 0;
    const uint32_t r = (uint32_t)rows, c = (uint32_t)cols;
#define OMC_CALL(T) (whole ? quantise<T, true>(x, ld, r, c, codes, scales, codes_t, scales_t, workspace, stream) \
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
    const uint32_t r = (uint32_t)rows, c = (uint32_t)cols;
    return type == OMC_TYPE_F32 ? dequantise<float>(codes, scales, r, c, out, ld, stream)
           : type == OMC_TYPE_F16 ? dequantise<__half>(codes, scales, r, c, out, ld, stream) : dequantise<__nv_bfloat16>(codes, scales, r, c, out, ld, stream);
}
