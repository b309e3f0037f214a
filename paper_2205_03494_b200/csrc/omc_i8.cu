// omc_byte_quantise / omc_byte_dequantise: 8-bit integers with a scale for each row (i8_format.cuh, i8_quantise.cuh).
#include <cuda_runtime.h>

#include <type_traits>

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

// Values back, value = code * scale.  Memory bounds it: 8192 x 8192 BF16 32.2 us (6.3 TB/s), 8192 x 2048 FP32 14.4 us (5.8).  A warp has four rows, whose
// codes are on their way together, blockIdx.x is a strip of columns, blockIdx.y the rows of eight warps: CTAs that run at a time work on neighbouring
// memory.  (A grid as large as the GPU that walks over the matrix: 8192 x 2048 FP32 15.6 us; a row a warp 14.7.)
// Rows on 32-byte boundaries: a thread makes 32 bytes, 8 or 16 values, with one store.
constexpr int WARPS = 8;
constexpr uint32_t EACH = 4;         // rows of a warp, their codes on their way together
template <typename T>
__global__ void __launch_bounds__(32 * WARPS) dequantise_kernel(const int8_t *codes, const float *scales, uint32_t rows, uint32_t cols, T *__restrict__ out, uint64_t ld)
{
    constexpr int N = Word<T>::N, E = 8 * N;
    el::enter_stream_order();
    const uint64_t pitch = i8::row_bytes(cols);
    const uint32_t col = (blockIdx.x * 32 + (threadIdx.x & 31)) * E;
    if (col >= cols) return;
    using Codes = typename std::conditional<E == 16, uint4, uint2>::type;
    for (uint64_t group = (uint64_t)blockIdx.y * WARPS + (threadIdx.x >> 5); group * EACH < rows; group += (uint64_t)gridDim.y * WARPS) {
        const uint32_t first = (uint32_t)group * EACH;
        Codes q[EACH];
        float s[EACH];
#pragma unroll
        for (uint32_t i = 0; i < EACH; ++i)
            if (first + i < rows) {
                q[i] = *reinterpret_cast<const Codes *>(codes + (first + i) * pitch + col);
                s[i] = scales[first + i];
            }
#pragma unroll
        for (uint32_t i = 0; i < EACH; ++i) {
            if (first + i >= rows) break;
            uint32_t w[E / 4];
            *reinterpret_cast<Codes *>(w) = q[i];
            float v[E];
#pragma unroll
            for (int j = 0; j < E; ++j) v[j] = (float)(int8_t)(w[j / 4] >> (8 * (j & 3))) * s[i];
            T *to = out + (first + i) * ld + col;
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
}
// Other rows: neighbouring lanes make neighbouring words (of 16-bit types two values from the word's boundary on, whose halves at the row's ends
// are stored alone), four of them a thread, 32 apart.  8192 x 4095 BF16 33.4 us (3.0 TB/s): four bytes a lane, and codes whose places in a word change.
template <typename T>
__global__ void __launch_bounds__(32 * WARPS) dequantise_words_kernel(const int8_t *codes, const float *scales, uint32_t rows, uint32_t cols, T *__restrict__ out, uint64_t ld)
{
    constexpr uint32_t N = Word<T>::N;
    el::enter_stream_order();
    const uint64_t pitch = i8::row_bytes(cols);
    const uint32_t word = blockIdx.x * 128 + (threadIdx.x & 31);
    for (uint32_t row = blockIdx.y * WARPS + (threadIdx.x >> 5); row < rows; row += gridDim.y * WARPS) {
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
    constexpr uint32_t N = Word<T>::N;
    const bool whole = reinterpret_cast<uintptr_t>(out) % 32 == 0 && ld * sizeof(T) % 32 == 0;
    const uint32_t strips = whole ? (cols - 1) / (256 * N) + 1 : (cols / N) / 128 + 1, groups = (rows - 1) / (whole ? WARPS * EACH : WARPS) + 1;
    return note_cuda(el::launch(whole ? dequantise_kernel<T> : dequantise_words_kernel<T>, dim3(strips, groups < 65535 ? groups : 65535), 32 * WARPS, 0, 1, stream, codes,
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
