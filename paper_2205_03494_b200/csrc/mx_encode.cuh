// Values of an element type on their way into the 4-bit microscaled format: loads and the encoding of a block.
#pragma once
#include "element.cuh"
#include "mx_format.cuh"

namespace omc {
namespace mx {

using el::Word;

// E consecutive values as they are stored, two to a word of 16-bit types.
template <typename T, bool VECTOR, int E>
__device__ __forceinline__ void load(const T *row, uint32_t col, uint32_t cols, uint32_t *w)
{
    constexpr int N = Word<T>::N, WORDS = E / N;
    if (VECTOR && col + E <= cols && WORDS == 8 && (reinterpret_cast<uintptr_t>(row + col) & 31u) == 0) {
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                     : "l"(row + col) : "memory");
    } else if (VECTOR && col + E <= cols) {
#pragma unroll
        for (int i = 0; i < WORDS; i += 4) {
            const uint4 q = *reinterpret_cast<const uint4 *>(row + col + i * N);
            w[i] = q.x;
            w[i + 1] = q.y;
            w[i + 2] = q.z;
            w[i + 3] = q.w;
        }
    } else {                       // zeros behind the row's end
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            if constexpr (sizeof(T) == 4) {
                w[i] = col + i < cols ? reinterpret_cast<const uint32_t *>(row)[col + i] : 0u;
            } else {
                const uint16_t *p = reinterpret_cast<const uint16_t *>(row) + col + 2 * i;
                const uint32_t lo = col + 2 * i < cols ? p[0] : 0u, hi = col + 2 * i + 1 < cols ? p[1] : 0u;
                w[i] = lo | (hi << 16);
            }
        }
    }
}

// Largest magnitude, two 16-bit values at a time: the order of the magnitudes is that of their bit patterns, Inf and
// NaN on top.
template <typename T>
__device__ __forceinline__ uint32_t max_magnitude(uint32_t acc, uint32_t w)
{
    if constexpr (sizeof(T) == 4) return max(acc, w & 0x7FFFFFFFu);
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(acc), "r"(w & 0x7FFF7FFFu));
    return r;
}
// A magnitude of T as FP32 bits (T 16 bits wide: the lower half of m).
template <typename T>
__device__ __forceinline__ uint32_t fp32_bits(uint32_t m)
{
    if constexpr (sizeof(T) == 4) return m;
    float f[2];
    Word<T>::unpack(m, f);
    return __float_as_uint(f[0]);
}

// Codes and scale of the block that 32 / E neighbouring lanes hold, E values each.
template <typename T, int E>
__device__ __forceinline__ void encode_block(const uint32_t *w, uint32_t *codes, uint32_t &scale)
{
    constexpr int N = Word<T>::N, WORDS = E / N;
    uint32_t top = w[0] & (sizeof(T) == 4 ? 0x7FFFFFFFu : 0x7FFF7FFFu);
#pragma unroll
    for (int i = 1; i < WORDS; ++i) top = max_magnitude<T>(top, w[i]);
    if constexpr (sizeof(T) == 2) top = max(top >> 16, top & 0xFFFFu);
#pragma unroll
    for (int d = 1; d < 32 / E; d *= 2) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    scale = scale_of(fp32_bits<T>(top));
    const float2 f = el::twice(inverse_scale(scale));
#pragma unroll
    for (int c = 0; c < E / 8; ++c) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8 / N; ++i) Word<T>::unpack(w[c * (8 / N) + i], v + N * i);
#pragma unroll
        for (int i = 0; i < 4; ++i) reinterpret_cast<float2 *>(v)[i] = el::mul2(reinterpret_cast<float2 *>(v)[i], f);
        codes[c] = scale == NAN_SCALE ? 0u : encode8(v);
    }
}
}  // namespace mx
}  // namespace omc
