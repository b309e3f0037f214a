// The 4-bit microscaled format: E2M1 codes in blocks of 32 under one E8M0 scale, and where they are stored.
#pragma once
#include <cuda_fp16.h>
#include <stdint.h>

namespace omc {
namespace mx {

constexpr uint32_t BLOCK = 32;           // values per scale
constexpr uint32_t NAN_SCALE = 255;      // E8M0 NaN: every value of the block is NaN

__host__ __device__ constexpr uint64_t row_bytes(uint64_t cols) { return (cols + 31) / 32 * 16; }
__host__ __device__ constexpr uint64_t codes_bytes(uint64_t rows, uint64_t cols) { return rows * row_bytes(cols); }
// The scales are stored as the tensor cores take them: 512 bytes hold 128 rows x 4 blocks (row r at
// 16 (r mod 32) + 4 (r / 32)), two of those cover 256 columns, one K step of the product.
__host__ __device__ constexpr uint64_t scales_bytes(uint64_t rows, uint64_t cols)
{
    return (rows + 127) / 128 * ((cols + 255) / 256) * 1024;
}
__host__ __device__ __forceinline__ uint64_t scale_offset(uint64_t r, uint64_t block, uint64_t ksteps)
{
    return ((r >> 7) * ksteps + (block >> 3)) * 1024 + ((block >> 2) & 1) * 512 + (r & 31) * 16 + ((r >> 5) & 3) * 4 + (block & 3);
}

// E8M0 byte of a block whose largest magnitude has this bit pattern: floor(log2) - 2 (the exponent of
// 4, the top binade of E2M1), never below 2^-127; an Inf or NaN in the block makes it NaN.
__device__ __forceinline__ uint32_t scale_of(uint32_t amax_bits)
{
    const uint32_t e = amax_bits >> 23;
    return e == 255u ? NAN_SCALE : max(e, 2u) - 2u;
}
// 2^(127 - scale): an exact factor (a normal number for scale <= 253); 0 for the NaN scale, whose codes are 0.
__device__ __forceinline__ float inverse_scale(uint32_t scale) { return scale == NAN_SCALE ? 0.f : __uint_as_float((254u - scale) << 23); }
// 2^(scale - 127), subnormal for scale = 0.
__device__ __forceinline__ float scale_value(uint32_t scale)
{
    return scale == NAN_SCALE ? __uint_as_float(0x7FC00000u) : scale == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(scale << 23);
}
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Eight values (already scaled) as eight codes: round to nearest even, saturate at +-6.
__device__ __forceinline__ uint32_t encode8(const float *v)
{
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
// Eight codes as FP32 values (every E2M1 value is an FP16 value).
__device__ __forceinline__ void decode8(uint32_t codes, float *v)
{
    uint32_t h[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h[i]));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

}  // namespace mx
}  // namespace omc
