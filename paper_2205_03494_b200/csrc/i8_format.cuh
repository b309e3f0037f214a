// The 8-bit integer format: rows of codes under one FP32 scale each, and what a sum of products of codes stands for.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace omc {
namespace i8 {

__host__ __device__ constexpr uint64_t row_bytes(uint64_t cols) { return (cols + 15) / 16 * 16; }

// Sums of products of codes are 32-bit integers: 2^17 - 1 products of -128 by -128 still fit.
constexpr uint64_t MOST_K = (1u << 17) - 1;

// Scale of a row whose largest magnitude has this FP32 bit pattern, and the factor that its values are multiplied by.  The floor
// keeps both normal numbers; a row with an Inf or a NaN has the scale NaN (and codes 0, which its values are masked to).
struct Scale {
    float s, r;
    __device__ __forceinline__ bool nan() const { return !(s == s); }
};
__device__ __forceinline__ Scale scale_of(uint32_t amax_bits)
{
    Scale v;
    v.s = fmaxf(__fdiv_rn(__uint_as_float(amax_bits), 127.f), 0x1p-126f);
    v.r = __frcp_rn(v.s);
    if (amax_bits >= 0x7F800000u) {
        v.s = __uint_as_float(0x7FC00000u);
        v.r = 0.f;
    }
    return v;
}

// x r + 1.5 2^23 has a last place of 1: the one rounding of the fused multiply-add makes the product, |x r| <= 127 (1 + 2^-22), the
// integer next to it, ties to even, and leaves it as the low bits of the sum.
constexpr float TO_INTEGER = 12582912.f;

// The low bytes of four such sums.
__device__ __forceinline__ uint32_t bytes4(float a, float b, float c, float d)
{
    const uint32_t lo = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040), hi = __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040);
    return __byte_perm(lo, hi, 0x5410);
}

// What a sum of products stands for: (sum sx) sw, three roundings whoever computes it.  The first product could leave the
// range for a scale of X above 2^97 although the second one brings it back, so such a scale is taken in two steps: f = sx 2^-64 first
// and 2^64 last (no rounding: f >= 1, and scales are at least 2^-126).  Rows without it take the short way, which gives the same bits.
struct RowScale {
    float f, g;
    __device__ __forceinline__ RowScale() : f(0.f), g(1.f) {}
    __device__ __forceinline__ explicit RowScale(float s) : f(s >= 0x1p64f ? s * 0x1p-64f : s), g(s >= 0x1p64f ? 0x1p64f : 1.f) {}
    __device__ __forceinline__ bool big() const { return g != 1.f; }
};
__device__ __forceinline__ float value(int32_t sum, const RowScale &x, float w) { return __int2float_rn(sum) * x.f * w; }
__device__ __forceinline__ float value_in_two(int32_t sum, const RowScale &x, float w) { return __int2float_rn(sum) * x.f * w * x.g; }

}  // namespace i8
}  // namespace omc
