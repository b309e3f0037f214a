// Activations of the gated layer y = act(a) b and their derivatives, from FP32 values.
//   sigmoid  s(a) = 1 / (1 + e^-a)          s'(a) = s (1 - s)
//   SiLU     a s(a)                         s (1 + a (1 - s))
//   GELU     a P(a), P = erfc(-a / sqrt 2) / 2       P + a e^(-a^2 / 2) / sqrt(2 pi)
// Exponential and reciprocal are the hardware's approximations, off by at most 2 and 1 units of 2^-23 of themselves; the exponential's argument of the first
// two is rounded to FP32, which makes it about (2 + |a|) units.  P is off by at most 8 units of itself, tails included.
#pragma once
#include <cuda_runtime.h>

#include "element.cuh"
#include "omc_internal.h"

namespace omc {
namespace gate {

// 2^x and 1 / x, results below the normal numbers as 0.
__device__ __forceinline__ float exp2_fast(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// The same, results below the normal numbers too.
__device__ __forceinline__ float exp2_wide(float x)
{
    float r;
    asm("ex2.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float reciprocal_fast(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
constexpr float LOG2_E = 1.44269504f;
__device__ __forceinline__ float sigmoid(float a) { return reciprocal_fast(1.f + exp2_fast(a * -LOG2_E)); }

__device__ __forceinline__ float2 neg2(float2 v) { return make_float2(-v.x, -v.y); }
// |v|, `most` at most; NaN stays NaN.
__device__ __forceinline__ float magnitude(float v, float most)
{
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(v)), "f"(most));
    return r;
}
// e^-(c x + y) = 2^-p e^-w, p = c log2(e) x rounded, w = what the rounding and the constant left, and y: |w| << 1.  c is 1 or 1/2; y may be 0.
template <int HALVES>
__device__ __forceinline__ float2 exp_neg2(float2 x, float2 y)
{
    constexpr float C = 0.5f * HALVES * 1.44269502f, C_REST = 0.5f * HALVES * 1.3349758e-8f;       // log2 e = 1.44269502.. + 1.92596e-8, the rest times ln 2
    const float2 p = el::mul2(x, el::twice(-C)), rest = el::fma2(x, el::twice(C), p);              // the product less its rounding, exact
    const float2 w = el::fma2(rest, el::twice(0.693147182f), el::fma2(x, el::twice(C_REST), y));
    const float2 e = make_float2(exp2_wide(p.x), exp2_wide(p.y));
    return el::fma2(e, neg2(w), e);
}
// e^(-a^2 / 2) and P(a).  The lower tail P(-|a|) = e^(-a^2 / 2) Q(|a|), Q(x) = e^(x^2 / 2) erfc(x / sqrt 2) / 2, as a polynomial in t = 1 / (1 + 0.36 x) whose
// relative error, 0.6 units of 2^-23, was made as small as possible over 0 <= x <= 16 by Remez's exchange; Horner's roundings make it 4.4.  The square's rounding
// goes into the exponential.  (Backward to codes at 8192 x 8192 BF16 287 us, with CUDA's erfcf 458; forward 8192 x 8192 x 2048 BF16 225 and 308.)
__device__ __forceinline__ void normal2(float2 a, float2 &e, float2 &P)
{
    const float2 x = make_float2(magnitude(a.x, 16.f), magnitude(a.y, 16.f)), square = el::mul2(x, x), rest = el::fma2(x, x, neg2(square));
    e = exp_neg2<1>(square, el::mul2(rest, el::twice(0.5f)));
    const float2 d = el::fma2(x, el::twice(0.36f), el::twice(1.f)), t = make_float2(reciprocal_fast(d.x), reciprocal_fast(d.y));
    constexpr float Q[9] = {0.143619731f, 0.143644631f, 0.124278106f, 0.0950212404f, 0.00183042313f, 0.104518518f, -0.221503928f, 0.138718486f, -0.0301272385f};
    float2 q = el::twice(Q[8]);
#pragma unroll
    for (int i = 7; i >= 0; --i) q = el::fma2(q, t, el::twice(Q[i]));
    const float2 h = el::mul2(el::mul2(q, t), e), up = el::fma2(h, el::twice(-1.f), el::twice(1.f));
    P = make_float2(a.x < 0.f ? h.x : up.x, a.y < 0.f ? h.y : up.y);
}

// The activation of two values.
template <int ACT>
__device__ __forceinline__ float2 act2(float2 a)
{
    if constexpr (ACT == OMC_GATE_GELU) {
        float2 e, P;
        normal2(a, e, P);
        return el::mul2(a, P);
    } else {
        const float2 s = make_float2(sigmoid(a.x), sigmoid(a.y));
        return ACT == OMC_GATE_SILU ? el::mul2(a, s) : s;
    }
}
// The activation and its derivative, of two values.
template <int ACT>
__device__ __forceinline__ void act_slope2(float2 a, float2 &v, float2 &d)
{
    if constexpr (ACT == OMC_GATE_GELU) {
        float2 e, P;
        normal2(a, e, P);
        v = el::mul2(a, P);
        d = el::fma2(el::mul2(a, el::twice(0.39894228f)), e, P);
    } else {
        const float2 e = el::mul2(a, el::twice(-LOG2_E));
        const float2 o = el::add2(make_float2(exp2_fast(e.x), exp2_fast(e.y)), el::twice(1.f));
        const float2 s = make_float2(reciprocal_fast(o.x), reciprocal_fast(o.y)), t = el::fma2(s, el::twice(-1.f), el::twice(1.f));
        v = ACT == OMC_GATE_SILU ? el::mul2(a, s) : s;
        d = ACT == OMC_GATE_SILU ? el::mul2(s, el::fma2(a, t, el::twice(1.f))) : el::mul2(s, t);
    }
}

}  // namespace gate
}  // namespace omc
