// Activations of the gated layer y = act(a) b and their derivatives, from FP32 values.
//   sigmoid  s(a) = 1 / (1 + e^-a)          s'(a) = s (1 - s)
//   SiLU     a s(a)                         s (1 + a (1 - s))
//   GELU     a P(a), P = (1 + erf(a / sqrt 2)) / 2       P + a e^(-a^2 / 2) / sqrt(2 pi)
// Exponential, reciprocal and quotient are the hardware's approximations (a few units of 2^-24 relative): far below half a step of a
// 16-bit result, about the error of an FP32 product's sum for an FP32 one.
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
__device__ __forceinline__ float reciprocal_fast(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
constexpr float LOG2_E = 1.44269504f;
__device__ __forceinline__ float sigmoid(float a) { return reciprocal_fast(1.f + exp2_fast(a * -LOG2_E)); }
__device__ __forceinline__ float normal_cdf(float a) { return __fmaf_rn(0.5f, erff(a * 0.70710678f), 0.5f); }

template <int ACT>
__device__ __forceinline__ float act(float a)
{
    if constexpr (ACT == OMC_GATE_SIGMOID) return sigmoid(a);
    else if constexpr (ACT == OMC_GATE_SILU) return a * sigmoid(a);
    else return a * normal_cdf(a);
}
// The activation and its derivative, of two values.
template <int ACT>
__device__ __forceinline__ void act_slope2(float2 a, float2 &v, float2 &d)
{
    if constexpr (ACT == OMC_GATE_GELU) {
        const float2 p = make_float2(normal_cdf(a.x), normal_cdf(a.y)), q = el::mul2(el::mul2(a, a), el::twice(-0.5f * LOG2_E));
        v = el::mul2(a, p);
        d = el::fma2(el::mul2(a, el::twice(0.39894228f)), make_float2(exp2_fast(q.x), exp2_fast(q.y)), p);
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
