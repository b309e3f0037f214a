// Activations of the gated layer y = act(a) b and their derivatives, from FP32 values.
//   sigmoid  s(a) = 1 / (1 + e^-a)          s'(a) = s (1 - s)
//   SiLU     a s(a)                         s (1 + a (1 - s))
//   GELU     a P(a), P = (1 + erf(a / sqrt 2)) / 2       P + a e^(-a^2 / 2) / sqrt(2 pi)
// Exponential, reciprocal and quotient are the hardware's approximations (a few units of 2^-24 relative): far below half a step of a
// 16-bit result, about the error of an FP32 product's sum for an FP32 one.
#pragma once
#include <cuda_runtime.h>

#include "omc_internal.h"

namespace omc {
namespace gate {

__device__ __forceinline__ float sigmoid(float a) { return __fdividef(1.f, 1.f + __expf(-a)); }
__device__ __forceinline__ float normal_cdf(float a) { return __fmaf_rn(0.5f, erff(a * 0.70710678f), 0.5f); }

template <int ACT>
__device__ __forceinline__ float act(float a)
{
    if constexpr (ACT == OMC_GATE_SIGMOID) return sigmoid(a);
    else if constexpr (ACT == OMC_GATE_SILU) return a * sigmoid(a);
    else return a * normal_cdf(a);
}
// The activation and its derivative.
template <int ACT>
__device__ __forceinline__ void act_slope(float a, float &v, float &d)
{
    if constexpr (ACT == OMC_GATE_GELU) {
        const float p = normal_cdf(a);
        v = a * p;
        d = __fmaf_rn(a * 0.39894228f, __expf(-0.5f * a * a), p);
    } else {
        const float s = sigmoid(a), t = 1.f - s;
        v = ACT == OMC_GATE_SILU ? a * s : s;
        d = ACT == OMC_GATE_SILU ? s * __fmaf_rn(a, t, 1.f) : s * t;
    }
}

}  // namespace gate
}  // namespace omc
