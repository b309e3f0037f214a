// Activations of the gated layer y = act(a) b and their derivatives, from FP32 values.
//   sigmoid  s(a) = 1 / (1 + e^-a)          s'(a) = s (1 - s)
//   SiLU     a s(a)                         s (1 + a (1 - s))
//   GELU     a P(a), P = erfc(-a / sqrt 2) / 2       P + a e^(-a^2 / 2) / sqrt(2 pi)
// Exponential and reciprocal are the hardware's approximations, off by at most 2 and 1 units of 2^-23 of themselves.  With what is made of them s, 1 - s and P are off
// by at most 7, 7 and 11 units of themselves, however small they are.  Where the result has 16 bits (FINE = false) the rounding of the exponent is left in, 0.7 |a| units more of the
// first two and 0.6 a^2 of P, far below half a step of the result (2^12 units of FP16), and an s or 1 - s below 2^-126 is 0.
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

constexpr float LOG2_E = 1.44269502f;        // less 1.92596e-8
__device__ __forceinline__ float2 neg2(float2 v) { return make_float2(-v.x, -v.y); }
// |v|, `most` at most; NaN stays NaN.
__device__ __forceinline__ float magnitude(float v, float most)
{
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(v)), "f"(most));
    return r;
}
// e^-(c x + y) as (2^-p)^2, p = c log2(e) x / 2 rounded; c is 1 or 1/2.  FINE: times e^w, w = what p's rounding, its constant and y left out, |w| << 1.  (A root, squared:
// results below the normal numbers are right too, in fewer instructions than by an exponential that makes such.)
template <int HALVES, bool FINE>
__device__ __forceinline__ float2 exp_neg2(float2 x, float2 y)
{
    constexpr float C = 0.25f * HALVES * LOG2_E, C_REST = 0.5f * HALVES * 1.3349758e-8f;       // (the rest times ln 2)
    const float2 p = el::mul2(x, el::twice(-C)), root = make_float2(exp2_fast(p.x), exp2_fast(p.y)), e = el::mul2(root, root);
    if constexpr (!FINE) return e;
    const float2 rest = el::fma2(x, el::twice(C), p);               // the product less its rounding, exact
    return el::fma2(e, el::fma2(rest, el::twice(-2 * 0.693147182f), el::fma2(x, el::twice(-C_REST), neg2(y))), e);
}
// s(a) and t = 1 - s(a) = e^-a s(a), which is a difference only where it is more than a half.  FINE: from e^-|a|, which does not overflow; else s and t below the
// normal numbers are 0.
template <bool FINE>
__device__ __forceinline__ void sigmoid2(float2 a, float2 &s, float2 &t)
{
    if constexpr (FINE) {
        const float2 e = exp_neg2<2, FINE>(make_float2(magnitude(a.x, 128.f), magnitude(a.y, 128.f)), el::twice(0.f)), o = el::add2(e, el::twice(1.f));
        const float2 r = make_float2(reciprocal_fast(o.x), reciprocal_fast(o.y)), q = el::mul2(e, r);
        s = make_float2(a.x < 0.f ? q.x : r.x, a.y < 0.f ? q.y : r.y);
        t = make_float2(a.x < 0.f ? r.x : q.x, a.y < 0.f ? r.y : q.y);
    } else {
        const float2 p = el::mul2(a, el::twice(-LOG2_E)), e = make_float2(exp2_fast(p.x), exp2_fast(p.y)), o = el::add2(e, el::twice(1.f));
        s = make_float2(reciprocal_fast(o.x), reciprocal_fast(o.y));
        const float2 low = el::mul2(e, s), high = el::fma2(s, el::twice(-1.f), el::twice(1.f));
        t = make_float2(a.x < 0.f ? high.x : low.x, a.y < 0.f ? high.y : low.y);
    }
}
// e^(-a^2 / 2) and P(a).  The lower tail P(-|a|) = e^(-a^2 / 2) Q(|a|), Q(x) = e^(x^2 / 2) erfc(x / sqrt 2) / 2, as a polynomial in t = 1 / (1 + 0.36 x) whose
// relative error, 0.6 units of 2^-23, was made as small as possible over 0 <= x <= 16 by Remez's exchange; Horner's roundings make it 4.4.  The square's rounding
// goes into the exponential.  (Backward to codes at 8192 x 8192 BF16 253 us, with CUDA's erfcf 458; forward 8192 x 8192 x 2048 BF16 239 and 308.)
template <bool FINE>
__device__ __forceinline__ void normal2(float2 a, float2 &e, float2 &P)
{
    const float2 x = make_float2(magnitude(a.x, 16.f), magnitude(a.y, 16.f)), square = el::mul2(x, x), rest = el::fma2(x, x, neg2(square));
    e = exp_neg2<1, FINE>(square, el::mul2(rest, el::twice(0.5f)));
    const float2 d = el::fma2(x, el::twice(0.36f), el::twice(1.f));
    float2 t = make_float2(reciprocal_fast(d.x), reciprocal_fast(d.y));
    if constexpr (FINE) {            // a step of Newton's method, with what d's rounding left out
        const float2 left = el::fma2(x, el::twice(0.36f), el::fma2(d, el::twice(-1.f), el::twice(1.f))), m = el::mul2(t, el::twice(-1.f));
        t = el::fma2(t, el::fma2(left, m, el::fma2(d, m, el::twice(1.f))), t);
    }
    constexpr float Q[9] = {0.143619731f, 0.143644631f, 0.124278106f, 0.0950212404f, 0.00183042313f, 0.104518518f, -0.221503928f, 0.138718486f, -0.0301272385f};
    float2 q = el::twice(Q[8]);
#pragma unroll
    for (int i = 7; i >= 0; --i) q = el::fma2(q, t, el::twice(Q[i]));
    const float2 h = el::mul2(el::mul2(q, t), e), up = el::fma2(h, el::twice(-1.f), el::twice(1.f));
    P = make_float2(a.x < 0.f ? h.x : up.x, a.y < 0.f ? h.y : up.y);
}

// The activation of two values.
template <int ACT, bool FINE>
__device__ __forceinline__ float2 act2(float2 a)
{
    if constexpr (ACT == OMC_GATE_GELU) {
        float2 e, P;
        normal2<FINE>(a, e, P);
        return el::mul2(a, P);
    } else {
        float2 s, t;
        sigmoid2<FINE>(a, s, t);
        return ACT == OMC_GATE_SILU ? el::mul2(a, s) : s;
    }
}
// The activation and its derivative, of two values.
template <int ACT, bool FINE>
__device__ __forceinline__ void act_slope2(float2 a, float2 &v, float2 &d)
{
    if constexpr (ACT == OMC_GATE_GELU) {
        float2 e, P;
        normal2<FINE>(a, e, P);
        v = el::mul2(a, P);
        d = el::fma2(el::mul2(a, el::twice(0.39894228f)), e, P);
    } else {
        float2 s, t;
        sigmoid2<FINE>(a, s, t);
        // SiLU of 16-bit values: a product of these by a slope or an s next to 1 often lies next to a tie of the result, so that these are to be off by their last
        // rounding alone (1 - t is; the reciprocal by as much as three times that).
        if constexpr (ACT == OMC_GATE_SILU && !FINE) {
            const float2 high = el::fma2(t, el::twice(-1.f), el::twice(1.f));
            s = make_float2(a.x < 0.f ? s.x : high.x, a.y < 0.f ? s.y : high.y);
        }
        v = ACT == OMC_GATE_SILU ? el::mul2(a, s) : s;
        // (SiLU: where FINE = false in the shorter form, whose parts are larger than d where they cancel, around a = -1.28)
        d = ACT == OMC_GATE_SIGMOID ? el::mul2(s, t) : FINE ? el::mul2(s, el::fma2(a, t, el::twice(1.f))) : el::fma2(v, t, s);
    }
}

}  // namespace gate
}  // namespace omc
