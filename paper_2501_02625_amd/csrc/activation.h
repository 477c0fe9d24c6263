// The activations of the epilogue and their slopes (halo_activation in halo.h), fp32.
//
// What bounds them is instructions: in a product's epilogue nothing hides them.  Hence the hardware's exp2 and reciprocal, one rounding
// off, without the library's special cases, and for gelu one exponential that serves both Phi and its density:
//   Phi(-a) = exp(-a^2 / 2) g(1 / (1 + c a)),  a >= 0,
// g a polynomial without a constant, fitted to the scaled complementary error function so that the largest relative error is as small as
// it gets: of degree 8 1.5e-7 (gelu over [-8, 8] is 2.4e-7 off at most), of degree 5 3.2e-5.  The shorter one is for results that
// are rounded to bf16 as they are, whose half steps are 60 to 120 times that: 0.24 % of them become the other neighbour.  In front of a
// residual's sum it is not taken: where the residual nearly cancels gelu, 3.2e-5 of gelu is many steps of what is left.  8192 x 14336 x
// 4096 with gelu and Z takes 426 us with the short one, 436 with the long one; with gelu and a residual 424 and 433.
#pragma once

#include <hip/hip_runtime.h>

#include "halo.h"

namespace halo {

constexpr float kLog2e = 1.44269504088896340736f;

// 1 / (1 + exp(-x)); e: exp(-x), for which x should be at least -80.
__device__ __forceinline__ float logistic(float x, float& e) {
    e = __builtin_amdgcn_exp2f(x * -kLog2e);
    return __builtin_amdgcn_rcpf(1.0f + e);
}
// Phi(-|x|), Phi the normal distribution function, and its density times sqrt(2 pi).  SHORT: the polynomial of degree 5.
template <bool SHORT>
__device__ __forceinline__ float normal_tail(float x, float& density) {
    const float a = __builtin_fabsf(x), t = __builtin_amdgcn_rcpf(__builtin_fmaf(SHORT ? 0.375f : 0.3f, a, 1.0f));
    float g;
    if constexpr (SHORT) {
        g = __builtin_fmaf(-0.090650067015f, t, 0.200297825896f);
        g = __builtin_fmaf(g, t, 0.083551545722f);
        g = __builtin_fmaf(g, t, 0.157737905872f);
        g = __builtin_fmaf(g, t, 0.149060613254f);
    } else {
        g = __builtin_fmaf(0.035679225315f, t, -0.157222291421f);
        g = __builtin_fmaf(g, t, 0.206387594394f);
        g = __builtin_fmaf(g, t, -0.053715773492f);
        g = __builtin_fmaf(g, t, 0.128578931072f);
        g = __builtin_fmaf(g, t, 0.099908185989f);
        g = __builtin_fmaf(g, t, 0.120754811127f);
        g = __builtin_fmaf(g, t, 0.119629243058f);
    }
    density = __builtin_amdgcn_exp2f(a * a * (-0.5f * kLog2e));
    return g * t * density;
}
// 2 sqrt(2 / pi) (x + 0.044715 x^3)
__device__ __forceinline__ float tanh_argument(float x) {
    return x * __builtin_fmaf(1.59576912160573071176f * 0.044715f, x * x, 1.59576912160573071176f);
}

// SHORT: the result is rounded to bf16, with nothing added to it before.
template <int ACT, bool SHORT>
__device__ __forceinline__ float activation(float x) {
    float unused;
    if constexpr (ACT == HALO_ACT_RELU) return x < 0.0f ? 0.0f : x;                    // NaN stays
    // x - x Phi(-x) or x Phi(x); the tail is 0 from 16 on, and infinity times it would be NaN (a NaN comes through the tail)
    else if constexpr (ACT == HALO_ACT_GELU)
        return __builtin_fmaf(-__builtin_fminf(__builtin_fabsf(x), 16.0f), normal_tail<SHORT>(x, unused), __builtin_fmaxf(x, 0.0f));
    else if constexpr (ACT == HALO_ACT_GELU_TANH) return x * logistic(tanh_argument(x), unused);
    else if constexpr (ACT == HALO_ACT_SILU) return x * logistic(x, unused);
    else return x;
}

// e act'(x).  Where |x| is beyond the limit the slope is within 1e-20 of 0 or 1, and is taken at the limit: x itself would make infinity
// times zero of it.
template <int ACT>
__device__ __forceinline__ float activation_slope(float e, float x) {
    if constexpr (ACT == HALO_ACT_NONE) return e;
    if constexpr (ACT == HALO_ACT_RELU) return x > 0.0f ? e : x <= 0.0f ? 0.0f : x;    // 0 where the slope is, also of an infinity
    constexpr float limit = ACT == HALO_ACT_SILU ? 80.0f : ACT == HALO_ACT_GELU ? 14.0f : 9.0f;
    const float c = x < -limit ? -limit : x > limit ? limit : x;
    float w, slope;
    if constexpr (ACT == HALO_ACT_GELU) {
        const float tail = normal_tail<false>(c, w);
        slope = __builtin_fmaf(c * 0.398942280401432677940f, w, c < 0.0f ? tail : 1.0f - tail);
    } else if constexpr (ACT == HALO_ACT_GELU_TANH) {
        const float p = logistic(tanh_argument(c), w);
        slope = __builtin_fmaf(c * p * (w * p), __builtin_fmaf(3.0f * 1.59576912160573071176f * 0.044715f, c * c, 1.59576912160573071176f), p);
    } else {
        const float p = logistic(c, w);
        slope = __builtin_fmaf(c * p, w * p, p);
    }
    return e * slope;
}

}  // namespace halo
