// Activation functions and their slopes, binary32.
//
// The normal distribution's tail Q(z) = erfc(z / sqrt 2) / 2, z >= 0, is taken as exp(-z^2/2) times a polynomial in
// t = 1 / (1 + p z) without constant term (the form of Hastings' approximations): erfc(u) exp(u^2) is smooth in t and tends
// to 0 with it.  The coefficients are a least-maximum fit of the relative error over 0 <= u <= 10: 9.3e-8, and 5.1e-7 with the
// roundings of the polynomial.  The exponential is the one that the slope needs anyway: the function and its slope cost one
// v_exp_f32 and one v_rcp_f32 (1 ulp each).  The library's erff needs about three times the instructions, with which these
// kernels would be bound by them and not by memory.
//
// Far below 0 the functions are as exact as their exponential.  Its argument is rounded to binary32, three times for GELU (x^2, the
// constant, their product) and twice for SiLU, and an argument that is off by d moves the result by d of itself: up to
// 5e-7 + 9e-8 x^2 of itself for GELU, 2e-7 + 1.2e-7 |x| for SiLU.  Carrying the remainders along would take four or five more
// instructions for values that are all but 0 beside the others of their row.
#ifndef MGWFBP_ACT_KINDS_H
#define MGWFBP_ACT_KINDS_H

#include <hip/hip_runtime.h>

#include "mgwfbp_layers.h"

namespace ops {

constexpr float LOG2_E = 1.44269504088896341f;

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * LOG2_E); }

// x and its kind to the function's value and slope; what is not used falls away.
template <int KIND> __device__ __forceinline__ void activate(float x, float& value, float& slope) {
    if constexpr (KIND == MGWFBP_IDENTITY) {
        value = x;
        slope = 1.f;
    } else if constexpr (KIND == MGWFBP_GELU) {
        const float e = __builtin_amdgcn_exp2f(x * x * (-0.5f * LOG2_E));
        const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.233345237791561f, __builtin_fabsf(x), 1.f));     // p = 0.33, z = |x|
        float p = -0.06768140680997151f;                       // the coefficients halved
        p = __builtin_fmaf(p, t, 0.2301546599299484f);
        p = __builtin_fmaf(p, t, -0.17563803381566054f);
        p = __builtin_fmaf(p, t, 0.20430967425440442f);
        p = __builtin_fmaf(p, t, 0.023577627350098162f);
        p = __builtin_fmaf(p, t, 0.10062231325500619f);
        p = __builtin_fmaf(p, t, 0.09147620121370333f);
        p = __builtin_fmaf(p, t, 0.09317902474729383f);
        const float tail = p * t * e;
        // The tail is 0 far before 2^100, so the bound changes no finite x's product; +inf keeps its value, -inf is -inf * 0 = NaN.
        value = __builtin_fmaf(-__builtin_fabsf(__builtin_fminf(x, 0x1p100f)), tail, __builtin_fmaxf(x, 0.f));
        const float below = x >= 0.f ? 1.f - tail : tail;      // Phi(x)
        slope = __builtin_fmaf(x * 0.3989422804014327f, e, below);
    } else if constexpr (KIND == MGWFBP_GELU_TANH) {
        // (1 + tanh u) / 2 is the logistic function of 2u
        constexpr float A = 1.5957691216057308f, B = 0.044715f;            // 2 sqrt(2/pi)
        const float s = __builtin_amdgcn_rcpf(1.f + exp_of(-A * x * __builtin_fmaf(B * x, x, 1.f)));
        value = x * s;
        // Beyond 64, s is 0 or 1 and the slope s to all digits; x^2 is bounded there, so that it is no infinity times 0.
        const float near = __builtin_fminf(__builtin_fabsf(x), 64.f);
        slope = __builtin_fmaf(value * (1.f - s), A * __builtin_fmaf(3.f * B * near, near, 1.f), s);
    } else {
        const float s = __builtin_amdgcn_rcpf(1.f + exp_of(-x));
        value = x * s;
        slope = __builtin_fmaf(value, 1.f - s, s);
    }
}

// Calls f with the kind as a constant.
template <int K> struct Kind { static constexpr int value = K; };
template <typename F> int with_kind(int32_t kind, F&& f) {
    switch (kind) {
        case MGWFBP_IDENTITY: return f(Kind<MGWFBP_IDENTITY>());
        case MGWFBP_GELU: return f(Kind<MGWFBP_GELU>());
        case MGWFBP_GELU_TANH: return f(Kind<MGWFBP_GELU_TANH>());
        case MGWFBP_SILU: return f(Kind<MGWFBP_SILU>());
        default: return MGWFBP_EINVAL;
    }
}

}  // namespace ops

#endif
