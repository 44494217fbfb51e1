// Activations of the feed-forward operators and their derivatives, in fp32:
//   none z; ReLU max(z, 0); GELU z Phi(z), Phi the normal distribution function; GELU by tanh z s(2u), u = sqrt(2/pi) (z + 0.044715 z^3)
//   (0.5 (1 + tanh u) = s(2u), s the logistic function); SiLU z s(z).
// A NaN stays one.  Where z is infinite the formulas' own 0 * infinity stays NaN for GELU and SiLU; finite z never overflow into one.
#pragma once

#include "block_prims.h"
#include "sgnn.h"

struct ff_act_pair { float f, d; };       // act(z) and act'(z)

// 1 / (1 + exp(-x)) from the exponential of -|x|, which cannot overflow.  QUICK, beside products of bfloat16
// operands: the exponential as 2^(-x log2 e) with the rounding of that product, x s(x) and its slope to within 2^-22 of the larger of |x| and 1, against
// the 2^-9 of the operands' rounding; 4 instructions instead of 15 (gated product of 65536 x 256 x 704 97 -> 92 us, its backward pass, ff_dx.hip, 260 -> 253)
template <bool QUICK = false> __device__ __forceinline__ float ff_logistic(float x)
{
    if constexpr (QUICK) return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * -1.44269502162933349609375f));
    const float e = exp_neg(-fabsf(x)), r = __builtin_amdgcn_rcpf(1.f + e);
    return x >= 0.f ? r : (x < 0.f ? e * r : x);           // the last for a NaN
}

// 2 sqrt(2/pi) (z + 0.044715 z^3); beyond 12 in magnitude the logistic function of it is 0 or 1 in fp32
__device__ __forceinline__ float ff_gelu_inner(float z)
{
    const float c = z != z ? z : fminf(fmaxf(z, -12.f), 12.f);
    return 1.5957691216057308f * c * fmaf(0.044715f * c, c, 1.f);
}

// Phi(z) and the density phi(z), both from exp(-z^2 / 2): 1 - Phi = phi-like polynomial of 1 / (1 + p |z| / sqrt 2) (C. Hastings, "Approximations for
// Digital Computers", 1955, sheet 43: the error function to 1.5e-7), so that a slope costs one exponential.
__device__ __forceinline__ ff_act_pair ff_normal(float z)
{
    const float c = z != z ? z : fminf(fabsf(z), 20.f);              // the exponential is 0 in fp32 beyond
    const float e = exp_neg(-0.5f * c * c), t = __builtin_amdgcn_rcpf(fmaf(0.3275911f * 0.70710678118654752f, c, 1.f));
    const float q = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    const float half = 0.5f * q * e;
    return {z >= 0.f ? 1.f - half : half, e * 0.3989422804014327f};
}

template <int ACT, bool QUICK = false> __device__ __forceinline__ float ff_act(float z)
{
    if constexpr (ACT == SGNN_ACT_RELU) return z > 0.f ? z : (z != z ? z : 0.f);
    else if constexpr (ACT == SGNN_ACT_GELU) return z * ff_normal(z).f;
    else if constexpr (ACT == SGNN_ACT_GELU_TANH) return z * ff_logistic<QUICK>(ff_gelu_inner(z));
    else if constexpr (ACT == SGNN_ACT_SILU) return z * ff_logistic<QUICK>(z);
    else return z;
}

template <int ACT, bool QUICK = false> __device__ __forceinline__ ff_act_pair ff_act_both(float z)
{
    if constexpr (ACT == SGNN_ACT_RELU) return {ff_act<ACT, QUICK>(z), z > 0.f ? 1.f : (z != z ? z : 0.f)};
    else if constexpr (ACT == SGNN_ACT_GELU) {
        const ff_act_pair n = ff_normal(z);
        const float c = z != z ? z : fminf(fmaxf(z, -20.f), 20.f);
        return {z * n.f, fmaf(c, n.d, n.f)};
    } else if constexpr (ACT == SGNN_ACT_GELU_TANH) {
        const float s = ff_logistic<QUICK>(ff_gelu_inner(z));
        const float c = z != z ? z : fminf(fmaxf(z, -12.f), 12.f);
        return {z * s, fmaf(c * s * (1.f - s), 1.5957691216057308f * fmaf(0.134145f * c, c, 1.f), s)};
    } else if constexpr (ACT == SGNN_ACT_SILU) {
        // (where z is a NaN s is one)
        const float s = ff_logistic<QUICK>(z), c = __builtin_amdgcn_fmed3f(z, -120.f, 120.f);
        return {z * s, s * fmaf(c, 1.f - s, 1.f)};
    } else return {z, 1.f};
}

// f(integral_constant<int, act>) for an activation known at run time only
template <class F> __device__ __forceinline__ void ff_with_act(int act, F f)
{
    switch (act) {
    case SGNN_ACT_RELU: f(std::integral_constant<int, SGNN_ACT_RELU>()); break;
    case SGNN_ACT_GELU: f(std::integral_constant<int, SGNN_ACT_GELU>()); break;
    case SGNN_ACT_GELU_TANH: f(std::integral_constant<int, SGNN_ACT_GELU_TANH>()); break;
    case SGNN_ACT_SILU: f(std::integral_constant<int, SGNN_ACT_SILU>()); break;
    default: f(std::integral_constant<int, SGNN_ACT_NONE>()); break;
    }
}
