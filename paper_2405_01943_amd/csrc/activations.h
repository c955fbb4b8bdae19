// The activations of Sec. 2.2 Eq. 2 (dass_act) and their slopes, shared by the kernels that apply them.
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/dass.h"

namespace dass {

template <int ACT>
__device__ __forceinline__ float glu_act_fast(float g)
{
    // exp2 and the reciprocal are the hardware's 1-ulp instructions; a true division costs a
    // dozen instructions per element and the bf16 path is good to 1e-6 without it.
    if constexpr (ACT == DASS_ACT_SILU) {
        return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * g));
    } else if constexpr (ACT == DASS_ACT_GELU_TANH) {
        // 0.5 g (1 + tanh z) = g / (1 + exp(-2 z)),  z = sqrt(2/pi) (g + 0.044715 g^3)
        // exp(-2 z) = exp2(g (c0 + c1 g^2)),  c0 = -2 sqrt(2/pi) log2(e),  c1 = 0.044715 c0
        const float e = g * fmaf(-0.10294324f, g * g, -2.3022082f);
        return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(e));
    } else if constexpr (ACT == DASS_ACT_GELU_ERF) {
        // erf by the classical five-term rational form in t = 1 / (1 + p z) times exp(-z^2)
        // (Abramowitz & Stegun 7.1.26, absolute error of erf below 1.5e-7), written on z = |g| / sqrt(2)
        // so that neither branch cancels: with h = (1 - erf z) / 2 = P(t) exp(-g^2 / 2) / 2,
        // GELU(g) = g (1 - h) for g >= 0 and g h for g < 0.  The library's erff is several times the
        // instructions; the norms are good to 1e-6 either way.
        const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(g), 0.3275911f * 0.70710678f, 1.0f));
        float P = fmaf(t, 1.061405429f, -1.453152027f);
        P = fmaf(t, P, 1.421413741f);
        P = fmaf(t, P, -0.284496736f);
        P = fmaf(t, P, 0.254829592f);
        const float h = 0.5f * t * P * __builtin_amdgcn_exp2f(g * g * -0.72134752f);   // exp(-g^2 / 2)
        return g * (g >= 0.0f ? 1.0f - h : h);
    } else {
        return fmaxf(g, 0.0f);
    }
}

__device__ __forceinline__ float glu_act_precise(float g, int act)
{
    switch (act) {
    case DASS_ACT_SILU:
        return g / (1.0f + expf(-g));
    case DASS_ACT_GELU_TANH: {
        const float z2 = 1.5957691216057308f * g * (1.0f + 0.044715f * g * g);
        return g / (1.0f + expf(-z2));
    }
    case DASS_ACT_GELU_ERF:
        return 0.5f * g * (1.0f + erff(g * 0.7071067811865476f));
    default:
        return fmaxf(g, 0.0f);
    }
}

// The same with none among them, for the linear layers.  FAST: the hardware's exponential and reciprocal, for results
// that are rounded to bf16.  The precise GELU takes erfc, which keeps its digits where 1 + erf cancels.  NaN stays NaN in every
// value and slope: maxima and minima would drop it, so relu and the slope of gelu_tanh compare.
template <bool FAST>
__device__ __forceinline__ float act_value(float x, int act)
{
    switch (act) {
    case DASS_ACT_NONE:
        return x;
    case DASS_ACT_SILU:
        return FAST ? glu_act_fast<DASS_ACT_SILU>(x) : glu_act_precise(x, DASS_ACT_SILU);
    case DASS_ACT_GELU_TANH:
        return FAST ? glu_act_fast<DASS_ACT_GELU_TANH>(x) : glu_act_precise(x, DASS_ACT_GELU_TANH);
    case DASS_ACT_GELU_ERF:
        return FAST ? glu_act_fast<DASS_ACT_GELU_ERF>(x) : 0.5f * x * erfcf(-0.7071067811865476f * x);
    default:
        return x <= 0.0f ? 0.0f : x;
    }
}

// act_value of N values at once: one decision for all of them.
template <bool FAST, int N>
__device__ __forceinline__ void act_values(float (&v)[N], int act)
{
    switch (act) {
    case DASS_ACT_NONE:
        break;
    case DASS_ACT_SILU:
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = act_value<FAST>(v[i], DASS_ACT_SILU);
        break;
    case DASS_ACT_GELU_TANH:
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = act_value<FAST>(v[i], DASS_ACT_GELU_TANH);
        break;
    case DASS_ACT_GELU_ERF:
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = act_value<FAST>(v[i], DASS_ACT_GELU_ERF);
        break;
    default:
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = act_value<FAST>(v[i], DASS_ACT_RELU);
    }
}

// act'(x):
//   silu       s (1 + x (1 - s)),       s = 1 / (1 + exp(-x))
//   gelu_tanh  s + x s (1 - s) z',      s = 1 / (1 + exp(-z)), z = 2 sqrt(2/pi) (x + 0.044715 x^3); x is held to
//              [-12, 12], where the slope is 0 and 1 to every bit, so that no overflow of z' meets a zero
//   gelu_erf   Phi(x) + x exp(-x^2 / 2) / sqrt(2 pi)
//   relu       1 for x > 0, 0 for x <= 0
template <bool FAST>
__device__ __forceinline__ float act_slope(float x, int act)
{
    switch (act) {
    case DASS_ACT_NONE:
        return 1.0f;
    case DASS_ACT_SILU: {
        const float s = FAST ? __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * x))
                             : 1.0f / (1.0f + expf(-x));
        return s * fmaf(x, 1.0f - s, 1.0f);
    }
    case DASS_ACT_GELU_TANH: {
        const float c = x > 12.0f ? 12.0f : x < -12.0f ? -12.0f : x, c2 = c * c;
        const float z = 1.5957691216057308f * c * fmaf(0.044715f, c2, 1.0f);
        const float s = FAST ? __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z))
                             : 1.0f / (1.0f + expf(-z));
        return fmaf(c * s * (1.0f - s), 1.5957691216057308f * fmaf(0.134145f, c2, 1.0f), s);
    }
    case DASS_ACT_GELU_ERF: {
        float cdf, bell;   // bell = exp(-x^2 / 2)
        if (FAST) {        // the rational form of glu_act_fast
            const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(x), 0.3275911f * 0.70710678f, 1.0f));
            float P = fmaf(t, 1.061405429f, -1.453152027f);
            P = fmaf(t, P, 1.421413741f);
            P = fmaf(t, P, -0.284496736f);
            P = fmaf(t, P, 0.254829592f);
            bell = __builtin_amdgcn_exp2f(x * x * -0.72134752f);
            const float h = 0.5f * t * P * bell;
            cdf = x >= 0.0f ? 1.0f - h : h;
        } else {
            bell = expf(-0.5f * x * x);
            cdf = 0.5f * erfcf(-0.7071067811865476f * x);
        }
        return fmaf(0.3989422804014327f * x, bell, cdf);
    }
    default:
        return x > 0.0f ? 1.0f : x <= 0.0f ? 0.0f : x;
    }
}

// act_slope of N values at once.
template <bool FAST, int N>
__device__ __forceinline__ void act_slopes(const float (&x)[N], float (&v)[N], int act)
{
    switch (act) {
    case DASS_ACT_NONE:
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = 1.0f;
        break;
    case DASS_ACT_SILU:
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = act_slope<FAST>(x[i], DASS_ACT_SILU);
        break;
    case DASS_ACT_GELU_TANH:
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = act_slope<FAST>(x[i], DASS_ACT_GELU_TANH);
        break;
    case DASS_ACT_GELU_ERF:
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = act_slope<FAST>(x[i], DASS_ACT_GELU_ERF);
        break;
    default:
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = act_slope<FAST>(x[i], DASS_ACT_RELU);
    }
}

}  // namespace dass
