// The activations of the gated projection and their slopes (internal header).
#pragma once

#include <type_traits>

#include "common.hpp"
#include "dropit_layers.h"

namespace dropit {
namespace {

// e^x, 1 / x: the hardware's (a relative 2^-22 or so, times |x| for the exponential's argument) where the result is rounded
// to bf16, the math library's where it stays fp32
template <bool FAST> __device__ inline float exp_of(float x) { return FAST ? __builtin_amdgcn_exp2f(x * 1.4426950408889634f) : expf(x); }
template <bool FAST> __device__ inline float inverse_of(float x) { return FAST ? __builtin_amdgcn_rcpf(x) : 1.f / x; }

template <bool FAST> __device__ inline float sigmoid_of(float z) { return inverse_of<FAST>(1.f + exp_of<FAST>(-z)); }

// Phi(-|z|) = 2^P(|z|), P of degree 7 fitted to log2 of it over [0, 5.5] (largest relative error of the result, weighted with
// |z| Phi beyond 4, made smallest): off by 3.4e-6 of itself up to |z| = 4 and never by more than 3.3e-7 / |z|; P falls for
// ever beyond.  Seven multiply-adds and an exponential, no reciprocal: ViT-B's forward pass leaves with a third less of it.
__device__ inline float normal_tail(float a)            // a = |z|
{
    float p = fmaf(a, -9.67966821e-07f, 4.85793513e-05f);
    p = fmaf(p, a, -0.000854563057f);
    p = fmaf(p, a, 0.00829118465f);
    p = fmaf(p, a, -0.0536483587f);
    p = fmaf(p, a, -0.458673029f);
    p = fmaf(p, a, -1.1512002f);
    return __builtin_amdgcn_exp2f(fmaf(p, a, -0.999997246f));
}

// Phi(z), and e^(-z^2 / 2) for the slope.  FAST: Abramowitz and Stegun, Handbook of Mathematical Functions, formula 7.1.26
// for erfc(|z| / sqrt 2), halved; off by at most 1.5e-7
template <bool FAST> __device__ inline float normal_cdf(float z, float &bell)
{
    bell = exp_of<FAST>(-0.5f * z * z);
    if constexpr (!FAST) {
        return 0.5f * erfcf(-0.70710678118654752f * z);
    } else {
        const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f * 0.70710678118654752f, fabsf(z), 1.f));
        float s = fmaf(t, 1.061405429f, -1.453152027f);
        s = fmaf(s, t, 1.421413741f);
        s = fmaf(s, t, -0.284496736f);
        s = fmaf(s, t, 0.254829592f);
        const float q = 0.5f * s * t * bell;
        return z < 0.f ? q : 1.f - q;
    }
}

constexpr float TANH_K = 0.7978845608028654f, TANH_C = 0.044715f;           // sqrt(2 / pi)

template <bool FAST> __device__ inline float activation(float z, int act)
{
    switch (act) {                                     // (the same branch in every thread of a launch)
    case DROPIT_ACT_SILU: return FAST ? z * sigmoid_of<true>(z) : z / (1.f + expf(-z));
    case DROPIT_ACT_GELU: {
        if constexpr (FAST) {                          // max(z, 0) - |z| Phi(-|z|); an infinity or a NaN stays one
            const float a = fminf(fabsf(z), 100.f);
            return fmaf(-a, normal_tail(a), z < 0.f ? 0.f : z);
        }
        float bell;
        return z * normal_cdf<FAST>(z, bell);
    }
    case DROPIT_ACT_GELU_TANH: return z * sigmoid_of<FAST>(2.f * TANH_K * (z + TANH_C * z * z * z));    // (1 + tanh y) / 2 = sigmoid(2 y)
    case DROPIT_ACT_RELU: return z < 0.f ? 0.f : z;    // (a NaN stays one)
    default: return sigmoid_of<FAST>(z);
    }
}

// act over N values at once: one branch for all of them, and their exponentials and reciprocals in flight together
template <bool FAST, int N> __device__ inline void activations(float (&z)[N], int act)
{
    auto each = [&](auto code) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = activation<FAST>(z[i], decltype(code)::value);
    };
    switch (act) {
    case DROPIT_ACT_SILU: return each(std::integral_constant<int, DROPIT_ACT_SILU>{});
    case DROPIT_ACT_GELU: return each(std::integral_constant<int, DROPIT_ACT_GELU>{});
    case DROPIT_ACT_GELU_TANH: return each(std::integral_constant<int, DROPIT_ACT_GELU_TANH>{});
    case DROPIT_ACT_RELU: return each(std::integral_constant<int, DROPIT_ACT_RELU>{});
    default: return each(std::integral_constant<int, DROPIT_ACT_SIGMOID>{});
    }
}

// act(z), and act'(z) in `slope`
template <bool FAST> __device__ inline float activation_slope(float z, int act, float &slope)
{
    switch (act) {
    case DROPIT_ACT_SILU: {
        const float s = sigmoid_of<FAST>(z);
        slope = s * (1.f + z * (1.f - s));
        return z * s;
    }
    case DROPIT_ACT_GELU: {
        float bell;
        const float phi = normal_cdf<FAST>(z, bell);
        slope = phi + z * bell * 0.3989422804014327f;  // 1 / sqrt(2 pi)
        return z * phi;
    }
    case DROPIT_ACT_GELU_TANH: {
        const float s = sigmoid_of<FAST>(2.f * TANH_K * (z + TANH_C * z * z * z));
        const float c = fminf(fmaxf(z, -64.f), 64.f);  // (s (1 - s) is zero there; z^2 overflows from 2^64 on)
        slope = s + c * s * (1.f - s) * (2.f * TANH_K) * (1.f + 3.f * TANH_C * c * c);
        return z * s;
    }
    case DROPIT_ACT_RELU:
        slope = z > 0.f ? 1.f : 0.f;
        return z < 0.f ? 0.f : z;
    default: {                                         // s(z) s(-z): 1 - s would have nothing left from z = 17 on
        const float e = exp_of<FAST>(-fabsf(z)), r = inverse_of<FAST>(1.f + e);
        slope = e * r * r;
        return z < 0.f ? e * r : r;
    }
    }
}

// the same over N values: act(z) in place of z, act'(z) in `slope`
template <bool FAST, int N> __device__ inline void activation_slopes(float (&z)[N], int act, float (&slope)[N])
{
    auto each = [&](auto code) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = activation_slope<FAST>(z[i], decltype(code)::value, slope[i]);
    };
    switch (act) {
    case DROPIT_ACT_SILU: return each(std::integral_constant<int, DROPIT_ACT_SILU>{});
    case DROPIT_ACT_GELU: return each(std::integral_constant<int, DROPIT_ACT_GELU>{});
    case DROPIT_ACT_GELU_TANH: return each(std::integral_constant<int, DROPIT_ACT_GELU_TANH>{});
    case DROPIT_ACT_RELU: return each(std::integral_constant<int, DROPIT_ACT_RELU>{});
    default: return each(std::integral_constant<int, DROPIT_ACT_SIGMOID>{});
    }
}

}  // namespace
}  // namespace dropit
