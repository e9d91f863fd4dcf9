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

// The forward pass's Phi, for a bf16 result: Phi(-a) = 2^P(a), P of degree 9 fitted to log2 of it over [0, 12.9], where fp32
// ends: off by 8e-6 of itself up to a = 4, 2.2e-5 up to 8 and 8.2e-5 at the end; P falls for ever beyond.  (Degree 7 fitted to
// the size of a Phi(-a) was off by 3.4e-6 up to 4, but by 3.6e-3 at 6 and a tenth at 8; its two multiply-adds less are 1.4 us of
// ViT-B's forward pass, 125.9 and 127.4 us.)  Nine multiply-adds and an exponential, no reciprocal.
__device__ inline float normal_tail(float a)            // 0 <= a <= 100
{
    float p = fmaf(a, -2.40522136e-09f, 1.67417483e-07f);
    p = fmaf(p, a, -5.13553641e-06f);
    p = fmaf(p, a, 9.20612656e-05f);
    p = fmaf(p, a, -0.00108233339f);
    p = fmaf(p, a, 0.00893035159f);
    p = fmaf(p, a, -0.0545950532f);
    p = fmaf(p, a, -0.458002746f);
    p = fmaf(p, a, -1.15137577f);
    return __builtin_amdgcn_exp2f(fmaf(p, a, -0.999989986f));
}

// The slopes' Phi, whose sums over the tokens leave in fp32: Phi(-a) = e^(-a^2 / 2) t Q(t), t = 1 / (1 + 0.305 a), Q of degree 7
// fitted to the ratio over [0, 13.3], largest relative error made smallest: 6e-8, in fp32 5e-7 with the reciprocal's, and the
// exponential's on top, which the slope needs anyhow.  (ViT-B's backward pass takes 137.3 us with it, 136.9 with formula 7.1.26 of
// Abramowitz and Stegun, which is 1 % off at 8.)
__device__ inline float normal_tail_of(float a, float bell)                 // bell = e^(-a^2 / 2)
{
    const float t = __builtin_amdgcn_rcpf(fmaf(0.304987103f, a, 1.f));
    float q = fmaf(t, 0.0368816517f, -0.153805956f);
    q = fmaf(q, t, 0.187227234f);
    q = fmaf(q, t, -0.0394248515f);
    q = fmaf(q, t, 0.121822082f);
    q = fmaf(q, t, 0.103164561f);
    q = fmaf(q, t, 0.122503579f);
    q = fmaf(q, t, 0.121631771f);
    return bell * t * q;
}

constexpr float TANH_K = 0.7978845608028654f, TANH_C = 0.044715f;           // sqrt(2 / pi)

template <bool FAST> __device__ inline float activation(float z, int act)
{
    switch (act) {                                     // (the same branch in every thread of a launch)
    case DROPIT_ACT_SILU: return FAST ? z * sigmoid_of<true>(z) : z / (1.f + expf(-z));
    case DROPIT_ACT_GELU:
        if constexpr (FAST) {                          // max(z, 0) - |z| Phi(-|z|); an infinity or a NaN stays one
            const float a = fminf(fabsf(z), 100.f);
            return fmaf(-a, normal_tail(a), z < 0.f ? 0.f : z);
        } else {
            return z * (0.5f * erfcf(-0.70710678118654752f * z));
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
    case DROPIT_ACT_GELU: {                            // Phi(z) + z e^(-z^2 / 2) / sqrt(2 pi)
        const float bell = exp_of<FAST>(-0.5f * z * z);
        float phi;
        if constexpr (FAST) {
            const float tail = normal_tail_of(fabsf(z), bell);
            phi = z < 0.f ? tail : 1.f - tail;
        } else {
            phi = 0.5f * erfcf(-0.70710678118654752f * z);
        }
        slope = phi + z * bell * 0.3989422804014327f;
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
