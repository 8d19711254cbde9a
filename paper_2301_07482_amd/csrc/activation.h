// The activations of the layers beside the path, and their slopes, in fp32.
#pragma once
#include <type_traits>

#include "common.h"

// 1 / (1 + e^-u) in four instructions: off by a few steps of 2^-24 and as many more as |u|, by which the exponential goes
__device__ __forceinline__ float fg_sigmoid(float u) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * u)); }
// The normal distribution function Phi(u), and e = e^(-u^2/2). With s = |u|: Phi(-s) e^(s^2/2) is a smooth function of t = 1 / (1 + p s), here a polynomial of degree 9
// in t without a constant term, fitted to relative error 2.5e-8 over s in [0, 14] (below which Phi(-s) leaves fp32); p = 0.26 gave the least. In fp32 off by a few steps of 2^-24 of the
// value and u^2 more, in either tail. About 20 instructions; with the library's erfc in its place an epilogue of 256 x 128 outputs took 20 us.
__device__ __forceinline__ float fg_normal_cdf(float u, float& e) {
    const float s = fabsf(u), t = __builtin_amdgcn_rcpf(fmaf(0.26f, s, 1.f));
    float q = 3.050470095e-02f;
    q = fmaf(q, t, -1.528279207e-01f);
    q = fmaf(q, t, 2.514894053e-01f);
    q = fmaf(q, t, -1.509467895e-01f);
    q = fmaf(q, t, 1.609463382e-01f);
    q = fmaf(q, t, 5.102833690e-02f);
    q = fmaf(q, t, 1.030300833e-01f);
    q = fmaf(q, t, 1.030167749e-01f);
    q = fmaf(q, t, 1.037590584e-01f);
    e = __builtin_amdgcn_exp2f(-0.72134752044448170f * u * u);
    const float tail = q * t * e;
    return u < 0.f ? tail : 1.f - tail;
}

template <int ACT>
__device__ __forceinline__ float fg_act(float u) {
    if constexpr (ACT == FG_ACT_RELU) return __builtin_elementwise_maximum(u, 0.f);      // (a NaN stays one)
    if constexpr (ACT == FG_ACT_SILU) return u * fg_sigmoid(u);
    if constexpr (ACT == FG_ACT_GELU) {
        float e;
        return u * fg_normal_cdf(u, e);
    }
    if constexpr (ACT == FG_ACT_SIGMOID) return fg_sigmoid(u);
    return u;
}
// f = act(u), slope = act'(u); ReLU's slope at 0 is 0
template <int ACT>
__device__ __forceinline__ void fg_act_slope(float u, float& f, float& slope) {
    f = u;
    slope = 1.f;
    if constexpr (ACT == FG_ACT_RELU) {
        f = __builtin_elementwise_maximum(u, 0.f);
        slope = u > 0.f ? 1.f : (u <= 0.f ? 0.f : u);
    } else if constexpr (ACT == FG_ACT_SILU) {
        const float s = fg_sigmoid(u);
        f = u * s;
        slope = s + f * (1.f - s);
    } else if constexpr (ACT == FG_ACT_GELU) {
        float e;
        const float c = fg_normal_cdf(u, e);
        f = u * c;
        slope = c + u * (0.39894228040143268f * e);
    } else if constexpr (ACT == FG_ACT_SIGMOID) {
        f = fg_sigmoid(u);
        slope = f * (1.f - f);
    }
}
// calls f with the activation as a constant
template <typename F>
__host__ __device__ __forceinline__ void fg_with_act(int act, const F& f) {
    switch (act) {
        case FG_ACT_RELU: return f(std::integral_constant<int, FG_ACT_RELU>());
        case FG_ACT_SILU: return f(std::integral_constant<int, FG_ACT_SILU>());
        case FG_ACT_GELU: return f(std::integral_constant<int, FG_ACT_GELU>());
        case FG_ACT_SIGMOID: return f(std::integral_constant<int, FG_ACT_SIGMOID>());
        default: return f(std::integral_constant<int, FG_ACT_NONE>());
    }
}
static inline bool fg_act_known(int act) { return act >= FG_ACT_NONE && act <= FG_ACT_SIGMOID; }
