// The activations of the layers beside the path, and their slopes, in fp32.
#pragma once
#include <type_traits>

#include "common.h"

__device__ __forceinline__ float fg_sigmoid(float u) { return 1.f / (1.f + expf(-u)); }
__device__ __forceinline__ float fg_normal_cdf(float u) { return 0.5f * erfcf(-0.70710678118654752f * u); }

template <int ACT>
__device__ __forceinline__ float fg_act(float u) {
    if constexpr (ACT == FG_ACT_RELU) return __builtin_elementwise_maximum(u, 0.f);      // (a NaN stays one)
    if constexpr (ACT == FG_ACT_SILU) return u * fg_sigmoid(u);
    if constexpr (ACT == FG_ACT_GELU) return u * fg_normal_cdf(u);
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
        const float c = fg_normal_cdf(u);
        f = u * c;
        slope = c + u * (0.39894228040143268f * expf(-0.5f * u * u));
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
