// Activations of the gated feed-forward block and their derivatives, in fp32.
#pragma once

#include "bsr.h"

namespace bsr {

// 1 / (1 + e^-x); FAST: the hardware's exponential, whose relative error of about
// 2^-21 is lost in a result rounded to bf16.
template <bool FAST>
__device__ __forceinline__ float logistic(float x) {
    return __fdividef(1.f, 1.f + (FAST ? __expf(-x) : expf(-x)));
}

constexpr float kGeluA = 0.7978845608028654f;   // sqrt(2 / pi)
constexpr float kGeluB = 0.044715f;

// Phi(g), the normal distribution
template <bool FAST>
__device__ __forceinline__ float normal_cdf(float g) {
    return FAST ? fmaf(0.5f, erff(0.70710678f * g), 0.5f) : normcdff(g);
}
// the tanh form of GELU is g / (1 + e^-2u), which is the same; 2u
__device__ __forceinline__ float gelu_2u(float g) { return 2.f * kGeluA * g * fmaf(kGeluB * g, g, 1.f); }

template <int ACT, bool FAST>
__device__ __forceinline__ float activate(float g) {
    if constexpr (ACT == BSR_ACT_SILU) return g * logistic<FAST>(g);
    else if constexpr (ACT == BSR_ACT_GELU) return g * normal_cdf<FAST>(g);
    else if constexpr (ACT == BSR_ACT_GELU_TANH) return g * logistic<FAST>(gelu_2u(g));
    else if constexpr (ACT == BSR_ACT_RELU) return g > 0.f ? g : (g != g ? g : 0.f);
    else return logistic<FAST>(g);
}

// act(g) and act'(g).
template <int ACT, bool FAST>
__device__ __forceinline__ float2 activate_slope(float g) {
    if constexpr (ACT == BSR_ACT_SILU) {
        const float p = logistic<FAST>(g);
        return make_float2(g * p, p * fmaf(g, 1.f - p, 1.f));
    } else if constexpr (ACT == BSR_ACT_GELU) {
        const float p = normal_cdf<FAST>(g), density = 0.3989422804f * (FAST ? __expf(-0.5f * g * g) : expf(-0.5f * g * g));
        return make_float2(g * p, fmaf(g, density, p));
    } else if constexpr (ACT == BSR_ACT_GELU_TANH) {
        const float p = logistic<FAST>(gelu_2u(g));
        return make_float2(g * p, fmaf(g * p * (1.f - p), 2.f * kGeluA * fmaf(3.f * kGeluB * g, g, 1.f), p));
    } else if constexpr (ACT == BSR_ACT_RELU) {
        return make_float2(g > 0.f ? g : (g != g ? g : 0.f), g > 0.f ? 1.f : (g != g ? g : 0.f));
    } else {
        const float p = logistic<FAST>(g);
        return make_float2(p, p * (1.f - p));
    }
}

// Calls f with the activation as a compile-time constant.
template <int N>
struct ActTag {
    static constexpr int value = N;
};
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
    switch (act) {
        case BSR_ACT_SILU: f(ActTag<BSR_ACT_SILU>{}); break;
        case BSR_ACT_GELU: f(ActTag<BSR_ACT_GELU>{}); break;
        case BSR_ACT_GELU_TANH: f(ActTag<BSR_ACT_GELU_TANH>{}); break;
        case BSR_ACT_RELU: f(ActTag<BSR_ACT_RELU>{}); break;
        default: f(ActTag<BSR_ACT_SIGMOID>{}); break;
    }
}

}  // namespace bsr
