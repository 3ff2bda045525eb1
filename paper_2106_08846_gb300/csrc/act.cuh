// Activations of the gated feed-forward block and their derivatives, in fp32, two
// values at a time.
#pragma once

#include "bsr.h"
#include "pair.cuh"

namespace bsr {

// 1 / (1 + e^-x); FAST: the hardware's exponential, whose relative error of about
// 2^-21 is lost in a result rounded to bf16.
template <bool FAST>
__device__ __forceinline__ F2 logistic(F2 x) {
    F2 e;
    if constexpr (FAST) {
        e = each2(mul2(x, all2(-1.4426950408889634f)), [](float t) {
            float r;
            asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
            return r;
        });
    } else {
        e = each2(x, [](float t) { return expf(-t); });
    }
    return each2(add2(e, all2(1.f)), [](float t) {
        float r;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
        return r;
    });
}

constexpr float kGeluA = 0.7978845608028654f;   // sqrt(2 / pi)
constexpr float kGeluB = 0.044715f;

// Phi(g), the normal distribution
template <bool FAST>
__device__ __forceinline__ F2 normal_cdf(F2 g) {
    return each2(g, [](float t) { return FAST ? fmaf(0.5f, erff(0.70710678f * t), 0.5f) : normcdff(t); });
}
// the tanh form of GELU is g / (1 + e^-2u), which is the same; 2u
__device__ __forceinline__ F2 gelu_2u(F2 g) {
    return mul2(mul2(all2(2.f * kGeluA), g), fma2(mul2(all2(kGeluB), g), g, all2(1.f)));
}
__device__ __forceinline__ F2 relu(F2 g) {
    return each2(g, [](float t) { return t > 0.f ? t : (t != t ? t : 0.f); });
}

template <int ACT, bool FAST>
__device__ __forceinline__ F2 activate(F2 g) {
    if constexpr (ACT == BSR_ACT_SILU) return mul2(g, logistic<FAST>(g));
    else if constexpr (ACT == BSR_ACT_GELU) return mul2(g, normal_cdf<FAST>(g));
    else if constexpr (ACT == BSR_ACT_GELU_TANH) return mul2(g, logistic<FAST>(gelu_2u(g)));
    else if constexpr (ACT == BSR_ACT_RELU) return relu(g);
    else return logistic<FAST>(g);
}

// act(g), and act'(g) in `slope`.
template <int ACT, bool FAST>
__device__ __forceinline__ F2 activate_slope(F2 g, F2 &slope) {
    const F2 one = all2(1.f), minus = all2(-1.f);
    if constexpr (ACT == BSR_ACT_SILU) {
        const F2 p = logistic<FAST>(g);
        slope = mul2(p, fma2(g, fma2(p, minus, one), one));
        return mul2(g, p);
    } else if constexpr (ACT == BSR_ACT_GELU) {
        const F2 p = normal_cdf<FAST>(g);
        const F2 density = each2(mul2(mul2(all2(-0.5f), g), g), [](float t) { return 0.3989422804f * (FAST ? __expf(t) : expf(t)); });
        slope = fma2(g, density, p);
        return mul2(g, p);
    } else if constexpr (ACT == BSR_ACT_GELU_TANH) {
        const F2 p = logistic<FAST>(gelu_2u(g)), a = mul2(g, p);
        const F2 rise = mul2(all2(2.f * kGeluA), fma2(mul2(all2(3.f * kGeluB), g), g, one));
        slope = fma2(mul2(a, fma2(p, minus, one)), rise, p);
        return a;
    } else if constexpr (ACT == BSR_ACT_RELU) {
        slope = each2(g, [](float t) { return t > 0.f ? 1.f : (t != t ? t : 0.f); });
        return relu(g);
    } else {
        const F2 p = logistic<FAST>(g);
        slope = mul2(p, fma2(p, minus, one));
        return p;
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
