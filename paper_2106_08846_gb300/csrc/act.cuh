// Activations of the gated feed-forward block and their derivatives, in fp32, two
// values at a time.
#pragma once

#include "bsr.h"
#include "pair.cuh"

namespace bsr {

// e^(s x); FAST: the hardware's exponential. Its relative error, about 2^-21 and that of
// rounding the argument, 2^-24 |s x| / ln 2 (2^-18 at 80), is lost in a result rounded
// to bf16.
template <bool FAST>
__device__ __forceinline__ F2 exp_of(float s, F2 x) {
    if constexpr (!FAST) return each2(x, [s](float t) { return expf(s * t); });
    return each2(mul2(x, all2(s * 1.4426950408889634f)), [](float t) {
        float r;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
        return r;
    });
}
__device__ __forceinline__ float reciprocal(float t) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
    return r;
}

// 1 / (1 + e^-x)
template <bool FAST>
__device__ __forceinline__ F2 logistic(F2 x) {
    return each2(add2(exp_of<FAST>(-1.f, x), all2(1.f)), reciprocal);
}

constexpr float kGeluA = 0.7978845608028654f;   // sqrt(2 / pi)
constexpr float kGeluB = 0.044715f;

// Phi(g), the normal distribution, and e^(-g^2 / 2), from which its density follows.
// Phi(-x) = e^(-x^2 / 2) (c1 t + .. + c8 t^8), t = 1 / (1 + 0.3 x), for 0 <= x <= 16: the
// coefficients are those with the least largest error of e^(x^2 / 2) Phi(-x), taken
// relative to it and over 1 + x: 3.2e-8 (1 + x). So a tail has as many correct bits as
// the middle. With the exponential that the derivative takes anyway; where it has all of
// fp32's bits, with what the rounding of g^2 left out of it. (fp32, 1000 tokens of 768 into
// 2048: 34.3 us, with normcdff 38.9.)
template <bool FAST>
__device__ __forceinline__ F2 normal_cdf(F2 g, F2 &e) {
    const F2 x = each2(g, [](float t) { return fminf(fabsf(t), 16.f); });   // (beyond, all of it is 0 in fp32)
    const F2 s = mul2(x, x);
    e = exp_of<FAST>(-0.5f, s);
    if constexpr (!FAST) e = fma2(mul2(fma2(x, x, mul2(s, all2(-1.f))), all2(-0.5f)), e, e);
    const F2 t = each2(fma2(x, all2(0.3f), all2(1.f)), reciprocal);
    F2 q = all2(0.0362917967f);
    q = fma2(q, t, all2(-0.159551069f));
    q = fma2(q, t, all2(0.209971488f));
    q = fma2(q, t, all2(-0.0565759316f));
    q = fma2(q, t, all2(0.129835695f));
    q = fma2(q, t, all2(0.0996122584f));
    q = fma2(q, t, all2(0.12078765f));
    q = fma2(q, t, all2(0.119628094f));
    const float2 u = unpack2(g), v = unpack2(mul2(q, mul2(t, e)));
    return pack2(u.x < 0.f ? v.x : 1.f - v.x, u.y < 0.f ? v.y : 1.f - v.y);
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
    if constexpr (ACT == BSR_ACT_SILU) {
        return mul2(g, logistic<FAST>(g));
    } else if constexpr (ACT == BSR_ACT_GELU) {
        F2 e;
        return mul2(g, normal_cdf<FAST>(g, e));
    } else if constexpr (ACT == BSR_ACT_GELU_TANH) {
        return mul2(g, logistic<FAST>(gelu_2u(g)));
    } else if constexpr (ACT == BSR_ACT_RELU) {
        return relu(g);
    } else {
        return logistic<FAST>(g);
    }
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
        F2 e;
        const F2 p = normal_cdf<FAST>(g, e), density = mul2(all2(0.3989422804f), e);   // (1 / sqrt(2 pi))
        slope = fma2(g, density, p);
        return mul2(g, p);
    } else if constexpr (ACT == BSR_ACT_GELU_TANH) {
        const F2 p = logistic<FAST>(gelu_2u(g)), a = mul2(g, p);
        // (2u)'; where p is 0 or 1 any finite value does, and g^2 may overflow
        const F2 x = each2(g, [](float t) { return fminf(fabsf(t), 1e4f); });
        const F2 rise = mul2(all2(2.f * kGeluA), fma2(mul2(all2(3.f * kGeluB), x), x, one));
        slope = fma2(mul2(a, fma2(p, minus, one)), rise, p);
        return a;
    } else if constexpr (ACT == BSR_ACT_RELU) {
        slope = each2(g, [](float t) { return t > 0.f ? 1.f : (t != t ? t : 0.f); });
        return relu(g);
    } else {
        // 1 - p as e^-g p, not as a difference, of which nothing is left from g = 17 on (where
        // e^-g overflows p is 0, and so is the slope)
        const F2 e = exp_of<FAST>(-1.f, g), p = each2(add2(e, one), reciprocal);
        slope = mul2(p, each2(mul2(e, p), [](float q) { return fminf(q, 1.f); }));
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
