// The activations of the feed-forward operators and their derivatives, in fp32.
#pragma once

#include <hip/hip_runtime.h>

#include "feedforward.h"

namespace spingtp {
namespace {

// exp(x), off by about 2^-23: the hardware's 2^t of t = x log2 e, and the rounding of t put back.  Where t is
// infinite that rounding is no number, nor is its sum with an infinite 2^t: 2^t stands as it is.
__device__ __forceinline__ float exp_of(float x) {
    const float t = x * 1.44269504088896f;
    const float rest = fmaf(x, 1.44269504088896f, -t) + x * 1.92596299e-8f;  // log2 e in two parts
    const float e = __builtin_amdgcn_exp2f(t);
    const float near = fmaf(e, rest * 0.69314718f, e);
    return near == near ? near : e;
}
// The same for x <= 0, as exact, in six operations in place of eight
__device__ __forceinline__ float exp_below(float x) {
    x = fmaxf(x, -256.f);  // zero from here on; an infinite x has no rest
    const float t = x * 1.44269504088896f;
    const float rest = fmaf(t, 1.904654300e-9f, fmaf(t, -0.693147182464599609f, x));  // x - t ln 2, ln 2 in two parts
    const float e = __builtin_amdgcn_exp2f(t);
    return fmaf(e, rest, e);
}
// The normal distribution's Phi(g), and `bell` e^(-g^2 / 2): e^(a^2 / 2) Phi(-a), a = |g|, is a polynomial in
// t = 1 / (1 + 0.35 a) times t, fitted for the least largest relative error over a up to 14.5 (beyond that Phi(-a) is
// below fp32's range); off by 6 2^-24 and g^2 / 2 of them by the exponent's rounding.  (1 + erf cancels below zero:
// x Phi(x) is off by 4 % at -5 and zero at -6.  The library's erfc is as exact: 20,000 x 128 x 512 forward 22.0 us
// against 18.7.)
template <bool BELOW = false>
__device__ __forceinline__ float normal(float g, float& bell) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.35f, fabsf(g), 1.f));
    bell = BELOW ? exp_below(-0.5f * g * g) : exp_of(-0.5f * g * g);
    float p = fmaf(-0.0291580297f, t, 0.144031614f);
    p = fmaf(p, t, -0.255840391f);
    p = fmaf(p, t, 0.159321249f);
    p = fmaf(p, t, -0.023213394f);
    p = fmaf(p, t, 0.105552927f);
    p = fmaf(p, t, 0.119821183f);
    p = fmaf(p, t, 0.139863536f);
    p = fmaf(p, t, 0.139621302f);
    if constexpr (BELOW) {  // nothing left to contract: the same bits in every kernel
        const float part = p * t;
        return g > 0.f ? fmaf(-part, bell, 1.f) : part * bell;
    }
    const float below = p * t * bell;
    return g > 0.f ? 1.f - below : below;
}
// act(g) and its derivative; the reciprocals are the hardware's, off by 2^-23
template <int ACT>
__device__ __forceinline__ float act(float g) {
    if constexpr (ACT == kSilu) return g * __builtin_amdgcn_rcpf(1.f + exp_of(-g));
    float bell;
    return g * normal(g, bell);
}
template <int ACT>
__device__ __forceinline__ void act_grad(float g, float& a, float& d) {
    if constexpr (ACT == kSilu) {
        const float t = __builtin_amdgcn_rcpf(1.f + exp_of(-g));
        a = g * t;
        d = t * (1.f + g * (1.f - t));
    } else {
        float bell;
        const float p = normal(g, bell);
        a = g * p;
        d = p + g * 0.39894228040143268f * bell;
    }
}
// The derivative alone, at a bf16 g, as exact as act_grad's.  silu's exponential in four operations in place of eight: g
// times the 16 leading bits of log2 e is exact, and the rest of it, at most 2^-11 of the result, goes on by its first
// order.  (An exponential that leaves out its argument's rounding is off by |g| 2^-23 and saves 1 %: all gradients of
// 100,000 x 512 by 128 97.5 us against 98.4 with silu, 108.1 against 109.2 with gelu.)
template <int ACT>
__device__ __forceinline__ float slope(float g) {
    if constexpr (ACT == kSilu) {
        const float e = __builtin_amdgcn_exp2f(g * -1.44268798828125f);
        const float t = __builtin_amdgcn_rcpf(1.f + fmaf(e, g * -4.88849507e-6f, e));
        return t * fmaf(g, 1.f - t, 1.f);
    }
    float bell;
    const float p = normal<true>(g, bell);
    return fmaf(g * 0.39894228040143268f, bell, p);
}

}  // namespace
}  // namespace spingtp
