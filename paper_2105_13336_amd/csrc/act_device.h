// Activations and their derivatives: GELU in both forms, SiLU.
#pragma once

#include "ops_device.h"

namespace tensile {

namespace {

// GELU in 16 bits: from the distribution function to 1e-7, absolutely.  A result's rounding is larger, but for x < -5.5 in bf16, where the result is below 2e-7
// and off by up to 1 %.  (The forms for 32 bits further down are 10 to 20 % slower where the data lie in the cache: 8192 x 3072 f16
// forward 17.5 and 21.4 us, bf16 backward with a checkpoint 24.5 and 27.3.)
// The normal distribution's tail by Abramowitz and Stegun 7.1.26 (error below 7.5e-8) from one exponential and one reciprocal:
// 1 - Phi(|x|) = t*(a1 + ... + a5 t^4)*exp(-x^2/2)/2, t = 1/(1 + p|x|/sqrt 2).  e: exp(-x^2/2).
__device__ __forceinline__ float normal_tail(float x, float &e) {
    e = __builtin_amdgcn_exp2f(-0.72134752044448170f * x * x);
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.23164189f, __builtin_fabsf(x), 1.0f));
    float s = __builtin_fmaf(0.5307027145f, t, -0.7265760135f);
    s = __builtin_fmaf(s, t, 0.7107068705f);
    s = __builtin_fmaf(s, t, -0.142248368f);
    s = __builtin_fmaf(s, t, 0.127414796f);
    return s * t * e;
}
// The tanh form: (1 + tanh u)/2 = 1/(1 + exp(-2u)).
__device__ __forceinline__ float tanh_cdf(float x, float x2) {
    const float u2 = x * __builtin_fmaf(0.071354816272f, x2, 1.5957691216f);            // 2u
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * u2));
}
// (from |x| = 100 on the distribution function is 0 or 1: no overflow on the way)
__device__ __forceinline__ float capped_square(float x) { return __builtin_amdgcn_fmed3f(x * x, 0.0f, 1e4f); }

// x*P(x) = max(x, 0) - |x|*(1 - P(|x|)), in which neither a small tail nor a small x cancels.  x_capped is x, or 100 where that is larger: inf
// stays out of the product, while -inf * 0 is NaN.  (By hand: fmin and fmax cost one and two more, to quiet a NaN; `tail` brings it in.)
__device__ __forceinline__ float capped(float x) {
    float least;
    asm("v_min_f32 %0, 0x42c80000, %1" : "=v"(least) : "v"(x));
    return least;
}
__device__ __forceinline__ float from_tail(float x, float x_capped, float tail) {
    float above;
    asm("v_max_f32 %0, 0, %1" : "=v"(above) : "v"(x));
    return __builtin_fmaf(-__builtin_fabsf(x_capped), tail, above);
}

// GELU in 32 bits, to a few units of the result (the product with a distribution function that is within 1e-7 absolutely is not, where x is below
// 0 or large).  The kernels wait for memory, so that it costs little: 8192 x 8192 94 us forward and 108 backward, 94 and 105 by the form above.
// Relative norm of the error, this and that (elementary operations in 32 bits: 3.3e-8, 3.8e-8, 3.2e-8, 5.3e-8): y 2.4e-8 and 7.0e-8, dx 3.5e-8 and
// 1.1e-7; tanh y 2.4e-8 and 4.0e-8, dx 3.6e-8 and 9.6e-8.
// 1 - Phi(|x|) = R*exp(-x^2/2): R falls slowly from 1/2, a polynomial in v = |x|/(1 + 0.35|x|), whose coefficients are fitted to the least
// relative error for |x| <= 14.5 (3.1e-8; beyond, exp(-x^2/2) is 0 in 32 bits).  The 1/2 is exact and added last: a small |x| keeps all
// its bits.  capped: x, no larger than 100.
struct Normal {
    float r, e;                       // R and exp(-x^2/2)
};
__device__ __forceinline__ Normal normal(float x, float capped) {
    const float a = __builtin_fabsf(capped), v = a * __builtin_amdgcn_rcpf(__builtin_fmaf(0.35f, a, 1.0f));
    float s = __builtin_fmaf(2.196936572e-06f, v, -2.552021214e-05f);
    s = __builtin_fmaf(s, v, 9.320835806e-05f);
    s = __builtin_fmaf(s, v, -7.410841436e-05f);
    s = __builtin_fmaf(s, v, 0.0002308475395f);
    s = __builtin_fmaf(s, v, -0.002482980739f);
    s = __builtin_fmaf(s, v, -0.006802681071f);
    s = __builtin_fmaf(s, v, 0.1103606986f);
    s = __builtin_fmaf(s, v, -0.3989416219f);
    return {__builtin_fmaf(s, v, 0.5f), __builtin_amdgcn_exp2f(-0.72134752044448170f * x * x)};
}
// The tanh form's tail: E*t with E = exp(-2|u|) <= 1 and t = 1/(1 + E).
struct Logistic {
    float tail, t;
};
__device__ __forceinline__ Logistic logistic(float x, float x2) {
    const float e = __builtin_amdgcn_exp2f(-__builtin_fabsf(x) * __builtin_fmaf(0.10294324f, x2, 2.3022082f));   // -2|u|/ln 2
    const float t = __builtin_amdgcn_rcpf(1.0f + e);
    return {e * t, t};
}

template <typename T>
constexpr bool kRoundsTo32 = sizeof(T) == 4;

template <bool kTanh, bool kTo32>
__device__ __forceinline__ float gelu(float x) {
    if constexpr (kTanh) {
        if constexpr (kTo32) return from_tail(x, capped(x), logistic(x, capped_square(x)).tail);
        return x * tanh_cdf(x, capped_square(x));
    } else {
        if constexpr (kTo32) {
            const float c = capped(x);
            const Normal n = normal(x, c);
            return from_tail(x, c, n.r * n.e);
        }
        float e;
        return from_tail(x, capped(x), normal_tail(x, e));
    }
}
// y and dy/dx = P + x*P', P the distribution function.  To 32 bits P is the tail where x is negative and 1 - tail elsewhere, and the tail is
// taken out of all but the 1, so that one rounding is the last: e*(x/sqrt(2 pi) -+ R), and of the tanh form tail*(x*t*d(2u)/dx -+ 1).
template <bool kTanh, bool kTo32>
__device__ __forceinline__ float gelu_slope(float x, float &y) {
    if constexpr (kTo32) {
        const bool negative = as_u32(x) >> 31;
        const float one = negative ? 0.0f : 1.0f;
        if constexpr (kTanh) {
            const float x2 = capped_square(x);
            const Logistic l = logistic(x, x2);
            y = from_tail(x, x, l.tail);                    // (a checkpoint holds no infinity: a tail of 0 wins over any x)
            const float m = __builtin_amdgcn_fmed3f(x, -100.0f, 100.0f) * l.t;
            return __builtin_fmaf(l.tail, __builtin_fmaf(m, __builtin_fmaf(0.214064448816f, x2, 1.5957691216f), negative ? 1.0f : -1.0f), one);
        } else {
            const float c = __builtin_amdgcn_fmed3f(x, -100.0f, 100.0f);
            const Normal n = normal(x, c);
            y = from_tail(x, c, n.r * n.e);
            return __builtin_fmaf(n.e, __builtin_fmaf(c, 0.39894228040143268f, negative ? n.r : -n.r), one);
        }
    } else if constexpr (kTanh) {
        const float x2 = capped_square(x), p = tanh_cdf(x, x2);
        const float dp = p * (1.0f - p) * __builtin_fmaf(0.214064448816f, x2, 1.5957691216f);   // p(1-p) * d(2u)/dx
        y = x * p;
        return __builtin_fmaf(x, dp, p);
    } else {
        float e;
        const float tail = normal_tail(x, e), p = x < 0.0f ? tail : 1.0f - tail;
        y = x * p;
        return __builtin_fmaf(x, 0.39894228040143268f * e, p);
    }
}

// SiLU, x*P with the logistic function P(x) = 1/(1 + exp(-x)).  E = exp(-|x|) <= 1 neither overflows nor cancels: of P and 1 - P one is
// t = 1/(1 + E), the other E*t.  (x*log2 e is rounded before the exponential: |x|/2 units of E; -inf * 0 is NaN, as in GELU.)
__device__ __forceinline__ float silu_slope(float x, float &y) {
    const float e = __builtin_amdgcn_exp2f(-1.4426950408889634f * __builtin_fabsf(x)), t = __builtin_amdgcn_rcpf(1.0f + e), r = e * t;
    const float p = x < 0.0f ? r : t, rest = x < 0.0f ? t : r;
    y = x * p;
    return p * __builtin_fmaf(x, rest, 1.0f);
}
// (In 16 bits without the two selections: exp(-x) is infinite from x = -88.7 on, where the result, below 1e-36, becomes 0.)
template <bool kTo32>
__device__ __forceinline__ float silu(float x) {
    if constexpr (kTo32) {
        const float e = __builtin_amdgcn_exp2f(-1.4426950408889634f * __builtin_fabsf(x)), t = __builtin_amdgcn_rcpf(1.0f + e);
        return x * (x < 0.0f ? e * t : t);
    }
    return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * x));
}

// The activations that a gated layer may have, in the order of their numbers in tensile.h.
struct Silu {
    template <bool kTo32>
    static __device__ __forceinline__ float value(float x) { return silu<kTo32>(x); }
    template <bool kTo32>
    static __device__ __forceinline__ float slope(float x, float &y) { return silu_slope(x, y); }
};
template <bool kTanh>
struct Gelu {
    template <bool kTo32>
    static __device__ __forceinline__ float value(float x) { return gelu<kTanh, kTo32>(x); }
    template <bool kTo32>
    static __device__ __forceinline__ float slope(float x, float &y) { return gelu_slope<kTanh, kTo32>(x, y); }
};

}  // namespace

}  // namespace tensile
