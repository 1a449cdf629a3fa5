// Activations and their derivatives, in 32 bits.
#pragma once
#include "tile.hpp"

namespace nsl {

enum Act { kNone = 0, kSilu = 1, kGelu = 2, kSigmoid = 3 };

// EXACT, for 32-bit results, makes up for what an exponent's product loses in
// 32 bits; for 16-bit results that is left out (1e-6 at |z| = 10).

// At infinite arguments, and where a product passes 32 bits, results are the
// limits: 0 wins over what it is multiplied by, and an exponent's argument is
// held where the result no longer changes. A NaN stays one. (v_mul_legacy_f32 is
// such a product, so that most of it costs nothing.)
__device__ __attribute__((const, noconvergent)) float zero_wins(float x, float y) __asm("llvm.amdgcn.fmul.legacy");
__device__ inline float at_most(float x, float most) { return __builtin_elementwise_minimum(x, most); }

// exp(-z). EXACT: what the exponent's product loses in 32 bits is added to
// first order: off by 2e-7 relative however large |z|.
template <bool EXACT> __device__ inline float exp_neg(float z) {
    constexpr float kHigh = -1.44269504f, kLow = -1.92596299e-8f;   // -log2(e)
    if (!EXACT) return __builtin_amdgcn_exp2f(z * kHigh);
    z = at_most(__builtin_elementwise_maximum(z, -128.f), 128.f);   // (infinite, 0)
    const float y = z * kHigh;
    const float rest = fmaf(z, kLow, fmaf(z, kHigh, -y));
    return __builtin_amdgcn_exp2f(y) * fmaf(rest, 0.69314718f, 1.f);
}

// 1 / (1 + exp(-z)), and into `other` the same of -z: their sum is 1, but the
// smaller one's last bits are not in the larger one (and past 88 exp(-z) is
// infinite where z is negative).
template <bool EXACT> __device__ inline float logistic(float z, float& other) {
    const float e = exp_neg<EXACT>(z), s = __builtin_amdgcn_rcpf(1.f + e);
    other = z < 0.f ? 1.f - s : e * s;
    return s;
}
template <bool EXACT> __device__ inline float logistic(float z) { return __builtin_amdgcn_rcpf(1.f + exp_neg<EXACT>(z)); }

// The normal distribution's Phi(z), and exp(-z^2 / 2) into `bell`. With w =
// |z| / sqrt(2) and t = 1 / (1 + 0.33 w): erfc(w) = exp(-w^2) t Q(t), Q the
// polynomial of degree 7 that fits exp(w^2) erfc(w) / t on (0, 1], by least
// squares with weights that even out the largest relative errors: 1e-7. EXACT:
// Phi is off by 5e-7 relative over |z| <= 9, also where it is small.
template <bool EXACT> __device__ inline float normal_cdf(float z, float& bell) {
    constexpr float kHigh = -0.721347520f, kLow = -9.62981497e-9f;   // -log2(e) / 2
    const float far = at_most(fabsf(z), 16.f);   // (exp(-128) is 0 in 32 bits)
    const float s = far * far, y = s * kHigh;
    bell = __builtin_amdgcn_exp2f(y);
    if (EXACT) {
        const float e = fmaf(far, far, -s), rest = fmaf(s, kLow, fmaf(s, kHigh, -y));
        bell *= fmaf(e, -0.5f, fmaf(rest, 0.69314718f, 1.f));
    }
    const float t = __builtin_amdgcn_rcpf(fmaf(far, 0.23334524f, 1.f));
    float q = fmaf(-0.134988993f, t, 0.458738714f);
    q = fmaf(q, t, -0.348531395f);
    q = fmaf(q, t, 0.406038553f);
    q = fmaf(q, t, 0.0485620759f);
    q = fmaf(q, t, 0.200800955f);
    q = fmaf(q, t, 0.183027253f);
    q = fmaf(q, t, 0.186352849f) * t;
    const float tail = 0.5f * bell * q;
    return z < 0.f ? tail : 1.f - tail;
}

template <int ACT, bool EXACT> __device__ inline float act_of(float z) {
    float bell;
    if constexpr (ACT == kSilu) return zero_wins(z, logistic<EXACT>(z));
    if constexpr (ACT == kGelu) return zero_wins(z, normal_cdf<EXACT>(z, bell));
    if constexpr (ACT == kSigmoid) return logistic<EXACT>(z);
    return z;
}

// act(z), and its derivative into slope.
template <int ACT, bool EXACT> __device__ inline float act_of(float z, float& slope) {
    if constexpr (ACT == kSilu) {
        float other;
        const float s = logistic<EXACT>(z, other), value = zero_wins(z, s);
        slope = zero_wins(value, other) + s;
        return value;
    } else if constexpr (ACT == kGelu) {
        float bell;
        const float phi = normal_cdf<EXACT>(z, bell);
        slope = zero_wins(0.39894228f * z, bell) + phi;
        return zero_wins(z, phi);
    } else if constexpr (ACT == kSigmoid) {
        float other;
        const float s = logistic<EXACT>(z, other);
        slope = s * other;
        return s;
    } else {
        slope = 1.f;
        return z;
    }
}

// f(integral constant of the activation)
template <class F> __device__ __attribute__((always_inline)) inline void by_act(int act, F f) {
    switch (act) {
        case kSilu: return f(std::integral_constant<int, kSilu>());
        case kGelu: return f(std::integral_constant<int, kGelu>());
        case kSigmoid: return f(std::integral_constant<int, kSigmoid>());
        default: return f(std::integral_constant<int, kNone>());
    }
}

}  // namespace nsl
