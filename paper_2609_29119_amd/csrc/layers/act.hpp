// Activations and their derivatives, in 32 bits.
#pragma once
#include "tile.hpp"

namespace nsl {

enum Act { kNone = 0, kSilu = 1, kGelu = 2, kSigmoid = 3 };

// exp(-z). What the exponent's product loses in 32 bits is added to first
// order: off by 2e-7 relative however large |z|.
__device__ inline float exp_neg(float z) {
    constexpr float kHigh = -1.44269504f, kLow = -1.92596299e-8f;   // -log2(e)
    const float y = z * kHigh, rest = fmaf(z, kLow, fmaf(z, kHigh, -y));
    return __builtin_amdgcn_exp2f(y) * fmaf(rest, 0.69314718f, 1.f);
}

// 1 / (1 + exp(-z)), and into `other` the same of -z (their sum is 1, but the
// smaller one's last bits are not in the larger one).
__device__ inline float logistic(float z, float& other) {
    // (past 80 the correction would meet an infinity; 1 / (1 + e^80) is below what any result shows beside it)
    const float e = exp_neg(fmaxf(z, -80.f)), s = __builtin_amdgcn_rcpf(1.f + e);
    other = e * s;
    return s;
}
__device__ inline float logistic(float z) {
    float other;
    return logistic(z, other);
}

// The normal distribution's Phi(z), and exp(-z^2 / 2) into `bell`. With w =
// |z| / sqrt(2) and t = 1 / (1 + 0.3 w): erfc(w) = exp(-w^2) t Q(t), Q the
// polynomial of degree 8 that fits exp(w^2) erfc(w) / t on (0, 1] with a
// relative error of 2e-8; in 32 bits Phi is off by 4.5e-7 relative over |z| <= 9,
// also where it is small. The square's rounding is made up for as above.
__device__ inline float normal_cdf(float z, float& bell) {
    constexpr float kHigh = -0.721347520f, kLow = -9.62981497e-9f;   // -log2(e) / 2
    z = fminf(fmaxf(z, -13.f), 13.f);   // (beyond, Phi is 0 or 1 in 32 bits)
    const float s = z * z, e = fmaf(z, z, -s), y = s * kHigh, rest = fmaf(s, kLow, fmaf(s, kHigh, -y));
    bell = __builtin_amdgcn_exp2f(y) * fmaf(e, -0.5f, fmaf(rest, 0.69314718f, 1.f));
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.212132034f, 1.f));
    float q = -0.129540965f;
    q = fmaf(q, t, 0.48565802f);
    q = fmaf(q, t, -0.5124914f);
    q = fmaf(q, t, 0.54798836f);
    q = fmaf(q, t, -0.0948568061f);
    q = fmaf(q, t, 0.215024844f);
    q = fmaf(q, t, 0.148310348f);
    q = fmaf(q, t, 0.170719892f);
    q = fmaf(q, t, 0.16918768f);
    const float tail = 0.5f * bell * t * q;
    return z < 0.f ? tail : 1.f - tail;
}

template <int ACT> __device__ inline float act_of(float z) {
    float bell;
    if constexpr (ACT == kSilu) return z * logistic(z);
    if constexpr (ACT == kGelu) return z * normal_cdf(z, bell);
    if constexpr (ACT == kSigmoid) return logistic(z);
    return z;
}

// act(z), and its derivative into slope.
template <int ACT> __device__ inline float act_of(float z, float& slope) {
    if constexpr (ACT == kSilu) {
        float other;
        const float s = logistic(z, other);
        slope = fmaf(z * s, other, s);
        return z * s;
    } else if constexpr (ACT == kGelu) {
        float bell;
        const float phi = normal_cdf(z, bell);
        slope = fmaf(0.39894228f * z, bell, phi);
        return z * phi;
    } else if constexpr (ACT == kSigmoid) {
        float other;
        const float s = logistic(z, other);
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
