// Activations of the update with an epilogue, and their slopes, in fp32.
#pragma once

#include <type_traits>

#include "internal.h"

namespace gnn {
namespace act {

// exp(x) = 2^(x log2 e): one multiplication and the hardware's exponential.
// Its relative error is about 2^-24 (|x| + 2): a probability or a tail far
// from its centre loses digits that its sum or its distance from 0 has lost
// already.
__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }
__device__ __forceinline__ float fast_rcp(float x) { return __builtin_amdgcn_rcpf(x); }

// s = 1 / (1 + exp(-x)) and w = s (1 - s), both from exp(-|x|): neither
// overflows, and 1 - s is never a difference (as one it is off by 2^-22 for
// positive x, which a slope multiplies by z).
__device__ __forceinline__ float sigmoid(float x, float *w) {
    const float e = fast_exp(-fabsf(x)), r = fast_rcp(1.f + e), q = e * r;
    *w = q * r;
    return x < 0.f ? q : r;
}
__device__ __forceinline__ float sigmoid(float x) { return fast_rcp(1.f + fast_exp(-x)); }

// Phi(z), the normal distribution's, and e = exp(-z^2 / 2): Abramowitz and
// Stegun 7.1.26 (erfc x = t (a1 + t (a2 + ...)) exp(-x^2), t = 1 / (1 + p x),
// within 1.5e-7 absolute, so Phi within 7.5e-8), whose exponential the slope
// of z Phi(z) needs anyway.  A dozen instructions; the library's erff takes
// three times as many, and an epilogue of 27 million values 20 us of them.
__device__ __forceinline__ float normal_cdf(float z, float *e) {
    const float x = fabsf(z) * 0.70710678118654752f;
    const float t = fast_rcp(fmaf(0.3275911f, x, 1.f));
    float p = fmaf(1.061405429f, t, -1.453152027f);
    p = fmaf(p, t, 1.421413741f);
    p = fmaf(p, t, -0.284496736f);
    p = fmaf(p, t, 0.254829592f);
    *e = fast_exp(-x * x);
    const float tail = 0.5f * p * t * *e;
    return z < 0.f ? tail : 1.f - tail;
}

// z (1 + tanh u) / 2 = z sigmoid(2 u), 2 u = z (c0 + c1 z^2)
constexpr float kTanh0 = 1.5957691216057308f, kTanh1 = 0.071354816272600247f;

template <int ACT> __device__ __forceinline__ float apply(float z) {
    if constexpr (ACT == GNN_ACT_RELU) return z > 0.f ? z : 0.f;
    if constexpr (ACT == GNN_ACT_GELU) {
        float e;
        return z * normal_cdf(z, &e);
    }
    if constexpr (ACT == GNN_ACT_GELU_TANH) return z * sigmoid(z * fmaf(kTanh1, z * z, kTanh0));
    if constexpr (ACT == GNN_ACT_SILU) return z * sigmoid(z);
    return z;
}

template <int ACT> __device__ __forceinline__ float slope(float z) {
    if constexpr (ACT == GNN_ACT_RELU) return z > 0.f ? 1.f : 0.f;
    if constexpr (ACT == GNN_ACT_GELU) {
        float e;
        const float p = normal_cdf(z, &e);
        return fmaf(z * 0.39894228040143268f, e, p);
    }
    if constexpr (ACT == GNN_ACT_GELU_TANH) {
        float w;
        const float s = sigmoid(z * fmaf(kTanh1, z * z, kTanh0), &w);
        // far out w is 0 and the other factor may be infinite
        return w == 0.f ? s : fmaf(z * w, fmaf(3.f * kTanh1, z * z, kTanh0), s);
    }
    if constexpr (ACT == GNN_ACT_SILU) {
        float w;
        const float s = sigmoid(z, &w);
        return fmaf(z, w, s);
    }
    return 1.f;
}

// go with the activation as a compile-time value (host side).
template <class F> void with(int code, F &&go) {
    if (code == GNN_ACT_RELU) go(std::integral_constant<int, GNN_ACT_RELU>{});
    else if (code == GNN_ACT_GELU) go(std::integral_constant<int, GNN_ACT_GELU>{});
    else if (code == GNN_ACT_GELU_TANH) go(std::integral_constant<int, GNN_ACT_GELU_TANH>{});
    else if (code == GNN_ACT_SILU) go(std::integral_constant<int, GNN_ACT_SILU>{});
    else go(std::integral_constant<int, GNN_ACT_NONE>{});
}

}  // namespace act
}  // namespace gnn
