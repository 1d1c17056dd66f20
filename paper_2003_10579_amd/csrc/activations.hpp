// Activations of a dense layer and their slopes in fp32, for the operators that fuse them.
#pragma once
#include "ops.hpp"

namespace ssgd {

// 2^x and 1 / x by one instruction each, an error of 2^-23 of the result or less.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + exp_of(-x)); }

// Phi(x), the normal distribution's function, and e^(-x^2 / 2), which its slope is made of too: Phi(-x) = (c1 t + ... + c7 t^7) e^(-x^2 / 2) with
// t = 1 / (1 + 0.32 x) for x >= 0, the form that Hastings gave the error function (Approximations for Digital Computers, 1955).  The coefficients are a minimax fit
// of Phi(-x) e^(x^2 / 2) on 0 <= x <= 9, made with Lawson's weighted least squares: 3.4e-9 off in Phi, 2.6e-6 relative to it at x = -3 and 8e-5 at -9.  What fp32
// rounds on the way is more: 2e-7 in Phi at most, 2.4e-8 as a mean over |x| < 3.
// NEAR: the exponent's own roundings, which are x^2 units of 2^-24 of the bell, are made good (three operations; a slope in the lower tail is the difference of two such
// terms, while the function itself is small there).
template <bool NEAR = false>
__device__ __forceinline__ float normal_function(float x, float& bell) {
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.32f, __builtin_fabsf(x), 1.0f));
    const float square = x * x, exponent = square * -0.72134752f;
    bell = __builtin_amdgcn_exp2f(exponent);
    if constexpr (NEAR) {
        // what x^2 and its product with -log2(e) / 2 lost, and what the constant has not (-log2(e) / 2 is 9.63e-9 below -0.72134752 as fp32 has it)
        const float lost = __builtin_fmaf(square, -9.6298e-9f, __builtin_fmaf(square, -0.72134752f, -exponent)) + __builtin_fmaf(x, x, -square) * -0.72134752f;
        bell = __builtin_fmaf(bell, bell > 0.0f ? lost * 0.69314718f : 0.0f, bell);
    }
    float sum = 0.0436521992f;
    sum = __builtin_fmaf(t, sum, -0.230651257f);
    sum = __builtin_fmaf(t, sum, 0.388124631f);
    sum = __builtin_fmaf(t, sum, -0.144964457f);
    sum = __builtin_fmaf(t, sum, 0.205880384f);
    sum = __builtin_fmaf(t, sum, 0.108671266f);
    sum = __builtin_fmaf(t, sum, 0.129287229f);
    const float tail = t * sum * bell;
    return x < 0.0f ? tail : 1.0f - tail;
}

// Of all V values; `act` is the same in all threads.  NaN stays NaN.
template <int V>
__device__ __forceinline__ void activate(int act, float (&x)[V]) {
    if (act == SSGD_ACT_RELU) {
#pragma unroll
        for (int q = 0; q < V; ++q) x[q] = x[q] < 0.0f ? 0.0f : x[q];
    } else if (act == SSGD_ACT_GELU) {
#pragma unroll
        for (int q = 0; q < V; ++q) { float bell; x[q] *= normal_function(x[q], bell); }
    } else if (act == SSGD_ACT_SILU) {
#pragma unroll
        for (int q = 0; q < V; ++q) x[q] *= sigmoid(x[q]);
    }
}

// The activation of x and its slope there (relu's at zero: zero).
__device__ __forceinline__ void activation_and_slope(int act, float x, float& y, float& slope) {
    if (act == SSGD_ACT_RELU) {
        y = x < 0.0f ? 0.0f : x;
        slope = x > 0.0f ? 1.0f : 0.0f;
    } else if (act == SSGD_ACT_GELU) {
        float bell;
        const float phi = normal_function<true>(x, bell);
        y = x * phi;
        slope = __builtin_fmaf(x, 0.39894228f * bell, phi);
    } else if (act == SSGD_ACT_SILU) {
        const float s = sigmoid(x);
        y = x * s;
        slope = s * __builtin_fmaf(x, 1.0f - s, 1.0f);
    } else {
        y = x;
        slope = 1.0f;
    }
}

}  // namespace ssgd
