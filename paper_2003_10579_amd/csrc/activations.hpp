// Activations of a dense layer and their slopes in fp32, for the operators that fuse them.
#pragma once
#include "ops.hpp"

namespace ssgd {

// 2^x and 1 / x by one instruction each, within 2^-23 of the result.  e^x rounds its exponent: |x| units of 2^-24 of the result, and 0.23 |x| for its constant, so that silu is
// 7 + 1.3 |x| units of itself off at most for x < 0 (1.4e-6 at -12), 8 for x >= 0; below -87.3
// the quotient is below fp32's normal numbers and may count as zero.  (The exponent made good is five instructions more for a value.)
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + exp_of(-x)); }

// Phi(x), the normal distribution's function, and e^(-x^2 / 2), which its slope is made of too: Phi(-x) = (c1 t + ... + c8 t^8) e^(-x^2 / 2) with
// t = 1 / (1 + 0.29 x) for x >= 0, the form that Hastings gave the error function (Approximations for Digital Computers, 1955).  The coefficients are a minimax fit of
// Phi(-x) e^(x^2 / 2) on 0 <= x <= 13.4, made with Lawson's weighted least squares and rounded to fp32 one after the other, the others fitted again each time.  Its weights let the error
// grow as that of the exponent does, whose roundings are up to x^2 units of 2^-24 of the bell: the fit is 0.06 + 0.56 x^2 units of 2^-24 of Phi(-x) off at most, 2.8e-9 of all, a half at
// zero, and makes good what the exponent's constant has not.  With all that fp32 rounds Phi is 16 + 1.6 x^2 units of itself off at most for x < 0 (1.0e-6 at -3, 4.4e-6 at -9), 3.2e-7 for
// x >= 0; past -13.2 the bell is below fp32's normal numbers and counts as zero.  (Seven coefficients are 3e-6 off at -3 and 8e-5 at -9, or, fitted to the tail, a fifth more near zero, for
// 1 us of 412 that 8192^3 with gelu takes; the exponent's roundings made good, for 16 units of itself everywhere, 12 us more.)
// NEAR: those roundings are made good (a slope in the lower tail has x times the bell, while the function itself is small there).
template <bool NEAR = false>
__device__ __forceinline__ float normal_function(float x, float& bell) {
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.29f, __builtin_fabsf(x), 1.0f));
    const float square = x * x, exponent = square * -0.72134752f;
    bell = __builtin_amdgcn_exp2f(exponent);
    if constexpr (NEAR) {
        // what x^2 and its product with -log2(e) / 2 lost
        const float lost = __builtin_fmaf(square, -0.72134752f, -exponent) + __builtin_fmaf(x, x, -square) * -0.72134752f;
        bell = __builtin_fmaf(bell, bell > 0.0f ? lost * 0.69314718f : 0.0f, bell);
    }
    float sum = 0.0373081192f;
    sum = __builtin_fmaf(t, sum, -0.182383567f);
    sum = __builtin_fmaf(t, sum, 0.283218861f);
    sum = __builtin_fmaf(t, sum, -0.123536706f);
    sum = __builtin_fmaf(t, sum, 0.165661201f);
    sum = __builtin_fmaf(t, sum, 0.0856717303f);
    sum = __builtin_fmaf(t, sum, 0.11853338f);
    sum = __builtin_fmaf(t, sum, 0.115526982f);
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
