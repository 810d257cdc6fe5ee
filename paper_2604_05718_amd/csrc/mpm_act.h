// Activations and their slopes, float32, shared by the kernels that end in one.
#pragma once

#include <hip/hip_runtime.h>

#include "mpm_launch.h"

namespace mpm {

__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }

// The normal distribution's integral up to z, half of erfc(-z / sqrt 2). PRECISE: the library's erfc. Otherwise
// formula 7.1.26 of Abramowitz and Stegun's Handbook of Mathematical Functions for erfc (absolute error
// below 1.5e-7), a reciprocal, an exponential and six multiply-adds: for results rounded to bfloat16.
template <bool PRECISE>
__device__ __forceinline__ float normal_integral(float z)
{
    if constexpr (PRECISE) return 0.5f * erfcf(z * -0.70710678118654752f);
    const float u = fabsf(z) * 0.70710678118654752f;
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, u, 1.0f));
    float p = fmaf(1.061405429f, t, -1.453152027f);
    p = fmaf(p, t, 1.421413741f);
    p = fmaf(p, t, -0.284496736f);
    p = fmaf(p, t, 0.254829592f);
    const float tail = 0.5f * p * t * __expf(-u * u);
    return z < 0.0f ? tail : 1.0f - tail;
}

// z times the normal distribution's integral, as z / (1 + e^-l) with l the logarithm of the integral's odds, an odd
// function of z close to a polynomial of seventh degree. The coefficients minimise the largest error of l over |z| <= 6
// where the result is 10^-4 or more, 0.00104: a quarter of bfloat16's half step for negative z, less for positive.
// Two thirds of the instructions of the integral itself: the product of 45920 x 4096 x 1024 with it 303 us
// against 330.
__device__ __forceinline__ float gelu_bf16(float z)
{
    constexpr float kLog2e = 1.4426950408889634f;
    const float u = z * z;
    float p = fmaf(-7.25138e-6f * kLog2e, u, 9.3992063e-4f * kLog2e);
    p = fmaf(p, u, -7.55007635e-2f * kLog2e);
    p = fmaf(p, u, -1.59312151f * kLog2e);
    return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(p * z));
}

// (max() would drop a NaN)
template <int ACT, bool PRECISE>
__device__ __forceinline__ float activate(float z)
{
    if constexpr (ACT == kActGelu && !PRECISE) return gelu_bf16(z);
    if constexpr (ACT == kActRelu) return z < 0.0f ? 0.0f : z;
    if constexpr (ACT == kActSilu) return z * sigmoid(z);
    if constexpr (ACT == kActGelu) return z * normal_integral<PRECISE>(z);
    return z;
}

template <int ACT, bool PRECISE>
__device__ __forceinline__ float activation_slope(float z)
{
    if constexpr (ACT == kActRelu) return z > 0.0f ? 1.0f : 0.0f;
    if constexpr (ACT == kActSilu) {
        const float s = sigmoid(z);
        return s * fmaf(z, 1.0f - s, 1.0f);
    }
    if constexpr (ACT == kActGelu)
        return fmaf(z * 0.39894228040143268f, __expf(-0.5f * z * z), normal_integral<PRECISE>(z));
    return 1.0f;
}

}  // namespace mpm
