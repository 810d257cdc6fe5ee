// Activations and their slopes, float32, shared by the kernels that end in one.
#pragma once

#include <hip/hip_runtime.h>

#include "mpm_launch.h"

namespace mpm {

__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }

// The normal distribution's integral up to z, half of erfc(-z / sqrt 2). PRECISE: the library's erfc. Otherwise, for results
// rounded to bfloat16, that of -|z| as two to the power of a polynomial of ninth degree in |z|, and for positive z one less
// it: an exponential and nine multiply-adds. The coefficients minimise the largest relative error over |z| <= 11, 2^-17, a
// five-hundredth of bfloat16's half step; rounding the exponent adds at most 4 z^2 2^-24. From there the polynomial falls on,
// off by 0.2% where the integral leaves the normal numbers (z = -13.2), below which it may become 0.
template <bool PRECISE>
__device__ __forceinline__ float normal_integral(float z)
{
    if constexpr (PRECISE) return 0.5f * erfcf(z * -0.70710678118654752f);
    const float a = fabsf(z);
    float p = fmaf(-2.5579749429738285e-9f, a, 1.7468622104388487e-7f);
    p = fmaf(p, a, -5.276353022054536e-6f);
    p = fmaf(p, a, 9.349359606858343e-5f);
    p = fmaf(p, a, -1.0905652306973934e-3f);
    p = fmaf(p, a, 8.957162499427795e-3f);
    p = fmaf(p, a, -5.464214086532593e-2f);
    p = fmaf(p, a, -4.579631984233856e-1f);
    p = fmaf(p, a, -1.1513879299163818f);
    const float tail = __builtin_amdgcn_exp2f(fmaf(p, a, -9.9998939037323e-1f));
    return z < 0.0f ? tail : 1.0f - tail;
}

// (max() would drop a NaN)
template <int ACT, bool PRECISE>
__device__ __forceinline__ float activate(float z)
{
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
