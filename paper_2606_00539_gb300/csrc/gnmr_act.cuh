// The activations of the gated blocks, in fp32.
#pragma once

#include <cuda_runtime.h>

#include "gnmr.h"

namespace gnmr_act {

// 1 / (1 + exp(-a)).  exp(-a) past fp32 is infinite and the quotient 0.  The approximate functions
// are 2 to 3 units of fp32's last place off at the magnitudes where the result is not next to
// nothing, which the 16-bit outputs do not see.
__device__ __forceinline__ float sigmoid(float a) { return __fdividef(1.0f, 1.0f + __expf(-a)); }

template <int kAct> __device__ __forceinline__ float activated(float a)
{
    if (kAct == GNMR_ACT_SILU)
        return a * sigmoid(a);
    return a * (0.5f * erfcf(a * -0.70710678f));             // erfc: 1 + erf would cancel below zero
}

// act(a), and its derivative.
template <int kAct> __device__ __forceinline__ float activated(float a, float &slope)
{
    if (kAct == GNMR_ACT_SILU) {
        const float s = sigmoid(a);
        slope = s * (1.0f + a * (1.0f - s));
        return a * s;
    }
    const float p = 0.5f * erfcf(a * -0.70710678f);
    slope = p + a * (0.39894228f * __expf(-0.5f * a * a));
    return a * p;
}

}  // namespace gnmr_act
