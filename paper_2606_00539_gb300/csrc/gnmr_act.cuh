// The activations of the gated blocks, in fp32.
#pragma once

#include <cuda_runtime.h>

#include "gnmr.h"

namespace gnmr_act {

// 1 / (1 + exp(-a)).  exp(-a) past fp32 is infinite and the quotient 0.  The approximate functions
// are 2 to 3 units of fp32's last place off at the magnitudes where the result is not next to
// nothing, which the 16-bit outputs do not see.
__device__ __forceinline__ float sigmoid(float a) { return __fdividef(1.0f, 1.0f + __expf(-a)); }

// The normal distribution function P(a) = erfc(-a / sqrt 2) / 2, and exp(-a^2 / 2).  Hastings' form (Abramowitz and
// Stegun 7.1.26): P(-|a|) = exp(-a^2 / 2) t Q(t), t = 1 / (1 + 0.375 |a|), with a Q of degree 8 fitted to
// 64-bit values (least squares of the relative error at 4,000 Chebyshev nodes of t in (0, 1], weights raised where it is large; 0.375 from
// a scan): 2.5e-7 relative over the whole range, and with fp32's roundings less than half of (8 + 1.2 |a| + a^2) 2^-23.
// (1 + erf would cancel below zero.  On the grid of that time erfcf took the gradient of 49,152 x 1408 168 us and this 123; now 105.)
__device__ __forceinline__ float normal(float a, float &bell)
{
    const float m = fabsf(a), t = __fdividef(1.0f, fmaf(0.375f, m, 1.0f));
    bell = __expf(-0.5f * a * a);
    float q = -0.03291367366909981f;
    q = fmaf(q, t, 0.1368897706270218f);
    q = fmaf(q, t, -0.18653617799282074f);
    q = fmaf(q, t, 0.050644271075725555f);
    q = fmaf(q, t, 0.015622680075466633f);
    q = fmaf(q, t, 0.0886395052075386f);
    q = fmaf(q, t, 0.12844553589820862f);
    q = fmaf(q, t, 0.14960458874702454f);
    q = fmaf(q, t, 0.14960338175296783f);
    const float tail = bell * (t * q);
    return a < 0.0f ? tail : 1.0f - tail;
}

template <int kAct> __device__ __forceinline__ float activated(float a)
{
    if (kAct == GNMR_ACT_SILU)
        return a * sigmoid(a);
    float bell;
    return a * normal(a, bell);
}

// act(a), and its derivative.
template <int kAct> __device__ __forceinline__ float activated(float a, float &slope)
{
    if (kAct == GNMR_ACT_SILU) {
        const float s = sigmoid(a);
        slope = s * (1.0f + a * (1.0f - s));
        return a * s;
    }
    float bell;
    const float p = normal(a, bell);
    slope = fmaf(a * 0.39894228f, bell, p);
    return a * p;
}

}  // namespace gnmr_act
