// Activations of the gated feed-forward block.
#pragma once

#include "ccdc_block.h"

// act(h); act'(h) through `slope`.  EXACT: the library's full-precision functions, for binary32 blocks; otherwise
// their fast forms, for results that are rounded to 16 bits.  With t the exponential's argument, act is off by less than
// |t| 2^-22 (t's own roundings) + (18 + 1.2 |t|) 2^-23 of itself: 2^-17 where |t| = 14, the negative tail of gelu_tanh at
// h = -4.5.  act' is off by twice that of its two terms' size.
template <int ACT, bool EXACT>
struct Act {
    __device__ __forceinline__ float operator()(float h, float *slope) const {
        if constexpr (ACT == CCDC_ACT_SILU) {
            const float s = EXACT ? 1.0f / (1.0f + expf(-h)) : __fdividef(1.0f, 1.0f + __expf(-h));
            *slope = s * (1.0f + h * (1.0f - s));
            return h * s;
        } else if constexpr (ACT == CCDC_ACT_GELU) {
            const float c = 0.5f * erfcf(-0.70710678118654752f * h);        // the normal distribution's integral up to h
            const float e = EXACT ? expf(-0.5f * h * h) : __expf(-0.5f * h * h);
            *slope = c + h * 0.39894228040143268f * e;
            return h * c;
        } else if constexpr (ACT == CCDC_ACT_GELU_TANH) {
            // (1 + tanh v) / 2 = s(2v) with s(x) = 1 / (1 + exp -x): 1 + tanh v itself cancels in the negative tail
            const float k = 1.59576912160573071f, q = 0.044715f;            // 2 sqrt(2/pi)
            const float hh = fminf(h * h, 1e30f);                           // finite, where the tails multiply it by zero
            const float v = k * h * fmaf(q, hh, 1.0f);
            const float s = EXACT ? 1.0f / (1.0f + expf(-v)) : __fdividef(1.0f, 1.0f + __expf(-v));
            *slope = s + h * s * (1.0f - s) * k * fmaf(3.0f * q, hh, 1.0f);
            return h * s;
        } else {        // NaN stays NaN, in the slope too: a fault upstream must not leave plausible values and gradients
            *slope = h > 0.0f ? 1.0f : h <= 0.0f ? 0.0f : h;
            return h <= 0.0f ? 0.0f : h;
        }
    }
};
// calls f with the activation's function object: one branch for a loop over many elements
template <bool EXACT, class F>
__device__ __forceinline__ void act_apply(int act, F f) {
    if (act == CCDC_ACT_SILU)
        f(Act<CCDC_ACT_SILU, EXACT>());
    else if (act == CCDC_ACT_GELU)
        f(Act<CCDC_ACT_GELU, EXACT>());
    else if (act == CCDC_ACT_GELU_TANH)
        f(Act<CCDC_ACT_GELU_TANH, EXACT>());
    else
        f(Act<CCDC_ACT_RELU, EXACT>());
}
