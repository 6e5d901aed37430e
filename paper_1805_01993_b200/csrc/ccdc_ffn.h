// Activations of the gated feed-forward block.
#pragma once

#include "ccdc_block.h"

// act(h); act'(h) through `slope`.  EXACT: the library's full-precision functions, for binary32 blocks; otherwise
// their fast forms (relative error below 2^-20 where it matters), for results that are rounded to 16 bits.
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
            const float k = 0.79788456080286536f, q = 0.044715f;            // sqrt(2/pi)
            const float v = k * (h + q * h * h * h);
            // tanh v = 1 - 2 / (1 + exp 2v)
            const float t = EXACT ? tanhf(v) : 1.0f - __fdividef(2.0f, 1.0f + __expf(fminf(2.0f * v, 80.0f)));
            *slope = 0.5f * (1.0f + t) + 0.5f * h * (1.0f - t * t) * k * (1.0f + 3.0f * q * h * h);
            return 0.5f * h * (1.0f + t);
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
