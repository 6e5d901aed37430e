// Activations of the gated feed-forward block.
#pragma once

#include "ccdc_block.h"

// act(h); act'(h) through `slope`
__device__ __forceinline__ float act_value(int act, float h, float *slope) {
    if (act == CCDC_ACT_SILU) {
        const float s = 1.0f / (1.0f + expf(-h));
        *slope = s * (1.0f + h * (1.0f - s));
        return h * s;
    }
    if (act == CCDC_ACT_GELU) {
        const float c = 0.5f * erfcf(-0.70710678118654752f * h);        // the normal distribution's integral up to h
        *slope = c + h * 0.39894228040143268f * expf(-0.5f * h * h);
        return h * c;
    }
    if (act == CCDC_ACT_GELU_TANH) {
        const float k = 0.79788456080286536f, q = 0.044715f;            // sqrt(2/pi)
        const float t = tanhf(k * (h + q * h * h * h));
        *slope = 0.5f * (1.0f + t) + 0.5f * h * (1.0f - t * t) * k * (1.0f + 3.0f * q * h * h);
        return 0.5f * h * (1.0f + t);
    }
    *slope = h > 0.0f ? 1.0f : 0.0f;
    return h > 0.0f ? h : 0.0f;
}
