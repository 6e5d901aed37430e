// Activations of the gated feed-forward block, and the planes of binary32 operands.
#pragma once

#include "ccdc_block.h"

// Binary32 values as three bf16 planes, v = hi + mid + lo, each plane what is left rounded to bf16: 24 bits between them.
// Takes the next plane off two values and returns it as a word, x's in the low half.
__device__ __forceinline__ uint32_t next_plane(float &x, float &y) {
    const uint32_t word = pack2<bf16>(x, y);
    const float2 f = unpack2<bf16>(word);
    x -= f.x, y -= f.y;
    return word;
}
// The first plane takes this form unless all values are below FIRST_MOST in size: above it they would round to infinity
// and are cut off to the largest bf16 instead; infinities and NaN stay in the first plane.  Other values as above.
constexpr float FIRST_MOST = 0x1.FFp127f;
__device__ __forceinline__ uint32_t first_plane_of_any(float &x, float &y) {
    float2 f = unpack2<bf16>(pack2<bf16>(x, y));
    if (!isfinite(f.x)) f.x = __bfloat162float(__float2bfloat16_rz(x));
    if (!isfinite(f.y)) f.y = __bfloat162float(__float2bfloat16_rz(y));
    x = isfinite(f.x) ? x - f.x : 0.0f, y = isfinite(f.y) ? y - f.y : 0.0f;
    return pack2<bf16>(f.x, f.y);
}

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
