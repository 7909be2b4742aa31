// Activations of a gated block.
#pragma once
#include <cuda_runtime.h>

namespace bmgdk {

enum { kActSilu = 0, kActGelu = 1, kActRelu = 2, kActSigmoid = 3 };
// Phi(g), the normal distribution's share below g, and e = e^(-g^2 / 2).  Below zero it is taken as a tail, e R(|g|) with R(a) = erfcx(a / sqrt 2) / 2, and keeps its relative
// accuracy: 1 + erf(g / sqrt 2) cancels there (4 % off at -5, nothing left at -6).  R(a) = t Q(t) with t = 1 / (1 + 0.35 a); Q is the polynomial of degree 8 of least relative
// error for 0 <= a <= 14, fitted to erfcx in 64 bits (0.5 units of 2^-24; with its evaluation in fp32 6).  e^(-g^2 / 2) is 0 beyond 13.2.  CUDA's erfcf instead: gates of
// 4096 x 11008 bf16 values 106 us, erff 72, this 57; of degree 7 56, with a quarter more error next to zero.
__device__ __forceinline__ float gelu_share(float g, float& e) {
    const float a = fabsf(g);
    float t;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(fmaf(a, 0.35f, 1.f)));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(g * g * -0.72134752f));  // log2(e) / 2
    float q = -0.029145926f;
    q = fmaf(q, t, 0.14397168f);
    q = fmaf(q, t, -0.25571424f);
    q = fmaf(q, t, 0.15917416f);
    q = fmaf(q, t, -0.02310983f);
    q = fmaf(q, t, 0.105508f);
    q = fmaf(q, t, 0.119832866f);
    q = fmaf(q, t, 0.13986187f);
    q = fmaf(q, t, 0.1396214f);
    const float tail = q * t * e;
    return g < 0.f ? tail : 1.f - tail;
}
// act(g) and act'(g) in fp32 (silu g s, gelu g Phi(g), relu, sigmoid s; s = 1 / (1 + exp(-g)))
// relu by comparisons alone: -inf gives 0, and NaN, which fails both, stays NaN
__device__ __forceinline__ float act_value(int act, float g) {
    if (act == kActRelu) return g <= 0.f ? 0.f : g;
    if (act == kActGelu) {
        float e;
        return g * gelu_share(g, e);
    }
    const float s = __fdividef(1.f, 1.f + __expf(-g));
    return act == kActSigmoid ? s : g * s;
}
__device__ __forceinline__ void act_both(int act, float g, float& value, float& slope) {
    if (act == kActRelu) {
        value = g <= 0.f ? 0.f : g;
        slope = g <= 0.f ? 0.f : g > 0.f ? 1.f : g;
    } else if (act == kActGelu) {
        float e;
        const float cdf = gelu_share(g, e);
        value = g * cdf;
        slope = cdf + g * e * 0.3989422804014327f;
    } else {
        const float s = __fdividef(1.f, 1.f + __expf(-g));
        if (act == kActSigmoid) { value = s; slope = s * (1.f - s); }
        else { value = g * s; slope = s * (1.f + g * (1.f - s)); }
    }
}


}  // namespace bmgdk
