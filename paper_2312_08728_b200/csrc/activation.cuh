// Activations of a gated block.
#pragma once
#include <cuda_runtime.h>

namespace bmgdk {

enum { kActSilu = 0, kActGelu = 1, kActRelu = 2, kActSigmoid = 3 };
// act(g) and act'(g) in fp32 (silu g s, gelu g Phi(g), relu, sigmoid s; s = 1 / (1 + exp(-g)))
// relu by comparisons alone: -inf gives 0, and NaN, which fails both, stays NaN
__device__ __forceinline__ float act_value(int act, float g) {
    if (act == kActRelu) return g <= 0.f ? 0.f : g;
    if (act == kActGelu) return 0.5f * g * (1.f + erff(g * 0.70710678118654752f));
    const float s = __fdividef(1.f, 1.f + __expf(-g));
    return act == kActSigmoid ? s : g * s;
}
__device__ __forceinline__ void act_both(int act, float g, float& value, float& slope) {
    if (act == kActRelu) {
        value = g <= 0.f ? 0.f : g;
        slope = g <= 0.f ? 0.f : g > 0.f ? 1.f : g;
    } else if (act == kActGelu) {
        const float cdf = 0.5f * (1.f + erff(g * 0.70710678118654752f));
        value = g * cdf;
        slope = cdf + g * __expf(-0.5f * g * g) * 0.3989422804014327f;
    } else {
        const float s = __fdividef(1.f, 1.f + __expf(-g));
        if (act == kActSigmoid) { value = s; slope = s * (1.f - s); }
        else { value = g * s; slope = s * (1.f + g * (1.f - s)); }
    }
}


}  // namespace bmgdk
