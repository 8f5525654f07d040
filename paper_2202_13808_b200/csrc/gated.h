// What the kernels of the gated linear share: the gate functions, and the forms of its products (gated.cu: entry points, element-wise
// backward pass, fp32 FMA products; gated_tc.cu: tensor cores).
#pragma once

#include "common.cuh"

namespace dropit {

// f(a) and, if asked, f'(a).  FAST: for results that are rounded to bf16.
template <int GATE, bool FAST>
__device__ __forceinline__ float gate_value(float a) {
    if constexpr (GATE == DROPIT_GATE_SILU) {
        return FAST ? __fdividef(a, 1.f + __expf(-a)) : a / (1.f + expf(-a));
    } else if constexpr (GATE == DROPIT_GATE_GELU) {
        return a * (0.5f * erfcf(a * -0.70710678f));
    } else {
        return a < 0.f ? 0.f : a;          // a NaN stays one
    }
}
template <int GATE, bool FAST>
__device__ __forceinline__ void gate_value_and_slope(float a, float& value, float& slope) {
    if constexpr (GATE == DROPIT_GATE_SILU) {
        const float s = FAST ? __fdividef(1.f, 1.f + __expf(-a)) : 1.f / (1.f + expf(-a));
        value = a * s;
        slope = s * (1.f + a * (1.f - s));
    } else if constexpr (GATE == DROPIT_GATE_GELU) {
        const float phi = 0.5f * erfcf(a * -0.70710678f);
        value = a * phi;
        slope = phi + a * 0.39894228f * (FAST ? __expf(-0.5f * a * a) : expf(-0.5f * a * a));
    } else {
        value = a < 0.f ? 0.f : a;
        slope = a > 0.f ? 1.f : 0.f;
    }
}

}  // namespace dropit
