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

// Tensor-core forms (bf16, C and H multiples of 8): false if the sizes are not theirs.
bool gated_tc_takes(int64_t M, int64_t C, int64_t H);
dropit_status gated_tc_forward(const void* x, const void* w, const void* bias, int64_t M, int64_t C, int64_t H, dropit_gate gate, void* h, void* gu,
                               int32_t* dev_status, cudaStream_t stream);
dropit_status gated_tc_input_grad(const void* dgu, const void* w, int64_t M, int64_t C, int64_t H, void* dx, int32_t* dev_status, cudaStream_t stream);

}  // namespace dropit
