// What the kernels of the gated linear share: the gate functions, and the forms of its products (gated.cu: entry points, element-wise
// backward pass, fp32 FMA products; gated_tc.cu: tensor cores).
#pragma once

#include "common.cuh"
#include "sm100_ptx.cuh"

namespace dropit {

__device__ __forceinline__ float exp2f_approx(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float rcp_approx(float x) {       // 0 above 2^126
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// f(a) and, if asked, f'(a).  FAST: for results that are rounded to bf16.
// The normal distribution's tail Q(|a|) = 1 - Phi(|a|) and its density's exponential e^(-a^2 / 2).  FAST: the exponential times a polynomial in
// t = 1 / (1 + 0.2966 |a|) without a constant term (the form of Abramowitz and Stegun 7.1.26, with one term more), fitted here for |a| < 13.4 where the
// exponential ends: off by 2.1e-5 of Q and by 3e-7 at most, beside what the approximate exponential and reciprocal add (a^2 2^-23 of Q).  a Q(-a) is the
// GELU in its lower tail, so that Q has to be right relative to itself.  A third of erfc's instructions.
template <bool FAST>
__device__ __forceinline__ float normal_tail(float a, float& e) {
    if constexpr (FAST) {
        e = exp2f_approx(a * (a * -0.72134752f));
        const float t = rcp_approx(fmaf(fabsf(a), 0.29656717f, 1.f));
        float p = fmaf(t, -0.082664676f, 0.24276581f);
        p = fmaf(t, p, -0.045114484f);
        p = fmaf(t, p, 0.15672298f);
        p = fmaf(t, p, 0.1093317f);
        p = fmaf(t, p, 0.118958525f);
        return t * p * e;
    } else {
        e = expf(-0.5f * a * a);
        return 0.5f * erfcf(fabsf(a) * 0.70710678f);
    }
}
template <int GATE, bool FAST>
__device__ __forceinline__ void gate_value_and_slope(float a, float& value, float& slope) {
    if constexpr (GATE == DROPIT_GATE_SILU) {
        const float s = FAST ? rcp_approx(1.f + exp2f_approx(a * -1.44269504f)) : 1.f / (1.f + expf(-a));
        value = a * s;
        slope = s * fmaf(a, 1.f - s, 1.f);
    } else if constexpr (GATE == DROPIT_GATE_GELU) {
        float e;
        const float q = normal_tail<FAST>(a, e), phi = a < 0.f ? q : 1.f - q;
        value = a * phi;
        slope = fmaf(a * 0.39894228f, e, phi);
    } else {
        value = a < 0.f ? 0.f : a;          // a NaN stays one
        slope = a > 0.f ? 1.f : 0.f;
    }
}
template <int GATE, bool FAST>
__device__ __forceinline__ float gate_value(float a) {
    float value, slope;
    gate_value_and_slope<GATE, FAST>(a, value, slope);
    return value;
}

// A launch that may be set up while the kernel in front of it in the stream ends: the kernel calls grid_dependency_wait before it touches memory.
template <typename... Params, typename... Args>
dropit_status launch_programmatic(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, cudaStream_t stream, Args... args) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...) != cudaSuccess) {
        (void)cudaGetLastError();
        return DROPIT_ERR_CUDA;
    }
    return check_launch();
}

// Tensor-core forms (bf16, C and H multiples of 8): false if the sizes are not theirs.
bool gated_tc_takes(int64_t M, int64_t C, int64_t H);
dropit_status gated_tc_forward(const void* x, const void* w, const void* bias, int64_t M, int64_t C, int64_t H, dropit_gate gate, void* h, void* gu,
                               int32_t* dev_status, cudaStream_t stream);
dropit_status gated_tc_input_grad(const void* dgu, const void* w, int64_t M, int64_t C, int64_t H, void* dx, int32_t* dev_status, cudaStream_t stream);

}  // namespace dropit
