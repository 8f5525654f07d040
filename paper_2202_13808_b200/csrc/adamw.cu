// One AdamW step over all tensors of a model in one launch (decoupled weight decay, bias correction):
//     m = b1 m + (1 - b1) g,   v = b2 v + (1 - b2) g^2,   p = (1 - lr wd) p - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps).
//
// The tensors come as a table in the kernel's arguments (up to kMaxEntries a launch), so that nothing is copied to the device for a step and
// a captured step replays.  The moments lie in arenas of whole blocks of 256 values; a block is a warp's unit of work, eight values a lane.
// The step numbers are on the device, and the last CTA to finish counts them up.
//
// Moments in 8 bits: m and sqrt(v) as 8-bit floats (4 exponent and 3 mantissa bits) under one fp32 scale per block.  A step
// changes v by a part in a thousand, far less than half of a code's spacing, so rounding to the nearest code would freeze it; codes
// are rounded up with the probability of the value's place between two codes (a 16-bit random fraction from a mixing function of seed,
// step, tensor and place), which is right on average.  sqrt(v) needs half the exponent range of v, and never becomes zero
// while v is not, so that no value moves by m / eps.
//
// Bound by HBM: gradients read, parameters and moments read and written, 28 bytes a value in fp32 and 10.06 with bf16 parameters and
// gradients and moments in 8 bits.
#include <math.h>

#include <algorithm>

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"

namespace dropit {

namespace {

constexpr int kBlock = DROPIT_ADAMW_BLOCK;
constexpr int kThreads = 256;
constexpr int kMaxEntries = 512;

struct Entry {
    void* p;
    const void* g;
    const float* lr_device;
    uint32_t first_block;       // in the arenas
    uint32_t before;            // blocks of this launch's tensors in front of this one
    uint32_t n;
    uint32_t ordinal;
    float lr, weight_decay;
    uint32_t vectors;           // p and g are aligned for loads of four values
    uint32_t reserved;
};
struct Args {
    float beta1, beta2, one_minus_beta1, one_minus_beta2, ln_beta1, ln_beta2, eps;
    uint32_t seed;              // already mixed
    uint32_t blocks, count;
    int dither;
    void* m;
    void* v;
    float* m_scale;
    float* v_scale;
    float* master;
    int32_t* steps;
    uint32_t* ticket;
    const float* grad_factor;
    Entry entry[kMaxEntries];
};
static_assert(sizeof(Args) <= 32764, "kernel arguments");

// A mixing function of 32-bit words: two multiplications, three shifts (the constants are those of C. Wellons' published search for low bias).
__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {
    x ^= x >> 16;
    x *= 0x7FEB352Du;
    x ^= x >> 15;
    x *= 0x846CA68Bu;
    return x ^ (x >> 16);
}

// Four values at p + at, of which the tensor has `left`.
__device__ __forceinline__ void load4(const float* p, int64_t at, int left, bool vec, float (&v)[4]) {
    if (vec && left >= 4) {
        const float4 q = *reinterpret_cast<const float4*>(p + at);
        v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = e < left ? p[at + e] : 0.f;
}
__device__ __forceinline__ float bf16_value(uint32_t b) { return __uint_as_float(b << 16); }
__device__ __forceinline__ void load4(const uint16_t* p, int64_t at, int left, bool vec, float (&v)[4]) {
    if (vec && left >= 4) {
        const uint2 q = *reinterpret_cast<const uint2*>(p + at);
        v[0] = bf16_value(q.x & 0xFFFFu); v[1] = bf16_value(q.x >> 16); v[2] = bf16_value(q.y & 0xFFFFu); v[3] = bf16_value(q.y >> 16);
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = e < left ? bf16_value(p[at + e]) : 0.f;
}
__device__ __forceinline__ void store4(float* p, int64_t at, int left, bool vec, const float (&v)[4], const uint32_t (&)[4], bool) {
    if (vec && left >= 4) {
        *reinterpret_cast<float4*>(p + at) = make_float4(v[0], v[1], v[2], v[3]);
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) p[at + e] = v[e];
}
// To the nearest bf16, or up with the probability of the value's place between two of them.
__device__ __forceinline__ uint32_t to_bf16(float v, uint32_t word, bool dither) {
    if (dither && (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u) return (__float_as_uint(v) + ((word * 0x9E3779B1u) >> 16)) >> 16;
    uint16_t r;
    asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ void store4(uint16_t* p, int64_t at, int left, bool vec, const float (&v)[4], const uint32_t (&word)[4], bool dither) {
    uint32_t b[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] = to_bf16(v[e], word[e], dither);
    if (vec && left >= 4) {
        *reinterpret_cast<uint2*>(p + at) = make_uint2(b[0] | (b[1] << 16), b[2] | (b[3] << 16));
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) p[at + e] = (uint16_t)b[e];
}

__device__ __forceinline__ float2 decode_pair(uint32_t codes16) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)codes16, __NV_E4M3);
    return __half22float2(__half2(h));
}
__device__ __forceinline__ void decode4(uint32_t codes, float scale, float (&v)[4]) {
    const float2 a = decode_pair(codes & 0xFFFFu), b = decode_pair(codes >> 16);
    v[0] = a.x * scale; v[1] = a.y * scale; v[2] = b.x * scale; v[3] = b.y * scale;
}
// A magnitude of up to 448 to one of the two codes around it: the random fraction is added below the three mantissa bits that stay.
// Under 2^-6 the codes are 2^-9 apart; there the sum is formed in the binade from 2^-6 on, whose codes have that spacing.
__device__ __forceinline__ float round_to_code(float a, uint32_t bits16) {
    const float low = a < 0x1p-6f ? 0x1p-6f : 0.f;
    const float t = __uint_as_float((__float_as_uint(a + low) + (bits16 << 4)) & 0xFFF00000u) - low;
    return fminf(t, 448.f);
}
__device__ __forceinline__ uint32_t encode4(const float (&t)[4]) {     // values that are codes already
    return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(t[0], t[1]), __NV_SATFINITE, __NV_E4M3) |
           ((uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(t[2], t[3]), __NV_SATFINITE, __NV_E4M3) << 16);
}
// Largest magnitude of the warp's values as bits (NaN patterns are above infinity), and from it the scale and its reciprocal.  Magnitudes
// below 1e-30 count as zero; a block with an infinity or a NaN gets the scale NaN and stays so.
__device__ __forceinline__ float block_scale(uint32_t top, float& inverse) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(kFullMask, top, o));
    const float amax = __uint_as_float(top);
    if (top >= 0x7F800000u) {
        inverse = 0.f;
        return __uint_as_float(0x7FC00000u);
    }
    const float scale = amax < 1e-30f ? 0.f : __fdiv_rn(amax, 448.f);
    inverse = scale > 0.f ? __frcp_rn(scale) : 0.f;
    return scale;
}

__device__ __forceinline__ float approx_sqrt(float x) {
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

template <typename P, typename G, bool BITS8>
__global__ void __launch_bounds__(kThreads)
adamw_kernel(const __grid_constant__ Args a) {
    const int lane = threadIdx.x & 31;
    const uint32_t warps = gridDim.x * (kThreads / 32);
    const float grad_factor = a.grad_factor ? *a.grad_factor : 1.f;
    uint32_t entry = 0, entry_first = 0, entry_end = 0;
    float decay = 0.f, rate = 0.f, root_correction = 0.f;
    uint32_t key = 0;
    for (uint32_t block = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); block < a.blocks; block += warps) {
        if (block >= entry_end) {           // the tensor that this block is part of
            uint32_t lo = entry, hi = a.count;
            while (hi - lo > 1) {
                const uint32_t mid = (lo + hi) / 2;
                if (a.entry[mid].before <= block) lo = mid; else hi = mid;
            }
            entry = lo;
            entry_first = a.entry[lo].before;
            entry_end = lo + 1 < a.count ? a.entry[lo + 1].before : a.blocks;
            const uint32_t step = (uint32_t)a.steps[a.entry[lo].ordinal] + 1u;
            const float t = (float)step;
            float lr = a.entry[lo].lr;
            if (a.entry[lo].lr_device) lr = *a.entry[lo].lr_device;
            decay = 1.f - lr * a.entry[lo].weight_decay;
            rate = lr / -expm1f(t * a.ln_beta1);
            root_correction = rsqrtf(-expm1f(t * a.ln_beta2));
            key = mix(mix(a.seed + step) + a.entry[lo].ordinal);
        }
        const Entry& e = a.entry[entry];
        const uint32_t inside = block - entry_first;
        const size_t arena = (size_t)e.first_block + inside;
        P* p = reinterpret_cast<P*>(e.p);
        const G* g = reinterpret_cast<const G*>(e.g);
        float gv[2][4], pv[2][4], mv[2][4], vv[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t at = (int64_t)inside * kBlock + h * 128 + lane * 4;
            const int left = (int)min((int64_t)4, max((int64_t)0, (int64_t)e.n - at));
            load4(g, at, left, e.vectors != 0, gv[h]);
            if (a.master) load4(a.master + arena * kBlock, h * 128 + lane * 4, 4, true, pv[h]);
            else load4(p, at, left, e.vectors != 0, pv[h]);
            const size_t quad = arena * (kBlock / 4) + h * 32 + lane;
            if constexpr (BITS8) {
                decode4(reinterpret_cast<const uint32_t*>(a.m)[quad], a.m_scale[arena], mv[h]);
                decode4(reinterpret_cast<const uint32_t*>(a.v)[quad], a.v_scale[arena], vv[h]);
            } else {
                load4(reinterpret_cast<const float*>(a.m), (int64_t)quad * 4, 4, true, mv[h]);
                load4(reinterpret_cast<const float*>(a.v), (int64_t)quad * 4, 4, true, vv[h]);
            }
        }
        uint32_t top_m = 0, top_v = 0, word[2][4] = {};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float gr = gv[h][i] * grad_factor;
                const float m = fmaf(a.one_minus_beta1, gr, a.beta1 * mv[h][i]);
                const float v = fmaf(a.one_minus_beta2, gr * gr, a.beta2 * (BITS8 ? vv[h][i] * vv[h][i] : vv[h][i]));
                const float root = approx_sqrt(v);
                pv[h][i] = fmaf(pv[h][i], decay, -rate * __fdividef(m, fmaf(root, root_correction, a.eps)));
                mv[h][i] = m;
                vv[h][i] = BITS8 ? root : v;
                if (BITS8) {
                    top_m = max(top_m, __float_as_uint(m) & 0x7FFFFFFFu);
                    top_v = max(top_v, __float_as_uint(root) & 0x7FFFFFFFu);
                }
                if (BITS8 || sizeof(P) == 2) word[h][i] = mix((inside * kBlock + h * 128 + lane * 4 + i) ^ key);
            }
        }
        float inv_m = 0.f, inv_v = 0.f, scale_m = 0.f, scale_v = 0.f;
        if constexpr (BITS8) {
            scale_m = block_scale(top_m, inv_m);
            scale_v = block_scale(top_v, inv_v);
            if (lane == 0) {
                a.m_scale[arena] = scale_m;
                a.v_scale[arena] = scale_v;
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t at = (int64_t)inside * kBlock + h * 128 + lane * 4;
            const int left = (int)min((int64_t)4, max((int64_t)0, (int64_t)e.n - at));
            if (a.master) store4(a.master + arena * kBlock, h * 128 + lane * 4, 4, true, pv[h], word[h], false);
            store4(p, at, left, e.vectors != 0, pv[h], word[h], a.dither != 0);
            const size_t quad = arena * (kBlock / 4) + h * 32 + lane;
            if constexpr (BITS8) {
                float tm[4], tv[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float y = mv[h][i] * inv_m, z = vv[h][i] * inv_v;
                    tm[i] = copysignf(round_to_code(fabsf(y), word[h][i] >> 16), y);
                    tv[i] = round_to_code(z, word[h][i] & 0xFFFFu);
                    if (z > 0.f) tv[i] = fmaxf(tv[i], 0x1p-9f);
                }
                reinterpret_cast<uint32_t*>(a.m)[quad] = encode4(tm);
                reinterpret_cast<uint32_t*>(a.v)[quad] = encode4(tv);
            } else {
                store4(reinterpret_cast<float*>(a.m), (int64_t)quad * 4, 4, true, mv[h], word[h], false);
                store4(reinterpret_cast<float*>(a.v), (int64_t)quad * 4, 4, true, vv[h], word[h], false);
            }
        }
    }
    // Every CTA has read the step numbers that it needed when it draws its ticket.
    __shared__ uint32_t drawn;
    __syncthreads();
    if (threadIdx.x == 0) drawn = atomicAdd(a.ticket, 1u);
    __syncthreads();
    if (drawn == gridDim.x - 1) {
        for (uint32_t i = threadIdx.x; i < a.count; i += kThreads) a.steps[a.entry[i].ordinal] += 1;
        if (threadIdx.x == 0) *a.ticket = 0u;
    }
}

using Kernel = void (*)(Args);
template <bool BITS8>
Kernel pick(dropit_dtype p, dropit_dtype g) {
    if (p == DROPIT_BF16) return g == DROPIT_BF16 ? adamw_kernel<uint16_t, uint16_t, BITS8> : adamw_kernel<uint16_t, float, BITS8>;
    return g == DROPIT_BF16 ? adamw_kernel<float, uint16_t, BITS8> : adamw_kernel<float, float, BITS8>;
}

int64_t blocks_of(int64_t n) { return (n + kBlock - 1) / kBlock; }

}  // namespace

}  // namespace dropit

using namespace dropit;

extern "C" dropit_status dropit_adamw_step(const dropit_adamw_tensor* tensors, int count, const dropit_adamw_options* options,
                                           const dropit_adamw_state* state, void* cuda_stream) {
    if (count < 0 || (count && !tensors) || !options || !state) return DROPIT_ERR_INVALID_ARG;
    const dropit_adamw_options& o = *options;
    const dropit_adamw_state& s = *state;
    auto type_ok = [](dropit_dtype t) { return t == DROPIT_BF16 || t == DROPIT_F32; };
    if (!type_ok(o.param_dtype) || !type_ok(o.grad_dtype) || (o.state_bits != 32 && o.state_bits != 8)) return DROPIT_ERR_INVALID_ARG;
    if (!(o.beta1 >= 0 && o.beta1 < 1) || !(o.beta2 >= 0 && o.beta2 < 1) || !(o.eps >= 0)) return DROPIT_ERR_INVALID_ARG;
    if (s.master && o.param_dtype != DROPIT_BF16) return DROPIT_ERR_INVALID_ARG;
    const int param_size = o.param_dtype == DROPIT_BF16 ? 2 : 4, grad_size = o.grad_dtype == DROPIT_BF16 ? 2 : 4;
    bool any = false;
    for (int i = 0; i < count; ++i) {
        const dropit_adamw_tensor& t = tensors[i];
        if (t.n < 0 || t.n >= ((int64_t)1 << 31) || t.first_block < 0 || t.first_block + blocks_of(t.n) > UINT32_MAX || t.ordinal < 0)
            return DROPIT_ERR_INVALID_ARG;
        if (!isfinite(t.lr) || !isfinite(t.weight_decay)) return DROPIT_ERR_INVALID_ARG;
        if (t.n && (!t.param || !t.grad || reinterpret_cast<uintptr_t>(t.param) % param_size || reinterpret_cast<uintptr_t>(t.grad) % grad_size))
            return DROPIT_ERR_INVALID_ARG;
        any |= t.n != 0;
    }
    if (!any) return DROPIT_OK;
    const void* arenas[] = {s.exp_avg, s.exp_avg_sq, s.steps, s.ticket, o.state_bits == 8 ? s.exp_avg_scale : s.exp_avg,
                            o.state_bits == 8 ? s.exp_avg_sq_scale : s.exp_avg, s.master ? s.master : s.exp_avg};
    for (const void* p : arenas)
        if (!p || reinterpret_cast<uintptr_t>(p) % 4) return DROPIT_ERR_INVALID_ARG;
    if (!is_aligned16(s.exp_avg) || !is_aligned16(s.exp_avg_sq) || (s.master && !is_aligned16(s.master))) return DROPIT_ERR_INVALID_ARG;

    Args a = {};
    a.beta1 = (float)o.beta1;
    a.beta2 = (float)o.beta2;
    a.one_minus_beta1 = (float)(1.0 - o.beta1);
    a.one_minus_beta2 = (float)(1.0 - o.beta2);
    a.ln_beta1 = (float)log(o.beta1);
    a.ln_beta2 = (float)log(o.beta2);
    a.eps = (float)o.eps;
    a.seed = mix(o.seed);
    a.dither = o.dither && o.param_dtype == DROPIT_BF16;
    a.m = s.exp_avg;
    a.v = s.exp_avg_sq;
    a.m_scale = s.exp_avg_scale;
    a.v_scale = s.exp_avg_sq_scale;
    a.master = s.master;
    a.steps = s.steps;
    a.ticket = s.ticket;
    a.grad_factor = s.grad_factor;
    const Kernel kernel = o.state_bits == 8 ? pick<true>(o.param_dtype, o.grad_dtype) : pick<false>(o.param_dtype, o.grad_dtype);
    int i = 0;
    while (i < count) {
        a.count = 0;
        uint64_t blocks = 0;
        for (; i < count && a.count < kMaxEntries; ++i) {
            const dropit_adamw_tensor& t = tensors[i];
            const uint64_t more = (uint64_t)blocks_of(t.n);
            if (t.n == 0) continue;
            if (blocks + more > INT32_MAX) break;
            Entry& e = a.entry[a.count++];
            const uintptr_t odd = (reinterpret_cast<uintptr_t>(t.param) % (4 * param_size)) | (reinterpret_cast<uintptr_t>(t.grad) % (4 * grad_size));
            e = {t.param, t.grad, t.lr_device, (uint32_t)t.first_block, (uint32_t)blocks, (uint32_t)t.n, (uint32_t)t.ordinal, t.lr,
                 t.weight_decay, odd == 0 ? 1u : 0u, 0u};
            blocks += more;
        }
        if (!a.count) break;
        a.blocks = (uint32_t)blocks;
        const int64_t grid = std::min<int64_t>(((int64_t)blocks + kThreads / 32 - 1) / (kThreads / 32), (int64_t)sm_count() * 8);
        kernel<<<(unsigned)grid, kThreads, 0, as_stream(cuda_stream)>>>(a);
        const dropit_status status = check_launch();
        if (status != DROPIT_OK) return status;
    }
    return DROPIT_OK;
}
