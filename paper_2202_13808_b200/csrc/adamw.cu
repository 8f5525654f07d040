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
__host__ __device__ __forceinline__ uint32_t mix_rest(uint32_t x) {       // all but its first line
    x *= 0x7FEB352Du;
    x ^= x >> 15;
    x *= 0x846CA68Bu;
    return x ^ (x >> 16);
}
__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) { return mix_rest(x ^ (x >> 16)); }

// ---- four values of a lane, FULL: all inside the tensor and aligned ----
template <bool FULL>
__device__ __forceinline__ void load4(const float* p, int64_t at, int64_t n, float (&v)[4]) {
    if constexpr (FULL) {
        const float4 q = *reinterpret_cast<const float4*>(p + at);
        v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = at + e < n ? p[at + e] : 0.f;
    }
}
template <bool FULL>
__device__ __forceinline__ void load4(const uint16_t* p, int64_t at, int64_t n, float (&v)[4]) {
    if constexpr (FULL) {
        const uint2 q = *reinterpret_cast<const uint2*>(p + at);
        v[0] = __uint_as_float(q.x << 16); v[1] = __uint_as_float(q.x & 0xFFFF0000u);
        v[2] = __uint_as_float(q.y << 16); v[3] = __uint_as_float(q.y & 0xFFFF0000u);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = at + e < n ? __uint_as_float((uint32_t)p[at + e] << 16) : 0.f;
    }
}
template <bool FULL>
__device__ __forceinline__ void store4(float* p, int64_t at, int64_t n, const float (&v)[4]) {
    if constexpr (FULL) {
        *reinterpret_cast<float4*>(p + at) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (at + e < n) p[at + e] = v[e];
    }
}
__device__ __forceinline__ uint32_t nearest_bf16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <bool FULL>
__device__ __forceinline__ void store4_bf16(uint16_t* p, int64_t at, int64_t n, uint32_t lo, uint32_t hi) {
    if constexpr (FULL) {
        *reinterpret_cast<uint2*>(p + at) = make_uint2(lo, hi);
    } else {
        const uint32_t b[4] = {lo & 0xFFFFu, lo >> 16, hi & 0xFFFFu, hi >> 16};
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (at + e < n) p[at + e] = (uint16_t)b[e];
    }
}
// Up to the next bf16 with the probability of the value's place between two of them: a 16-bit random fraction is added to the half that goes.  An
// infinity stays one; a NaN could carry into the sign and is kept by the caller.
__device__ __forceinline__ uint32_t dithered(float v, uint32_t word) { return __float_as_uint(v) + ((word * 0x9E3779B1u) >> 16); }

__device__ __forceinline__ float2 decode_pair(uint32_t codes16) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)codes16, __NV_E4M3);
    return __half22float2(__half2(h));
}
__device__ __forceinline__ void decode4(uint32_t codes, float (&v)[4]) {
    const float2 a = decode_pair(codes & 0xFFFFu), b = decode_pair(codes >> 16);
    v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
}
// A value of up to 448 to one of the two codes around it, in the top byte and without its sign.  Times 2^-120 the 8-bit floats' normal numbers
// are fp32's (exponent field 1 to 15) and their subnormals fp32's subnormals, so that the code is seven bits of the fp32 pattern; the 20 bits
// below them are the place between two codes, to which the random fraction is added.
// (The product in assembly: as C++, nvcc 12.9 pairs it with its neighbour's and returns zeros.)
__device__ __forceinline__ uint32_t code_of(float y, uint32_t bits16_in_the_middle) {
    float z;
    asm("mul.rn.f32 %0, %1, %2;" : "=f"(z) : "f"(y), "f"(0x1p-120f));
    return min((__float_as_uint(z) << 4) + bits16_in_the_middle, 0x7EFFFFFFu);
}
__device__ __forceinline__ uint32_t top_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// Largest magnitude of the warp's values (NaN if there is one), and from it the scale and its reciprocal.  Magnitudes
// below 1e-30 count as zero; a block with an infinity or a NaN gets the scale NaN and stays so.
__device__ __forceinline__ float block_scale(float top, float& inverse) {
    uint32_t bits = __float_as_uint(top) & 0x7FFFFFFFu;
    bits = __reduce_max_sync(kFullMask, bits);
    const float amax = __uint_as_float(bits);
    if (bits >= 0x7F800000u) {
        inverse = 0.f;
        return __uint_as_float(0x7FC00000u);
    }
    const float scale = amax < 1e-30f ? 0.f : __fdiv_rn(amax, 448.f);
    inverse = scale > 0.f ? __frcp_rn(scale) : 0.f;
    return scale;
}

// FTZ: values below 2^-126 have the root 0.
template <bool FTZ>
__device__ __forceinline__ float approx_sqrt(float x) {
    float r;
    if (FTZ) asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    else asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float approx_rcp(float x) {       // x is no subnormal: at least the root of the smallest v, 2^-75
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// What holds for a tensor.
struct Step {
    float beta1, beta2, gain1, gain2;       // gain: (1 - beta) times the gradients' factor, squared for the second moment
    float eps, decay, rate, root_correction;
    uint32_t key;
};

template <typename P, typename G, bool BITS8, bool FULL>
__device__ __forceinline__ void step_block(const Args& a, const Entry& e, const Step& k, uint32_t inside, int lane) {
    const size_t arena = (size_t)e.first_block + inside;
    P* p = reinterpret_cast<P*>(e.p);
    const G* g = reinterpret_cast<const G*>(e.g);
    const int64_t at = (int64_t)inside * kBlock + lane * 4;
    float* master = sizeof(P) == 2 && a.master ? a.master + arena * kBlock : nullptr;
    float gv[2][4], pv[2][4], mv[2][4], vv[2][4];
    float m_scale = 1.f, v_scale = 1.f;
    if constexpr (BITS8) {
        m_scale = a.m_scale[arena];
        v_scale = a.v_scale[arena];
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        load4<FULL>(g, at + h * 128, e.n, gv[h]);
        if (master) load4<true>(master, h * 128 + lane * 4, kBlock, pv[h]);
        else load4<FULL>(p, at + h * 128, e.n, pv[h]);
        const size_t quad = arena * (kBlock / 4) + h * 32 + lane;
        if constexpr (BITS8) {
            decode4(reinterpret_cast<const uint32_t*>(a.m)[quad], mv[h]);
            decode4(reinterpret_cast<const uint32_t*>(a.v)[quad], vv[h]);
        } else {
            load4<true>(reinterpret_cast<const float*>(a.m), (int64_t)quad * 4, 0, mv[h]);
            load4<true>(reinterpret_cast<const float*>(a.v), (int64_t)quad * 4, 0, vv[h]);
        }
    }
    float top_m = 0.f, top_v = 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float gr = gv[h][i];
            const float root0 = vv[h][i] * v_scale;
            const float m = fmaf(k.gain1, gr, k.beta1 * (BITS8 ? mv[h][i] * m_scale : mv[h][i]));
            const float v = fmaf(k.gain2, gr * gr, k.beta2 * (BITS8 ? root0 * root0 : vv[h][i]));
            const float root = approx_sqrt<BITS8>(v);
            pv[h][i] = fmaf(pv[h][i], k.decay, -k.rate * (m * approx_rcp(fmaf(root, k.root_correction, k.eps))));
            mv[h][i] = m;
            vv[h][i] = BITS8 ? root : v;
            if (BITS8) {
                top_m = max_nan(top_m, fabsf(m));
                top_v = max_nan(top_v, root);
            }
        }
    }
    float inv_m = 0.f, inv_v = 0.f;
    if constexpr (BITS8) {
        m_scale = block_scale(top_m, inv_m);
        v_scale = block_scale(top_v, inv_v);
        if (lane == 0) {
            a.m_scale[arena] = m_scale;
            a.v_scale[arena] = v_scale;
        }
    }
    const bool dither = sizeof(P) == 2 && a.dither;
    // The word of place i is mix(i ^ key); the high halves of the eight i are the same, and so is what the first shift brings down.
    const uint32_t start = ((uint32_t)at ^ k.key) ^ (((uint32_t)at ^ k.key) >> 16);
    float sum = 0.f;
    if (dither) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += pv[h][i];
    }
    const bool finite = (__float_as_uint(sum) & 0x7F800000u) != 0x7F800000u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t word[4];
        if (BITS8 || dither) {
#pragma unroll
            for (int i = 0; i < 4; ++i) word[i] = mix_rest(start ^ (uint32_t)(h * 128 + i));
        }
        if (master) store4<true>(master, h * 128 + lane * 4, kBlock, pv[h]);
        if constexpr (sizeof(P) == 2) {
            uint32_t lo, hi;
            if (dither) {
                uint32_t b[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    b[i] = dithered(pv[h][i], word[i]);
                    if (!finite && !isfinite(pv[h][i])) b[i] = __float_as_uint(pv[h][i]);
                }
                lo = __byte_perm(b[0], b[1], 0x7632);
                hi = __byte_perm(b[2], b[3], 0x7632);
            } else {
                lo = nearest_bf16x2(pv[h][0], pv[h][1]);
                hi = nearest_bf16x2(pv[h][2], pv[h][3]);
            }
            store4_bf16<FULL>(p, at + h * 128, e.n, lo, hi);
        } else {
            store4<FULL>(p, at + h * 128, e.n, pv[h]);
        }
        const size_t quad = arena * (kBlock / 4) + h * 32 + lane;
        if constexpr (BITS8) {
            uint32_t tm[4], tv[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                tm[i] = code_of(mv[h][i] * inv_m, __byte_perm(word[i], 0, 0x4324));      // the high half, one byte up
                tv[i] = code_of(vv[h][i] * inv_v, __byte_perm(word[i], 0, 0x4104));      // the low half
                if (vv[h][i] > 0.f) tv[i] = max(tv[i], 0x01000000u);
            }
            const uint32_t signs = top_bytes(__float_as_uint(mv[h][0]), __float_as_uint(mv[h][1]), __float_as_uint(mv[h][2]), __float_as_uint(mv[h][3]));
            reinterpret_cast<uint32_t*>(a.m)[quad] = (top_bytes(tm[0], tm[1], tm[2], tm[3]) & 0x7F7F7F7Fu) | (signs & 0x80808080u);
            reinterpret_cast<uint32_t*>(a.v)[quad] = top_bytes(tv[0], tv[1], tv[2], tv[3]) & 0x7F7F7F7Fu;
        } else {
            store4<true>(reinterpret_cast<float*>(a.m), (int64_t)quad * 4, 0, mv[h]);
            store4<true>(reinterpret_cast<float*>(a.v), (int64_t)quad * 4, 0, vv[h]);
        }
    }
}

template <typename P, typename G, bool BITS8>
__global__ void __launch_bounds__(kThreads)
adamw_kernel(const __grid_constant__ Args a) {
    const int lane = threadIdx.x & 31;
    const uint32_t warps = gridDim.x * (kThreads / 32);
    Step k;
    const float grad_factor = a.grad_factor ? *a.grad_factor : 1.f;
    k.beta1 = a.beta1;
    k.beta2 = a.beta2;
    k.gain1 = a.one_minus_beta1 * grad_factor;
    k.gain2 = a.one_minus_beta2 * grad_factor * grad_factor;
    k.eps = a.eps;
    uint32_t entry = 0, entry_first = 0, entry_end = 0;
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
            k.decay = 1.f - lr * a.entry[lo].weight_decay;
            k.rate = lr / -expm1f(t * a.ln_beta1);
            k.root_correction = rsqrtf(-expm1f(t * a.ln_beta2));
            k.key = mix(mix(a.seed + step) + a.entry[lo].ordinal);
        }
        const Entry& e = a.entry[entry];
        const uint32_t inside = block - entry_first;
        if (e.vectors && (int64_t)(inside + 1) * kBlock <= (int64_t)e.n) step_block<P, G, BITS8, true>(a, e, k, inside, lane);
        else step_block<P, G, BITS8, false>(a, e, k, inside, lane);
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
