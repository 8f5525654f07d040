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
#include <type_traits>

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"

namespace dropit {

namespace {

constexpr int kBlock = DROPIT_ADAMW_BLOCK;
constexpr int kThreads = 128;
constexpr int kMaxEntries = 512;
constexpr uint32_t kMaxRun = 16;                    // blocks of a run (8 bits, 86.6 M values: 315 / 225 / 217 / 211 us with 1 / 8 / 16 / 32; at other sizes 16 and 32 take turns)
constexpr int kResident8 = 5, kResident32 = 4;          // CTAs per SM: 8 bits 219 / 217 / 231 us with 4 / 5 / 6, which spills

struct Entry {
    void* p;
    const void* g;
    const float* lr_device;
    uint32_t first_block;       // in the arenas
    uint32_t before;            // runs of this launch's tensors in front of this one
    uint32_t n;
    uint32_t ordinal;
    float lr, weight_decay;
    uint32_t vectors;           // p and g are aligned to 16 bytes
    uint32_t reserved;
};
struct Args {
    float beta1, beta2, one_minus_beta1, one_minus_beta2, ln_beta1, ln_beta2, eps;
    uint32_t seed;              // already mixed
    uint32_t runs, run, count;      // run: blocks of one
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

// ---- a lane's eight values of a block: neighbours where moments are in 8 bits (16 bytes of bf16, 8 of codes), else two quads of fp32 ----
template <bool BITS8>
__device__ __forceinline__ int lane_start(int lane) { return BITS8 ? lane * 8 : lane * 4; }
template <bool BITS8>
__host__ __device__ constexpr int place_of(int i) { return BITS8 ? i : (i >> 2) * 128 + (i & 3); }

// The words that eight values of type T are held in, and how they come and go.  at: the lane's first value; left: values from there to the tensor's end.
template <typename T> constexpr int kWords = sizeof(T) * 2;
template <typename T, bool BITS8, bool FULL>
__device__ __forceinline__ void load8(const T* p, int64_t left, uint32_t (&w)[kWords<T>]) {
    if constexpr (FULL) {
        if constexpr (sizeof(T) == 4 || !BITS8) {
            using Quad = typename std::conditional<sizeof(T) == 4, uint4, uint2>::type;
            const Quad q[2] = {*reinterpret_cast<const Quad*>(p), *reinterpret_cast<const Quad*>(p + place_of<BITS8>(4))};
            if constexpr (sizeof(T) == 4) {
                w[0] = q[0].x; w[1] = q[0].y; w[2] = q[0].z; w[3] = q[0].w; w[4] = q[1].x; w[5] = q[1].y; w[6] = q[1].z; w[7] = q[1].w;
            } else {
                w[0] = q[0].x; w[1] = q[0].y; w[2] = q[1].x; w[3] = q[1].y;
            }
        } else {
            const uint4 q = *reinterpret_cast<const uint4*>(p);
            w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kWords<T>; ++i) w[i] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (place_of<BITS8>(i) >= left) continue;
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(p[place_of<BITS8>(i)]);
            else w[i / 2] |= (uint32_t)p[place_of<BITS8>(i)] << (16 * (i & 1));
        }
    }
}
template <typename T, bool BITS8, bool FULL>
__device__ __forceinline__ void store8(T* p, int64_t left, const uint32_t (&w)[kWords<T>]) {
    if constexpr (FULL) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
            *reinterpret_cast<uint4*>(p + place_of<BITS8>(4)) = make_uint4(w[4], w[5], w[6], w[7]);
        } else if constexpr (!BITS8) {
            *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
            *reinterpret_cast<uint2*>(p + place_of<BITS8>(4)) = make_uint2(w[2], w[3]);
        } else {
            *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (place_of<BITS8>(i) >= left) continue;
            if constexpr (sizeof(T) == 4) p[place_of<BITS8>(i)] = __uint_as_float(w[i]);
            else p[place_of<BITS8>(i)] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
        }
    }
}
template <int WORDS>
__device__ __forceinline__ float value_of(const uint32_t (&w)[WORDS], int i) {
    if constexpr (WORDS == 8) return __uint_as_float(w[i]);
    else return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
}
__device__ __forceinline__ uint32_t nearest_bf16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Up to the next bf16 with the probability of the value's place between two of them: a 16-bit random fraction is added to the half that goes.  An
// infinity stays one; a NaN could carry into the sign and is kept by the caller.
__device__ __forceinline__ uint32_t dithered(float v, uint32_t word) { return __float_as_uint(v) + ((word * 0x9E3779B1u) >> 16); }

// Products in assembly: nvcc 12.9 otherwise pairs them into 64-bit registers, which costs more moves than it saves products (and for products with
// 2^-120 it returned zeros).
__device__ __forceinline__ float mul(float a, float b) {
    float r;
    asm("mul.rn.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float fma(float a, float b, float c) {
    float r;
    asm("fma.rn.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// Two 8-bit floats.
__device__ __forceinline__ float2 decode_pair(uint32_t codes16) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)codes16, __NV_E4M3);
    return __half22float2(__half2(h));
}
// A value of up to 448 (1 + 2^-20) to one of the two codes around it, in the top byte and without its sign (448 itself stays: the fraction is below one); z is
// the pattern of 2^-120 times the value.  There
// the 8-bit floats' normal numbers are fp32's (exponent field 1 to 15) and their subnormals fp32's subnormals, so that the code is seven bits
// of the pattern; the 20 bits below them are the place between two codes, to which the random fraction is added.
__device__ __forceinline__ uint32_t code_of(uint32_t z, uint32_t bits16_in_the_middle) { return (z << 4) + bits16_in_the_middle; }
__device__ __forceinline__ uint32_t top_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}
__device__ __forceinline__ float max_nan(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float approx_rcp(float x) {       // neither x nor 1 / x is subnormal
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float approx_sqrt(float x) {
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// The root to the nearest fp32 for x of 2^-102 and more: x times its approximate reciprocal root, and a Newton step whose residue is exact (P. Markstein,
// "Computation of elementary functions on the IBM RISC System/6000 processor", 1990): compared with __fsqrt_rn for all of them.  Smaller ones, whose residue
// has digits under 2^-149, are multiplied with 2^64 first where ANY.  Zero, infinity and NaN come out as NaN, with ANY as themselves.
// 86.6 M values: 217 us; with __fsqrt_rn 5 more, with __frcp_rn too 9.
constexpr float kSmallestFast = 0x1p-102f;
template <bool ANY>
__device__ __forceinline__ float rounded_sqrt(float x) {
    const bool small = ANY && x < kSmallestFast;
    const float big = small ? mul(x, 0x1p64f) : x;
    float y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(big));
    const float r = mul(big, y);
    float root = fma(fma(-r, r, big), mul(0.5f, y), r);
    if (small) root = mul(root, 0x1p-32f);
    return ANY && root != root ? x : root;
}
// The same way for the reciprocal of a scale, which is normal and so is its reciprocal: compared with __frcp_rn for all from 2^-126 to 2^125.
__device__ __forceinline__ float rounded_rcp(float x) {
    const float r = approx_rcp(x);
    return fma(fma(-x, r, 1.f), r, r);
}
__device__ __forceinline__ float min3(float a, float b, float c) {        // of the numbers among them
    float r;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// Largest magnitude of the warp's values (NaN if there is one), and from it the scale.  Magnitudes below 1e-30 count as zero; a block with an infinity
// or a NaN gets the scale NaN and stays so.  `factor` takes the values to 2^-120 of their share of 448, which is 448 (1 + 2^-22) at most: the scale's
// reciprocal times 2^-120.  Where that product would be subnormal (magnitudes above 2^14), the values take the reciprocal first.
__device__ __forceinline__ float block_scale(float top, float (&values)[8], float& factor) {
    uint32_t bits = __float_as_uint(top) & 0x7FFFFFFFu;
    bits = __reduce_max_sync(kFullMask, bits);
    const float amax = __uint_as_float(bits), scale = mul(amax, 1.f / 448.f);
    if (bits - 0x0DA24260u < 0x46800000u - 0x0DA24260u) {           // 1e-30 <= amax < 2^14
        factor = mul(rounded_rcp(scale), 0x1p-120f);
        return scale;
    }
    const bool none = amax < 1e-30f, bad = bits >= 0x7F800000u;
    const float inverse = none || bad ? 0.f : rounded_rcp(scale);
#pragma unroll
    for (int i = 0; i < 8; ++i) values[i] = mul(values[i], inverse);
    factor = 0x1p-120f;
    return bad ? __uint_as_float(0x7FC00000u) : none ? 0.f : scale;
}

// What holds for a tensor.
struct Step {
    float beta1, beta2, gain1, gain2;       // gain: 1 - beta
    float factor;                           // of the gradients
    float eps, decay, rate, root_correction;
    uint32_t key;
    void* p;
    const void* g;
    uint32_t first_block, n, whole;         // whole: its first blocks, all inside and aligned
};

// How a bf16 parameter is stepped: rounded to nearest, rounded with a dither, or in an fp32 copy of it (then either).
enum { kNearest = 0, kDither = 1, kMaster = 2, kMasterDither = 3 };

// A lane's share of a block as it lies in memory.
template <typename P, typename G, bool BITS8, int FORM>
struct Raw {
    uint32_t p[(FORM & kMaster) ? 8 : kWords<P>], g[kWords<G>], m[BITS8 ? 2 : 8], v[BITS8 ? 2 : 8];
    float m_scale, r_scale;
};

template <typename P, typename G, bool BITS8, int FORM, bool FULL>
__device__ __forceinline__ void load_block(const Args& a, const Step& k, uint32_t inside, int lane, Raw<P, G, BITS8, FORM>& raw) {
    const size_t arena = (size_t)k.first_block + inside;
    const uint32_t at = inside * kBlock + lane_start<BITS8>(lane);
    const int64_t left = (int64_t)k.n - at;
    load8<G, BITS8, FULL>(reinterpret_cast<const G*>(k.g) + at, left, raw.g);
    if constexpr ((FORM & kMaster) != 0) load8<float, BITS8, true>(a.master + arena * kBlock + lane_start<BITS8>(lane), 0, raw.p);
    else load8<P, BITS8, FULL>(reinterpret_cast<const P*>(k.p) + at, left, raw.p);
    if constexpr (BITS8) {
        const uint2 m = reinterpret_cast<const uint2*>(a.m)[arena * 32 + lane], v = reinterpret_cast<const uint2*>(a.v)[arena * 32 + lane];
        raw.m[0] = m.x; raw.m[1] = m.y; raw.v[0] = v.x; raw.v[1] = v.y;
    } else {
        load8<float, false, true>(reinterpret_cast<const float*>(a.m) + arena * kBlock + lane_start<false>(lane), 0, raw.m);
        load8<float, false, true>(reinterpret_cast<const float*>(a.v) + arena * kBlock + lane_start<false>(lane), 0, raw.v);
    }
}

// A lane's share of a block after the step: p, m, and v or its root.
struct Stepped {
    float p[8], m[8], v[8];
    float top_m, top_r;         // largest magnitudes
    float low_v;                // smallest second moment
};

// ANY: roots of everything; without it those below kSmallestFast may be off, and zero, infinity and NaN come out as NaN, in s.top_r as well.
template <bool ANY, typename P, typename G, bool BITS8, int FORM>
__device__ __forceinline__ void compute_as(const Step& k, const Raw<P, G, BITS8, FORM>& raw, Stepped& s) {
    s.top_m = s.top_r = 0.f;
    s.low_v = kSmallestFast;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        float m0[2], v0[2], v1[2];
        if constexpr (BITS8) {
            const int shift = 16 * ((i >> 1) & 1);
            const float2 m = decode_pair((raw.m[i / 4] >> shift) & 0xFFFFu), r = decode_pair((raw.v[i / 4] >> shift) & 0xFFFFu);
            m0[0] = m.x, m0[1] = m.y, v0[0] = r.x, v0[1] = r.y;
        } else {
            m0[0] = __uint_as_float(raw.m[i]), m0[1] = __uint_as_float(raw.m[i + 1]);
            v0[0] = __uint_as_float(raw.v[i]), v0[1] = __uint_as_float(raw.v[i + 1]);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float g = mul(value_of(raw.g, i + e), k.factor);      // before it is squared: what the factor brings back into fp32's range may have no square there
            float m, v, root;
            if constexpr (BITS8) {
                // every product, sum and root is rounded by itself: a code turns on the last bit, and one of a block's largest value changes all
                // of its scale, so that another implementation in fp32 is met bit by bit or not at all
                const float r = mul(v0[e], raw.r_scale);
                m = mul(k.beta1, mul(m0[e], raw.m_scale)) + mul(k.gain1, g);
                v = mul(k.beta2, mul(r, r)) + mul(mul(k.gain2, g), g);
                root = rounded_sqrt<ANY>(v);
                v1[e] = v;
            } else {
                m = fma(k.gain1, g, mul(m0[e], k.beta1));
                v = fma(k.gain2, mul(g, g), mul(v0[e], k.beta2));
                root = approx_sqrt(v);
            }
            const float move = mul(m, approx_rcp(fma(root, k.root_correction, k.eps)));
            s.p[i + e] = fma(value_of(raw.p, i + e), k.decay, mul(-k.rate, move));
            s.m[i + e] = m;
            s.v[i + e] = BITS8 ? root : v;
        }
        if constexpr (BITS8) {
            s.top_m = max_nan(s.top_m, fabsf(s.m[i]), fabsf(s.m[i + 1]));
            s.top_r = max_nan(s.top_r, s.v[i], s.v[i + 1]);
            s.low_v = min3(s.low_v, v1[0], v1[1]);
        }
    }
}

template <typename P, typename G, bool BITS8, int FORM>
__device__ __forceinline__ void compute(const Step& k, const Raw<P, G, BITS8, FORM>& raw, Stepped& s) {
    compute_as<false>(k, raw, s);
    if (BITS8 && (s.top_r != s.top_r || s.low_v < kSmallestFast)) compute_as<true>(k, raw, s);
}

template <typename P, typename G, bool BITS8, int FORM, bool FULL>
__device__ __forceinline__ void write(const Args& a, const Step& k, uint32_t inside, int lane, Stepped& s, float& m_scale, float& r_scale) {
    constexpr bool kCopy = (FORM & kMaster) != 0, kDithers = (FORM & kDither) != 0;
    const size_t arena = (size_t)k.first_block + inside;
    const uint32_t at = inside * kBlock + lane_start<BITS8>(lane);
    const int64_t left = (int64_t)k.n - at;
    // The word of place i is mix(i ^ key); the high halves of a lane's eight i are the same, and so is what the first shift brings down.
    uint32_t word[8];
    if constexpr (BITS8 || kDithers) {
        const uint32_t start = (at ^ k.key) ^ ((at ^ k.key) >> 16);
#pragma unroll
        for (int i = 0; i < 8; ++i) word[i] = mix_rest(start ^ (uint32_t)place_of<BITS8>(i));
    }
    if constexpr (kCopy) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(s.p[i]);
        store8<float, BITS8, true>(a.master + arena * kBlock + lane_start<BITS8>(lane), 0, w);
    }
    if constexpr (sizeof(P) == 2) {
        uint32_t w[4];
        if constexpr (kDithers) {
#pragma unroll
            for (int i = 0; i < 8; i += 2) w[i / 2] = __byte_perm(dithered(s.p[i], word[i]), dithered(s.p[i + 1], word[i + 1]), 0x7632);
            const float sum = ((s.p[0] + s.p[1]) + (s.p[2] + s.p[3])) + ((s.p[4] + s.p[5]) + (s.p[6] + s.p[7]));
            if (!isfinite(sum)) {
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    const uint32_t lo = isfinite(s.p[i]) ? w[i / 2] & 0xFFFFu : __float_as_uint(s.p[i]) >> 16;
                    const uint32_t hi = isfinite(s.p[i + 1]) ? w[i / 2] >> 16 : __float_as_uint(s.p[i + 1]) >> 16;
                    w[i / 2] = lo | (hi << 16);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; i += 2) w[i / 2] = nearest_bf16x2(s.p[i], s.p[i + 1]);
        }
        store8<P, BITS8, FULL>(reinterpret_cast<P*>(k.p) + at, left, w);
    } else {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(s.p[i]);
        store8<P, BITS8, FULL>(reinterpret_cast<P*>(k.p) + at, left, w);
    }
    if constexpr (BITS8) {
        float for_m, for_r;
        m_scale = block_scale(s.top_m, s.m, for_m);
        r_scale = block_scale(s.top_r, s.v, for_r);
        uint32_t m[2], r[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t tm[4], tr[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t zm = __float_as_uint(mul(s.m[4 * h + i], for_m));
                tm[i] = (code_of(zm, __byte_perm(word[4 * h + i], 0, 0x4324)) & 0x7FFFFFFFu) | (zm & 0x80000000u);      // the high half, one byte up
                tr[i] = code_of(__float_as_uint(mul(s.v[4 * h + i], for_r)), __byte_perm(word[4 * h + i], 0, 0x4104));   // the low half
            }
            m[h] = top_bytes(tm[0], tm[1], tm[2], tm[3]);
            r[h] = top_bytes(tr[0], tr[1], tr[2], tr[3]);
            if ((r[h] - 0x01010101u) & ~r[h] & 0x80808080u) {         // a code is zero: the smallest one where the root is not
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (s.v[4 * h + i] > 0.f && !(r[h] >> (8 * i) & 0xFFu)) r[h] |= 1u << (8 * i);
            }
        }
        reinterpret_cast<uint2*>(a.m)[arena * 32 + lane] = make_uint2(m[0], m[1]);
        reinterpret_cast<uint2*>(a.v)[arena * 32 + lane] = make_uint2(r[0], r[1]);
    } else {
        uint32_t m[8], v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) m[i] = __float_as_uint(s.m[i]), v[i] = __float_as_uint(s.v[i]);
        store8<float, false, true>(reinterpret_cast<float*>(a.m) + arena * kBlock + lane_start<false>(lane), 0, m);
        store8<float, false, true>(reinterpret_cast<float*>(a.v) + arena * kBlock + lane_start<false>(lane), 0, v);
    }
}

// Warps take runs of a tensor's blocks in turn (a.run of them, fewer where that leaves warps without any), so that the tensor's constants are
// looked up and the scales of a run come and go once; the next block's loads are under way while one is rounded and written.
// 86.6 M bf16 values with moments in 8 bits: 217 us; 315 with single blocks dealt out (nearly every one another tensor's).  One stretch of blocks a CTA,
// whose streams keep in step, took 295 where this form took 205 (before its roots were exact).
template <typename P, typename G, bool BITS8, int FORM>
__global__ void __launch_bounds__(kThreads, BITS8 ? kResident8 : kResident32)
adamw_kernel(const __grid_constant__ Args a) {
    const int lane = threadIdx.x & 31;
    Step k;
    k.factor = a.grad_factor ? *a.grad_factor : 1.f;
    k.beta1 = a.beta1;
    k.beta2 = a.beta2;
    k.gain1 = a.one_minus_beta1;
    k.gain2 = a.one_minus_beta2;
    k.eps = a.eps;
    uint32_t entry = 0, entry_end = 0;
    Raw<P, G, BITS8, FORM> raw;
    Stepped stepped;
    for (uint32_t run = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); run < a.runs; run += gridDim.x * (kThreads / 32)) {
        if (run >= entry_end) {             // the tensor that this run is part of
            uint32_t lo = entry, hi = a.count;
            while (hi - lo > 1) {
                const uint32_t mid = (lo + hi) / 2;
                if (a.entry[mid].before <= run) lo = mid; else hi = mid;
            }
            entry = lo;
            entry_end = lo + 1 < a.count ? a.entry[lo + 1].before : a.runs;
            const uint32_t step = (uint32_t)a.steps[a.entry[lo].ordinal] + 1u;
            const float t = (float)step;
            float lr = a.entry[lo].lr;
            if (a.entry[lo].lr_device) lr = *a.entry[lo].lr_device;
            k.decay = 1.f - lr * a.entry[lo].weight_decay;
            k.rate = lr / -expm1f(t * a.ln_beta1);
            k.root_correction = rsqrtf(-expm1f(t * a.ln_beta2));
            k.key = mix(mix(a.seed + step) + a.entry[lo].ordinal);
            k.p = a.entry[lo].p;
            k.g = a.entry[lo].g;
            k.first_block = a.entry[lo].first_block;
            k.n = a.entry[lo].n;
            k.whole = a.entry[lo].vectors ? k.n / kBlock : 0u;
        }
        const uint32_t first = (run - a.entry[entry].before) * a.run, last = min(first + a.run, (k.n + kBlock - 1) / kBlock);
        float m_scales = 0.f, r_scales = 0.f;               // lane j: of the run's block j
        const bool scaled = BITS8 && first + lane < last;
        if (scaled) {
            m_scales = a.m_scale[(size_t)k.first_block + first + lane];
            r_scales = a.v_scale[(size_t)k.first_block + first + lane];
        }
        bool loaded = false;
        for (uint32_t inside = first; inside < last; ++inside) {
            raw.m_scale = __shfl_sync(kFullMask, m_scales, inside - first);
            raw.r_scale = __shfl_sync(kFullMask, r_scales, inside - first);
            float m_scale = 0.f, r_scale = 0.f;
            if (inside < k.whole) {
                if (!loaded) load_block<P, G, BITS8, FORM, true>(a, k, inside, lane, raw);
                compute(k, raw, stepped);
                loaded = inside + 1 < min(last, k.whole);
                if (loaded) load_block<P, G, BITS8, FORM, true>(a, k, inside + 1, lane, raw);
                write<P, G, BITS8, FORM, true>(a, k, inside, lane, stepped, m_scale, r_scale);
            } else {
                load_block<P, G, BITS8, FORM, false>(a, k, inside, lane, raw);
                compute(k, raw, stepped);
                write<P, G, BITS8, FORM, false>(a, k, inside, lane, stepped, m_scale, r_scale);
            }
            if (BITS8 && first + lane == inside) {
                m_scales = m_scale;
                r_scales = r_scale;
            }
        }
        if (scaled) {
            a.m_scale[(size_t)k.first_block + first + lane] = m_scales;
            a.v_scale[(size_t)k.first_block + first + lane] = r_scales;
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
template <typename G, bool BITS8>
Kernel pick(dropit_dtype p, int form) {
    if (p == DROPIT_F32) return adamw_kernel<float, G, BITS8, kNearest>;
    if (form == kMasterDither) return adamw_kernel<uint16_t, G, BITS8, kMasterDither>;
    return form == kMaster ? adamw_kernel<uint16_t, G, BITS8, kMaster>
           : form == kDither ? adamw_kernel<uint16_t, G, BITS8, kDither> : adamw_kernel<uint16_t, G, BITS8, kNearest>;
}
template <bool BITS8>
Kernel pick(dropit_dtype p, dropit_dtype g, int form) { return g == DROPIT_BF16 ? pick<uint16_t, BITS8>(p, form) : pick<float, BITS8>(p, form); }

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
    a.m = s.exp_avg;
    a.v = s.exp_avg_sq;
    a.m_scale = s.exp_avg_scale;
    a.v_scale = s.exp_avg_sq_scale;
    a.master = s.master;
    a.steps = s.steps;
    a.ticket = s.ticket;
    a.grad_factor = s.grad_factor;
    const int form = (o.dither ? kDither : 0) | (s.master ? kMaster : 0);
    const Kernel kernel = o.state_bits == 8 ? pick<true>(o.param_dtype, o.grad_dtype, form) : pick<false>(o.param_dtype, o.grad_dtype, form);
    const int64_t resident = (int64_t)sm_count() * (o.state_bits == 8 ? kResident8 : kResident32);
    int i = 0;
    while (i < count) {
        a.count = 0;
        int64_t blocks = 0;
        for (; i < count && a.count < kMaxEntries; ++i) {
            const dropit_adamw_tensor& t = tensors[i];
            if (t.n == 0) continue;
            if (blocks + blocks_of(t.n) > INT32_MAX) break;
            const bool vectors = (reinterpret_cast<uintptr_t>(t.param) | reinterpret_cast<uintptr_t>(t.grad)) % 16 == 0;
            a.entry[a.count++] = {t.param, t.grad, t.lr_device, (uint32_t)t.first_block, 0u, (uint32_t)t.n, (uint32_t)t.ordinal, t.lr, t.weight_decay,
                                  vectors ? 1u : 0u, 0u};
            blocks += blocks_of(t.n);
        }
        if (!a.count) break;
        a.run = kMaxRun;                                       // every warp gets two runs at least, or runs are single blocks
        while (a.run > 1 && blocks < 2 * (int64_t)a.run * resident * (kThreads / 32)) a.run /= 2;
        a.runs = 0;
        for (uint32_t e = 0; e < a.count; ++e) {
            a.entry[e].before = a.runs;
            a.runs += (uint32_t)((blocks_of(a.entry[e].n) + a.run - 1) / a.run);
        }
        const int64_t grid = std::min<int64_t>((a.runs + kThreads / 32 - 1) / (kThreads / 32), resident);
        kernel<<<(unsigned)grid, kThreads, 0, as_stream(cuda_stream)>>>(a);
        const dropit_status status = check_launch();
        if (status != DROPIT_OK) return status;
    }
    return DROPIT_OK;
}
