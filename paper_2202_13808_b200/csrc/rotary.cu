// Rotary positions with several axes (rows and columns of an image; time, height and width of a video) on queries and keys.
// Pair j of a head turns by p[axis(j)] * theta^e(j): (a, b) -> (a cos - b sin, a sin + b cos); the gradient is the same with -sin.
//
// The angle is formed in turns: a whole-number position times the pair's turns per position as a 64-bit binary fraction, wrapping.
// The product's high word is the angle's place within its turn, exact to 2^-32 for positions up to 2^31, where an fp32 product has
// lost every digit (2^24 steps of one radian are known to a radian).  Positions that are fp32 take the product in 64-bit floats.
//
// Bound by HBM: every value is read and written once.  The angles of a block's tokens are formed once, in shared memory, and
// serve all heads of queries and keys; one launch does both.
#include <math.h>

#include <algorithm>

#include "common.cuh"

namespace dropit {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxAngles = 1024;            // angles of one block's tokens: 8 KB of shared memory

struct RotaryTensor {
    const void* in;
    void* out;
    int64_t in_batch, in_token, in_head, out_batch, out_token, out_head;
    int heads;
};
struct RotaryArgs {
    RotaryTensor t[2];                      // queries, keys
    const void* positions;
    int64_t pos_batch, pos_token, pos_axis;
    int64_t tokens;                         // batch * length
    int length, head_dim, tokens_per_block;
    float sign;                             // -1: the inverse rotation
    dropit_position_type position_type;
    dropit_rotary_plan plan;
};

template <int BYTES> struct Bits;
template <> struct Bits<2> { using type = uint16_t; };
template <> struct Bits<4> { using type = uint32_t; };
template <> struct Bits<8> { using type = uint2; };
template <> struct Bits<16> { using type = uint4; };

template <typename T, int N>
struct Values {
    union {
        typename Bits<N * sizeof(T)>::type bits;
        T v[N];
    };
    __device__ Values() {}
};
__device__ __forceinline__ float to_float(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ void from_float(float v, uint16_t& out) {
    uint16_t r;
    asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(r) : "f"(v));
    out = r;
}
__device__ __forceinline__ void from_float(float v, float& out) { out = v; }

// The angle in half turns, within [-1, 1].
__device__ __forceinline__ float half_turns(const RotaryArgs& a, int64_t at, uint64_t turns) {
    if (a.position_type == DROPIT_POSITION_F32) {
        const double t = (double)reinterpret_cast<const float*>(a.positions)[at] * ((double)turns * 0x1p-64);
        return (float)(2.0 * (t - rint(t)));
    }
    const int64_t p = a.position_type == DROPIT_POSITION_I64 ? reinterpret_cast<const int64_t*>(a.positions)[at]
                                                            : (int64_t)reinterpret_cast<const int32_t*>(a.positions)[at];
    return (float)(int32_t)(((uint64_t)p * turns) >> 32) * 0x1p-31f;
}

// A unit is VP pairs of one head (two vectors of VP values), or VP of the values behind the rotated ones, which are copied.  A thread keeps its
// place in the head and steps through the rows (token, head) of the block without dividing; two rows' loads are in flight at a time.
template <typename T, int VP, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads)
rotary_kernel(const __grid_constant__ RotaryArgs a) {
    extern __shared__ float2 angles[];                                   // [tokens][pairs], then the tokens' places
    const int pairs = a.plan.pairs;
    const int64_t first = (int64_t)blockIdx.x * a.tokens_per_block;
    const int tokens = (int)min((int64_t)a.tokens_per_block, a.tokens - first);
    longlong4* places = reinterpret_cast<longlong4*>(angles + (a.tokens_per_block * pairs + 3) / 4 * 4);   // q in, q out, k in, k out
    uint64_t* turns = reinterpret_cast<uint64_t*>(places + a.tokens_per_block);                          // [pairs], then the pairs' axes
    uint8_t* axes = reinterpret_cast<uint8_t*>(turns + pairs);
    // The plan's constants are read one address a warp: 32 different ones take 32 turns.
    for (int j = threadIdx.x >> 5; j < pairs; j += kThreads / 32) {
        const uint64_t t = a.plan.turns[j];
        const uint8_t x = a.plan.axis[j];
        if ((threadIdx.x & 31) == 0) turns[j] = t, axes[j] = x;
    }
    for (int i = threadIdx.x; i < tokens; i += kThreads) {
        const int64_t token = first + i, batch = token / a.length, at = token - batch * a.length;
        places[i] = make_longlong4(batch * a.t[0].in_batch + at * a.t[0].in_token, batch * a.t[0].out_batch + at * a.t[0].out_token,
                                   batch * a.t[1].in_batch + at * a.t[1].in_token, batch * a.t[1].out_batch + at * a.t[1].out_token);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < tokens * pairs; i += kThreads) {
        const int local = i / pairs, j = i - local * pairs;
        const int64_t token = first + local, batch = token / a.length;
        float2 cs;
        sincospif(half_turns(a, batch * a.pos_batch + (token - batch * a.length) * a.pos_token + axes[j] * a.pos_axis, turns[j]), &cs.y, &cs.x);
        cs.y *= a.sign;
        angles[i] = cs;
    }
    __syncthreads();
    const int rotating = pairs / VP;
    const int units = rotating + (a.head_dim - 2 * pairs) / VP;
    const int heads = a.t[0].heads + a.t[1].heads;
    using Vec = Values<T, VP>;
    using B = typename Bits<VP * sizeof(T)>::type;
    const RotaryTensor q = a.t[0], k = a.t[1];
    for (int unit0 = 0; unit0 < units; unit0 += kThreads) {              // one round, unless a head has more units than the block threads
        const int width = min(units - unit0, kThreads), step = kThreads / width;
        const int unit = unit0 + threadIdx.x % width;
        int head = threadIdx.x / width, local = 0;
        if (head >= step) continue;
        const int c0 = unit >= rotating ? 2 * pairs + (unit - rotating) * VP : INTERLEAVED ? 2 * unit * VP : unit * VP;
        const int c1 = INTERLEAVED ? c0 + VP : pairs + c0;
        const bool copies = unit >= rotating;
        while (head >= heads) head -= heads, ++local;
        while (local < tokens) {
            const T* in[2];
            T* out[2];
            int token[2], live = 0;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                token[r] = local;
                if (local < tokens) {
                    const longlong4 place = places[local];
                    const bool key = head >= q.heads;
                    const int h = key ? head - q.heads : head;
                    in[r] = reinterpret_cast<const T*>(key ? k.in : q.in) + (key ? place.z : place.x) + h * (key ? k.in_head : q.in_head);
                    out[r] = reinterpret_cast<T*>(key ? k.out : q.out) + (key ? place.w : place.y) + h * (key ? k.out_head : q.out_head);
                    ++live;
                    head += step;
                    while (head >= heads) head -= heads, ++local;
                }
            }
            Vec x[2], y[2];
#pragma unroll
            for (int r = 0; r < 2; ++r)
                if (r < live) {
                    x[r].bits = *reinterpret_cast<const B*>(in[r] + c0);
                    if (!copies) y[r].bits = *reinterpret_cast<const B*>(in[r] + c1);
                }
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                if (r >= live) break;
                if (!copies) {
                    const float2* cs = angles + token[r] * pairs + unit * VP;
#pragma unroll
                    for (int e = 0; e < VP; ++e) {
                        // halves: pair e is (x[e], y[e]); neighbours: values 2e and 2e + 1 of x followed by y
                        T& one = INTERLEAVED ? (2 * e < VP ? x[r].v[2 * e % VP] : y[r].v[2 * e % VP]) : x[r].v[e];
                        T& two = INTERLEAVED ? (2 * e + 1 < VP ? x[r].v[(2 * e + 1) % VP] : y[r].v[(2 * e + 1) % VP]) : y[r].v[e];
                        const float u = to_float(one), v = to_float(two);
                        from_float(u * cs[e].x - v * cs[e].y, one);
                        from_float(u * cs[e].y + v * cs[e].x, two);
                    }
                    *reinterpret_cast<B*>(out[r] + c1) = y[r].bits;
                }
                *reinterpret_cast<B*>(out[r] + c0) = x[r].bits;
            }
        }
    }
}

template <typename T, int VP>
void launch(const RotaryArgs& a, unsigned blocks, cudaStream_t stream) {
    const size_t smem = (size_t)((a.tokens_per_block * a.plan.pairs + 3) / 4 * 4) * sizeof(float2) + (size_t)a.tokens_per_block * sizeof(longlong4) + (size_t)a.plan.pairs * 9;
    if (a.plan.interleaved) rotary_kernel<T, VP, true><<<blocks, kThreads, smem, stream>>>(a);
    else rotary_kernel<T, VP, false><<<blocks, kThreads, smem, stream>>>(a);
}

// Whether vectors of `n` values of `size` bytes fit everywhere.
bool takes(const RotaryArgs& a, int n, int size) {
    if (a.plan.pairs % n || a.head_dim % n) return false;
    for (const RotaryTensor& t : a.t) {
        if (!t.heads) continue;
        const uintptr_t base = reinterpret_cast<uintptr_t>(t.in) | reinterpret_cast<uintptr_t>(t.out);
        const int64_t strides = t.in_batch | t.in_token | t.in_head | t.out_batch | t.out_token | t.out_head;
        if (base % (uintptr_t)(n * size) || strides % n) return false;
    }
    return true;
}

}  // namespace

}  // namespace dropit

using namespace dropit;

extern "C" dropit_status dropit_rotary_make_plan(int head_dim, const int* sections, int axes, double theta, int shared, int interleaved,
                                                 dropit_rotary_plan* plan) {
    if (!plan || !sections || axes < 1 || axes > DROPIT_ROTARY_MAX_AXES || head_dim < 2 || !(theta >= 1) || !isfinite(theta))
        return DROPIT_ERR_INVALID_ARG;
    int64_t rotated = 0;
    for (int s = 0; s < axes; ++s) {
        if (sections[s] < 0 || sections[s] % 2) return DROPIT_ERR_INVALID_ARG;
        rotated += sections[s];
    }
    if (rotated < 2 || rotated > head_dim) return DROPIT_ERR_INVALID_ARG;
    if (rotated > 2 * DROPIT_ROTARY_MAX_PAIRS) return DROPIT_ERR_UNSUPPORTED;
    plan->head_dim = head_dim;
    plan->pairs = (int)(rotated / 2);
    plan->axes = axes;
    plan->interleaved = interleaved != 0;
    int j = 0;
    for (int s = 0; s < axes; ++s) {
        for (int i = 0; i < sections[s] / 2; ++i, ++j) {
            const double exponent = shared ? 2.0 * j / (double)rotated : 2.0 * i / (double)sections[s];
            // Turns per position, at most 1 / (2 pi), as a fraction of 2^64.
            const long double part = powl((long double)theta, -(long double)exponent) / 6.283185307179586476925286766559L;
            const long double high = floorl(part * 0x1p32L), low = floorl((part * 0x1p32L - high) * 0x1p32L + 0.5L);
            plan->turns[j] = ((uint64_t)high << 32) + (uint64_t)low;
            plan->axis[j] = (uint8_t)s;
        }
    }
    for (; j < DROPIT_ROTARY_MAX_PAIRS; ++j) plan->turns[j] = 0, plan->axis[j] = 0;
    return DROPIT_OK;
}

extern "C" dropit_status dropit_rotary(const dropit_rotary_plan* plan, int64_t batch, int64_t length, const dropit_rotary_tensor* q,
                                       const dropit_rotary_tensor* k, const void* positions, dropit_position_type position_type,
                                       int64_t pos_batch, int64_t pos_token, int64_t pos_axis, dropit_dtype dtype, int inverse,
                                       void* cuda_stream) {
    if (!plan || !q || batch < 0 || length < 0 || length > INT32_MAX) return DROPIT_ERR_INVALID_ARG;
    if (plan->pairs < 1 || plan->pairs > DROPIT_ROTARY_MAX_PAIRS || plan->head_dim < 2 * plan->pairs) return DROPIT_ERR_INVALID_ARG;
    if (dtype != DROPIT_BF16 && dtype != DROPIT_F32) return DROPIT_ERR_INVALID_ARG;
    if (position_type != DROPIT_POSITION_I32 && position_type != DROPIT_POSITION_I64 && position_type != DROPIT_POSITION_F32)
        return DROPIT_ERR_INVALID_ARG;
    const int size = dtype == DROPIT_BF16 ? 2 : 4;
    RotaryArgs a = {};
    int64_t heads = 0;
    for (int i = 0; i < 2; ++i) {
        const dropit_rotary_tensor* t = i ? k : q;
        if (!t) continue;
        if (t->heads < 0) return DROPIT_ERR_INVALID_ARG;
        heads += t->heads;
        a.t[i] = {t->in, t->out, t->in_batch, t->in_token, t->in_head, t->out_batch, t->out_token, t->out_head, t->heads};
        if (t->heads && batch && length &&
            (!t->in || !t->out || (reinterpret_cast<uintptr_t>(t->in) | reinterpret_cast<uintptr_t>(t->out)) % (uintptr_t)size))
            return DROPIT_ERR_INVALID_ARG;
    }
    if (length && batch > INT64_MAX / length) return DROPIT_ERR_INVALID_ARG;
    const int64_t tokens = batch * length;
    if (tokens == 0 || heads == 0) return DROPIT_OK;
    if (!positions || reinterpret_cast<uintptr_t>(positions) % (position_type == DROPIT_POSITION_I64 ? 8 : 4)) return DROPIT_ERR_INVALID_ARG;
    if (heads * plan->head_dim > (1 << 20)) return DROPIT_ERR_UNSUPPORTED;      // a block's work is counted in 32 bits
    a.positions = positions;
    a.pos_batch = pos_batch;
    a.pos_token = pos_token;
    a.pos_axis = pos_axis;
    a.tokens = tokens;
    a.length = (int)length;
    a.head_dim = plan->head_dim;
    a.sign = inverse ? -1.f : 1.f;
    a.position_type = position_type;
    a.plan = *plan;
    // Vectors of 16 bytes, else of 8, else single values.
    int vec = 1;
    for (int n = 16 / size; n >= 4; n /= 2)
        if (takes(a, n, size)) { vec = n; break; }
    // Four units a thread, as far as the angles fit and every SM has blocks.
    const int64_t units = heads * ((plan->head_dim - plan->pairs) / vec);
    int64_t per_block = (4 * kThreads + units - 1) / units;
    per_block = std::min<int64_t>(std::min<int64_t>(per_block, kMaxAngles / plan->pairs), 256);
    per_block = std::min<int64_t>(per_block, std::max<int64_t>(1, tokens / (2 * sm_count())));
    a.tokens_per_block = (int)std::max<int64_t>(1, per_block);
    const int64_t blocks = (tokens + a.tokens_per_block - 1) / a.tokens_per_block;
    if (blocks > INT32_MAX) return DROPIT_ERR_UNSUPPORTED;
    cudaStream_t stream = as_stream(cuda_stream);
    if (dtype == DROPIT_BF16) {
        if (vec == 8) launch<uint16_t, 8>(a, (unsigned)blocks, stream);
        else if (vec == 4) launch<uint16_t, 4>(a, (unsigned)blocks, stream);
        else launch<uint16_t, 1>(a, (unsigned)blocks, stream);
    } else {
        if (vec == 4) launch<float, 4>(a, (unsigned)blocks, stream);
        else launch<float, 1>(a, (unsigned)blocks, stream);
    }
    return check_launch();
}
