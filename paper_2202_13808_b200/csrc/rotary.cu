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
constexpr int kMaxAngles = 640;             // angles of one block's tokens: 5 KB of shared memory
constexpr int kMaxTokens = 64;              // of a block
constexpr int kResident = 5;                // blocks of an SM
constexpr int kMaxRows = 512;               // rows (token, head) whose places are looked up at a time

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

// N neighbouring values of a head in memory and as fp32.
template <typename T, int N> struct Vec;
template <int N> struct Vec<uint16_t, N> {
    uint32_t w[N / 2];
    __device__ void load(const uint16_t* p) {
        if constexpr (N == 8) {
            const uint4 q = *reinterpret_cast<const uint4*>(p);
            w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
        } else {
            const uint2 q = *reinterpret_cast<const uint2*>(p);
            w[0] = q.x; w[1] = q.y;
        }
    }
    __device__ void store(uint16_t* p) const {
        if constexpr (N == 8) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        else *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    }
    __device__ float get(int i) const { return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16); }
    __device__ void set2(int i, float lo, float hi) { asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i / 2]) : "f"(hi), "f"(lo)); }
};
template <> struct Vec<uint16_t, 1> {
    uint32_t w;
    __device__ void load(const uint16_t* p) { w = *p; }
    __device__ void store(uint16_t* p) const { *p = (uint16_t)w; }
    __device__ float get(int) const { return __uint_as_float(w << 16); }
    __device__ void set(float v) { asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(0.f), "f"(v)); }
};
template <int N> struct Vec<float, N> {
    float v[N];
    __device__ void load(const float* p) {
        if constexpr (N == 4) {
            const float4 q = *reinterpret_cast<const float4*>(p);
            v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
        } else {
            v[0] = *p;
        }
    }
    __device__ void store(float* p) const {
        if constexpr (N == 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
        else *p = v[0];
    }
    __device__ float get(int i) const { return v[i]; }
    __device__ void set2(int i, float lo, float hi) { v[i] = lo; v[i + 1] = hi; }
    __device__ void set(float x) { v[0] = x; }
};

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

// Where pair j of a token has its cosine and sine: two pairs are 16 bytes, and the same two of neighbouring units lie side by side, so that the units' reads
// do not meet in the banks.
template <int VP>
__device__ __forceinline__ int angle_place(int j, int units) {
    if constexpr (VP == 1) return j;
    else return ((j % VP / 2) * units + j / VP) * 2 + (j & 1);
}

// A unit is VP pairs of one head (two vectors of VP values), or VP of the values behind the rotated ones, which are copied.  A thread keeps its
// place in the head and steps through the rows (token, head) of the block, whose places are looked up once for all units; two rows' loads are in
// flight at a time, the first of them while the angles are formed.
template <typename T, int VP, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads, kResident)
rotary_kernel(const __grid_constant__ RotaryArgs a) {
    extern __shared__ __align__(16) float2 angles[];                    // [token][angle_place]
    __shared__ ulonglong2 places[kMaxRows];                              // of a row: in, out
    __shared__ int token_of[kMaxRows];
    __shared__ int64_t starts[5][kMaxTokens];                            // of a token: queries in and out, keys in and out, positions
    __shared__ uint64_t turns[DROPIT_ROTARY_MAX_PAIRS];
    __shared__ uint8_t axes[DROPIT_ROTARY_MAX_PAIRS];
    const int pairs = a.plan.pairs, rotating = pairs / VP, units = rotating + (a.head_dim - 2 * pairs) / VP;
    const int64_t first = (int64_t)blockIdx.x * a.tokens_per_block;
    const int tokens = (int)min((int64_t)a.tokens_per_block, a.tokens - first);
    const int q_heads = a.t[0].heads, heads = q_heads + a.t[1].heads, rows = tokens * heads;
    // The plan's constants are read one address a warp: 32 different ones take 32 turns.
    for (int j = threadIdx.x >> 5; j < pairs; j += kThreads / 32) {
        const uint64_t t = a.plan.turns[j];
        const uint8_t x = a.plan.axis[j];
        if ((threadIdx.x & 31) == 0) turns[j] = t, axes[j] = x;
    }
    for (int i = threadIdx.x; i < tokens; i += kThreads) {
        const int64_t token = first + i, batch = token / a.length, at = token - batch * a.length;
        starts[0][i] = batch * a.t[0].in_batch + at * a.t[0].in_token;
        starts[1][i] = batch * a.t[0].out_batch + at * a.t[0].out_token;
        starts[2][i] = batch * a.t[1].in_batch + at * a.t[1].in_token;
        starts[3][i] = batch * a.t[1].out_batch + at * a.t[1].out_token;
        starts[4][i] = batch * a.pos_batch + at * a.pos_token;
    }
    __syncthreads();
    // Quotients of up to kMaxRows rows or kMaxAngles angles: the product's error is far below half a divisor's share.
    const float per_heads = 1.f / (float)heads, per_pairs = 1.f / (float)pairs;
    auto look_up = [&](int row0) {
        for (int i = threadIdx.x; i < min(kMaxRows, rows - row0); i += kThreads) {
            const int row = row0 + i;                                    // more than kMaxRows heads come with one token a block
            const int local = tokens == 1 ? 0 : (int)(((float)row + 0.5f) * per_heads), head = row - local * heads;
            const T* in;
            T* out;
            if (head < q_heads) {
                in = reinterpret_cast<const T*>(a.t[0].in) + starts[0][local] + head * a.t[0].in_head;
                out = reinterpret_cast<T*>(a.t[0].out) + starts[1][local] + head * a.t[0].out_head;
            } else {
                in = reinterpret_cast<const T*>(a.t[1].in) + starts[2][local] + (head - q_heads) * a.t[1].in_head;
                out = reinterpret_cast<T*>(a.t[1].out) + starts[3][local] + (head - q_heads) * a.t[1].out_head;
            }
            places[i] = make_ulonglong2(reinterpret_cast<uint64_t>(in), reinterpret_cast<uint64_t>(out));
            token_of[i] = local;
        }
    };
    bool angles_there = false;
    for (int row0 = 0; row0 < rows; row0 += kMaxRows) {
        if (row0) __syncthreads();
        look_up(row0);
        __syncthreads();
        const int here = min(rows - row0, kMaxRows);
        for (int unit0 = 0; unit0 < units; unit0 += kThreads) {          // one round, unless a head has more units than the block threads
            const int width = min(units - unit0, kThreads), step = kThreads / width;
            const int unit = unit0 + threadIdx.x % width, slot = threadIdx.x / width;
            const bool copies = unit >= rotating;
            const int c0 = copies ? 2 * pairs + (unit - rotating) * VP : INTERLEAVED ? 2 * unit * VP : unit * VP;
            const int c1 = INTERLEAVED ? c0 + VP : pairs + c0;
            Vec<T, VP> x[2], y[2];
            uint64_t out[2];
            int row = slot < step ? slot : here;
            auto load = [&](int r, int at) {
                if (at >= here) return;
                const ulonglong2 place = places[at];
                const T* in = reinterpret_cast<const T*>(place.x);
                out[r] = place.y;
                x[r].load(in + c0);
                if (!copies) y[r].load(in + c1);
            };
            load(0, row);
            load(1, row + step);
            if (!angles_there) {
                for (int i = threadIdx.x; i < tokens * pairs; i += kThreads) {
                    const int local = (int)(((float)i + 0.5f) * per_pairs), j = i - local * pairs;
                    float2 cs;
                    sincospif(half_turns(a, starts[4][local] + axes[j] * a.pos_axis, turns[j]), &cs.y, &cs.x);
                    cs.y *= a.sign;
                    angles[local * pairs + angle_place<VP>(j, rotating)] = cs;
                }
                __syncthreads();
                angles_there = true;
            }
            for (; row < here; row += 2 * step) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    if (row + r * step >= here) continue;
                    T* to = reinterpret_cast<T*>(out[r]);
                    if (!copies) {
                        const float2* of_token = angles + token_of[row + r * step] * pairs;
                        if constexpr (VP == 1) {
                            const float2 cs = of_token[unit];
                            const float u = x[r].get(0), v = y[r].get(0);
                            x[r].set(u * cs.x - v * cs.y);
                            y[r].set(u * cs.y + v * cs.x);
                        } else {
#pragma unroll
                            for (int e = 0; e < VP; e += 2) {
                                const float4 cs = *reinterpret_cast<const float4*>(of_token + ((e / 2) * rotating + unit) * 2);
                                if constexpr (INTERLEAVED) {        // pair e is two neighbours of x followed by y
                                    Vec<T, VP>& home = 2 * e < VP ? x[r] : y[r];
                                    const int i = 2 * e % VP;
                                    const float u0 = home.get(i), v0 = home.get(i + 1), u1 = home.get(i + 2), v1 = home.get(i + 3);
                                    home.set2(i, u0 * cs.x - v0 * cs.y, u0 * cs.y + v0 * cs.x);
                                    home.set2(i + 2, u1 * cs.z - v1 * cs.w, u1 * cs.w + v1 * cs.z);
                                } else {
                                    const float u0 = x[r].get(e), v0 = y[r].get(e), u1 = x[r].get(e + 1), v1 = y[r].get(e + 1);
                                    x[r].set2(e, u0 * cs.x - v0 * cs.y, u1 * cs.z - v1 * cs.w);
                                    y[r].set2(e, u0 * cs.y + v0 * cs.x, u1 * cs.w + v1 * cs.z);
                                }
                            }
                        }
                        y[r].store(to + c1);
                    }
                    x[r].store(to + c0);
                    load(r, row + (2 + r) * step);       // on its way while the other row is turned
                }
            }
        }
    }
}

template <typename T, int VP>
void launch(const RotaryArgs& a, unsigned blocks, cudaStream_t stream) {
    const size_t smem = (size_t)a.tokens_per_block * a.plan.pairs * sizeof(float2);
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
    if (plan->axes < 1 || plan->axes > DROPIT_ROTARY_MAX_AXES) return DROPIT_ERR_INVALID_ARG;
    uint8_t last_axis = 0;                              // positions are read by them
    for (int j = 0; j < plan->pairs; ++j) last_axis = std::max(last_axis, plan->axis[j]);
    if (last_axis >= plan->axes) return DROPIT_ERR_INVALID_ARG;
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
    // As many tokens as there is room for, in whole waves of blocks: 12608 tokens of 24 heads 17 us in one wave, 20 with a second one that is nearly empty.
    const int64_t room = std::max<int64_t>(1, std::min<int64_t>(kMaxTokens, std::min<int64_t>(kMaxAngles / plan->pairs, kMaxRows / heads))), wave = (int64_t)kResident * sm_count();
    const int64_t waves = (tokens + room * wave - 1) / (room * wave), per_block = (tokens + waves * wave - 1) / (waves * wave);
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
