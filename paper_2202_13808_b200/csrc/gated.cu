// The gated linear (see include/dropit.h): entry points, the element-wise part of the backward pass, and the products in fp32 FMA.
#include "gated.h"

#include <algorithm>

#include "layer_ops.h"

namespace dropit {

namespace {

__device__ __forceinline__ float to_float(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void put(uint16_t* p, float v) { *p = (uint16_t)pack_bf16(v, 0.f); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }

// ---------------------------------------------------------------------------------------------
// Products in fp32 FMA: fp32 tensors, and bf16 widths that the tensor-core kernels do not take.  32 x 32 outputs a CTA, so that small layers fill the SMs; its
// four groups of 64 threads share out the summed axis, 16 of every 64 values each, 4 x 4 outputs a thread (two of them in the forward pass: the
// gate's and the other), and add up in order at the end.  The next 64 values are on their way while these are multiplied.
// A tile lies as [k][32] with its quads of outputs exchanged by k mod 8: conflict-free both for the transposing stores and for the reads.
// Up to four CTAs of a cluster share out the summed axis too, where that evens out the SMs; the first one adds what the others send.
// fp32 197 x 387 -> 771 and back: forward 23 us, dx 17 (one CTA a tile: 24 and 36; 64 x 64 tiles without groups: 87 and 265).
// ---------------------------------------------------------------------------------------------
constexpr int kTile = 32, kStep = 64, kFmaThreads = 256, kGroups = 4;
struct __align__(16) FmaTile {
    float v[kStep][kTile];
    __device__ float& at(int k, int c) { return v[k][((c >> 2) ^ (k & 7)) * 4 + (c & 3)]; }
    __device__ float4 quad(int k, int q) const { return *reinterpret_cast<const float4*>(&v[k][(q ^ (k & 7)) * 4]); }
};

// kStep values of 32 rows of a row-major matrix [rows x K] from (row0, k0): 8 values x 4 rows a warp and load.  (All matrices have fewer than 2^31 values.)
template <typename T>
__device__ __forceinline__ void fetch_rows(float (&r)[8], const T* a, uint32_t row0, uint32_t rows, uint32_t k0, uint32_t K) {
    const uint32_t k = k0 + (threadIdx.x >> 5) * 8 + (threadIdx.x & 7), row = row0 + ((threadIdx.x >> 3) & 3);
    const uint32_t there = k < K && row < rows ? min((rows - row + 3) / 4, 8u) : 0u, at = row * K + k;
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) r[j] = j < there ? to_float(a[at + 4 * j * K]) : 0.f;
}
__device__ __forceinline__ void stage_rows(FmaTile& t, const float (&r)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) t.at((threadIdx.x >> 5) * 8 + (threadIdx.x & 7), ((threadIdx.x >> 3) & 3) + 4 * j) = r[j];
}
// kStep rows x 32 columns of a row-major matrix [K x cols]
template <typename T>
__device__ __forceinline__ void fetch_cols(float (&r)[8], const T* b, uint32_t k0, uint32_t K, uint32_t col0, uint32_t cols) {
    const uint32_t c = col0 + (threadIdx.x & 31), k = k0 + (threadIdx.x >> 5);
    const uint32_t there = c < cols && k < K ? min((K - k + 7) / 8, 8u) : 0u, at = k * cols + c;
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) r[j] = j < there ? to_float(b[at + 8 * j * cols]) : 0.f;
}
__device__ __forceinline__ void stage_cols(FmaTile& t, const float (&r)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) t.at((threadIdx.x >> 5) + 8 * j, threadIdx.x & 31) = r[j];
}
__device__ __forceinline__ void multiply(float (&acc)[4][4], const float4& p, const float4& q) {
    const float pv[4] = {p.x, p.y, p.z, p.w}, qv[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(pv[i], qv[j], acc[i][j]);
}
// The groups' sums of output (r, c) of the tile for thread i's outputs i, i + 256, ..: added in the groups' order.
__device__ __forceinline__ void join(float (&out)[4], const float (&acc)[4][4], float* room) {
    const int group = threadIdx.x / 64, ty = (threadIdx.x / 8) % 8, tx = threadIdx.x % 8;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(room + group * kTile * kTile + (ty * 4 + i) * kTile + tx * 4) = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
    __syncthreads();
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        float s = 0.f;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) s += room[g * kTile * kTile + n * kFmaThreads + threadIdx.x];
        out[n] = s;
    }
}

// The part of the summed axis that a CTA of a cluster takes, in whole steps.
__device__ __forceinline__ void my_part(uint32_t K, uint32_t& begin, uint32_t& end) {
    const uint32_t steps = (K + kStep - 1) / kStep;
    begin = steps * blockIdx.z / gridDim.z * kStep;
    end = min(K, steps * (blockIdx.z + 1) / gridDim.z * kStep);
}
// Sums of the cluster's CTAs in the first one, added in order; false in the others.  room: of every CTA, kCluster - 1 times N tiles.
constexpr int kMaxCluster = 4;
template <int N>
__device__ __forceinline__ bool gather(float (&sums)[N][4], float* room) {
    if (gridDim.z == 1) return true;
    ptx::cluster_sync_all();             // the room is free in all of them
    if (blockIdx.z) {
        const uint32_t to = ptx::map_shared_to_cta(ptx::smem_u32(room + (blockIdx.z - 1) * N * kTile * kTile + threadIdx.x), 0);
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int n = 0; n < 4; ++n) ptx::st_cluster_u32(to + (t * kTile * kTile + n * kFmaThreads) * 4, __float_as_uint(sums[t][n]));
    }
    ptx::cluster_sync_all();
    if (blockIdx.z) return false;
    for (int r = 0; r < (int)gridDim.z - 1; ++r)
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int n = 0; n < 4; ++n) sums[t][n] += room[(r * N + t) * kTile * kTile + n * kFmaThreads + threadIdx.x];
    return true;
}

template <typename T, int GATE>
__global__ void __launch_bounds__(kFmaThreads, 2)
gated_fma_kernel(const T* __restrict__ x, const T* __restrict__ w, const T* __restrict__ bias, uint32_t M, uint32_t C, uint32_t H, T* __restrict__ h,
                 T* __restrict__ gu) {
    __shared__ FmaTile tiles[3];
    const uint32_t row0 = blockIdx.x * kTile, col0 = blockIdx.y * kTile;
    const int group = threadIdx.x / 64, ty = (threadIdx.x / 8) % 8, tx = threadIdx.x % 8;
    float g[4][4] = {}, u[4][4] = {}, ra[8], rg[8], ru[8];
    uint32_t begin, end;
    my_part(C, begin, end);
    fetch_rows(ra, x, row0, M, begin, C);
    fetch_rows(rg, w, col0, H, begin, C);
    fetch_rows(ru, w + (size_t)H * C, col0, H, begin, C);
    for (uint32_t k0 = begin; k0 < end; k0 += kStep) {
        __syncthreads();
        stage_rows(tiles[0], ra);
        stage_rows(tiles[1], rg);
        stage_rows(tiles[2], ru);
        __syncthreads();
        if (k0 + kStep < end) {
            fetch_rows(ra, x, row0, M, k0 + kStep, C);
            fetch_rows(rg, w, col0, H, k0 + kStep, C);
            fetch_rows(ru, w + (size_t)H * C, col0, H, k0 + kStep, C);
        }
#pragma unroll 8
        for (int i = 0; i < kStep / kGroups; ++i) {
            const int k = group * (kStep / kGroups) + i;
            const float4 p = tiles[0].quad(k, ty);
            multiply(g, p, tiles[1].quad(k, tx));
            multiply(u, p, tiles[2].quad(k, tx));
        }
    }
    float sums[2][4];
    join(sums[0], g, &tiles[0].v[0][0]);
    join(sums[1], u, &tiles[0].v[0][0]);
    if (!gather(sums, &tiles[0].v[0][0])) return;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        const size_t r = row0 + (n * kFmaThreads + threadIdx.x) / kTile, c = col0 + threadIdx.x % kTile;
        if (r >= M || c >= H) continue;
        const float gv = sums[0][n] + (bias ? to_float(bias[c]) : 0.f), uv = sums[1][n] + (bias ? to_float(bias[H + c]) : 0.f);
        put(h + r * H + c, gate_value<GATE, false>(gv) * uv);
        if (gu) {
            put(gu + r * 2 * H + c, gv);
            put(gu + r * 2 * H + H + c, uv);
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kFmaThreads, 2)
input_grad_fma_kernel(const T* __restrict__ dgu, const T* __restrict__ w, uint32_t M, uint32_t C, uint32_t K, T* __restrict__ dx) {
    __shared__ FmaTile tiles[2];
    const uint32_t row0 = blockIdx.x * kTile, col0 = blockIdx.y * kTile;
    const int group = threadIdx.x / 64, ty = (threadIdx.x / 8) % 8, tx = threadIdx.x % 8;
    float acc[4][4] = {}, ra[8], rb[8];
    uint32_t begin, end;
    my_part(K, begin, end);
    fetch_rows(ra, dgu, row0, M, begin, K);
    fetch_cols(rb, w, begin, K, col0, C);
    for (uint32_t k0 = begin; k0 < end; k0 += kStep) {
        __syncthreads();
        stage_rows(tiles[0], ra);
        stage_cols(tiles[1], rb);
        __syncthreads();
        if (k0 + kStep < end) {
            fetch_rows(ra, dgu, row0, M, k0 + kStep, K);
            fetch_cols(rb, w, k0 + kStep, K, col0, C);
        }
#pragma unroll 8
        for (int i = 0; i < kStep / kGroups; ++i) {
            const int k = group * (kStep / kGroups) + i;
            multiply(acc, tiles[0].quad(k, ty), tiles[1].quad(k, tx));
        }
    }
    float sums[1][4];
    join(sums[0], acc, &tiles[0].v[0][0]);
    if (!gather(sums, &tiles[0].v[0][0])) return;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        const size_t r = row0 + (n * kFmaThreads + threadIdx.x) / kTile, c = col0 + threadIdx.x % kTile;
        if (r < M && c < C) put(dx + r * C + c, sums[0][n]);
    }
}

// ---------------------------------------------------------------------------------------------
// Few rows (bf16): a warp takes one column of h, i.e. a row of the gate's weights and the same one of the other half, and all rows of x, which lie in
// shared memory as fp32.  Bound by reading W once: every warp's first 2 x 4 x 512 bytes are under way before x is.
// 1 x 768 -> 2048 2.9 us, 8 rows 5.4 (2.3 and 4.9 one behind the other in a graph), where the tensor-core kernel takes 9 for 9 rows as for 256.
// ---------------------------------------------------------------------------------------------
constexpr int kFewRows = 8, kFewWarps = 8, kFewAhead = 4, kFewFloats = 12288;
template <int GATE, int MT>
__global__ void __launch_bounds__(32 * kFewWarps)
gated_few_kernel(const uint16_t* __restrict__ x, const uint16_t* __restrict__ w, const uint16_t* __restrict__ bias, int M, int C, int H,
                 uint16_t* __restrict__ h, uint16_t* __restrict__ gu) {
    extern __shared__ __align__(16) float4 xs[];            // [row][first or second half of eight channels][C / 8]: lanes' loads lie side by side
    ptx::grid_dependency_wait();
    ptx::launch_dependents();
    const int lane = threadIdx.x & 31, j = blockIdx.x * kFewWarps + (threadIdx.x >> 5), groups = C / 8;
    const uint4* wg = reinterpret_cast<const uint4*>(w + (size_t)min(j, H - 1) * C);
    const uint4* wu = reinterpret_cast<const uint4*>(w + ((size_t)H + min(j, H - 1)) * C);
    uint4 g[kFewAhead], u[kFewAhead];
#pragma unroll
    for (int i = 0; i < kFewAhead; ++i) {
        const int k = i * 32 + lane;
        g[i] = u[i] = make_uint4(0, 0, 0, 0);
        if (k < groups) g[i] = ld_stream(wg + k), u[i] = ld_stream(wu + k);
    }
    for (int i = threadIdx.x; i < M * groups; i += 32 * kFewWarps) {
        const int m = i / groups, k = i - m * groups;
        const uint4 q = reinterpret_cast<const uint4*>(x)[i];
        xs[(2 * m) * groups + k] = make_float4(__uint_as_float(q.x << 16), __uint_as_float(q.x & 0xFFFF0000u), __uint_as_float(q.y << 16),
                                               __uint_as_float(q.y & 0xFFFF0000u));
        xs[(2 * m + 1) * groups + k] = make_float4(__uint_as_float(q.z << 16), __uint_as_float(q.z & 0xFFFF0000u), __uint_as_float(q.w << 16),
                                                   __uint_as_float(q.w & 0xFFFF0000u));
    }
    __syncthreads();
    float a[MT] = {}, b[MT] = {};
    for (int k0 = 0; k0 < groups; k0 += 32 * kFewAhead) {
#pragma unroll
        for (int i = 0; i < kFewAhead; ++i) {
            const int k = k0 + i * 32 + lane;
            if (k >= groups) continue;
            const uint32_t gw[4] = {g[i].x, g[i].y, g[i].z, g[i].w}, uw[4] = {u[i].x, u[i].y, u[i].z, u[i].w};
            if (k + 32 * kFewAhead < groups) g[i] = ld_stream(wg + k + 32 * kFewAhead), u[i] = ld_stream(wu + k + 32 * kFewAhead);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                if (m >= M) break;
                const float4 p = xs[(2 * m) * groups + k], q = xs[(2 * m + 1) * groups + k];
                const float v[8] = {p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    a[m] = fmaf(v[e], __uint_as_float(e & 1 ? gw[e / 2] & 0xFFFF0000u : gw[e / 2] << 16), a[m]);
                    b[m] = fmaf(v[e], __uint_as_float(e & 1 ? uw[e / 2] & 0xFFFF0000u : uw[e / 2] << 16), b[m]);
                }
            }
        }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
        for (int o = 16; o > 0; o >>= 1) {
            a[m] += __shfl_xor_sync(kFullMask, a[m], o);
            b[m] += __shfl_xor_sync(kFullMask, b[m], o);
        }
    if (j >= H) return;
    float av = a[0], bv = b[0];
#pragma unroll
    for (int m = 1; m < MT; ++m)
        if (lane == m) av = a[m], bv = b[m];
    if (lane >= M) return;
    if (bias) {
        av += to_float(bias[j]);
        bv += to_float(bias[H + j]);
    }
    put(h + (size_t)lane * H + j, gate_value<GATE, true>(av) * bv);
    if (gu) {
        put(gu + (size_t)lane * 2 * H + j, av);
        put(gu + (size_t)lane * 2 * H + H + j, bv);
    }
}
bool few_takes(int64_t M, int64_t C) { return M <= kFewRows && C % 8 == 0 && M * C <= kFewFloats; }
template <int GATE>
dropit_status launch_few(const void* x, const void* w, const void* bias, int M, int C, int H, void* h, void* gu, cudaStream_t stream) {
    auto kernel = M == 1 ? gated_few_kernel<GATE, 1> : M == 2 ? gated_few_kernel<GATE, 2> : M <= 4 ? gated_few_kernel<GATE, 4> : gated_few_kernel<GATE, 8>;
    return launch_programmatic(kernel, dim3((unsigned)((H + kFewWarps - 1) / kFewWarps)), 32 * kFewWarps, (size_t)M * C * 4, stream, (const uint16_t*)x,
                               (const uint16_t*)w, (const uint16_t*)bias, M, C, H, (uint16_t*)h, (uint16_t*)gu);
}

// ---------------------------------------------------------------------------------------------
// dgu = dh u f'(a) | dh f(a), and their column sums.  A warp walks down a strip of 32 * VEC columns, so that every thread keeps the sums of
// its columns; a block's eight warps meet in shared memory, the blocks of a strip in `partial` [chunks x 2H].
// Bound by HBM: three values read and two written for every two sums (12608 x 2048 in bf16: 258 MB in 42 us).  dgu in bf16 is rounded once, as the products
// take it; the column sums are of what is not rounded yet.
// ---------------------------------------------------------------------------------------------
constexpr int kBackThreads = 256, kBackWarps = kBackThreads / 32;

template <typename T, int VEC> struct Pack;
template <> struct Pack<uint16_t, 8> {
    using bits = uint4;
    static __device__ void unpack(const uint4& q, float (&v)[8]) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = __uint_as_float(w[e] << 16);
            v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
        }
    }
    static __device__ uint4 pack(const float (&v)[8]) {
        return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    }
};
template <> struct Pack<float, 4> {
    using bits = float4;
    static __device__ void unpack(const float4& q, float (&v)[4]) { v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w; }
    static __device__ float4 pack(const float (&v)[4]) { return make_float4(v[0], v[1], v[2], v[3]); }
};
template <> struct Pack<uint16_t, 1> {
    using bits = uint16_t;
    static __device__ void unpack(const uint16_t& q, float (&v)[1]) { v[0] = to_float(q); }
    static __device__ uint16_t pack(const float (&v)[1]) { return (uint16_t)pack_bf16(v[0], 0.f); }
};
template <> struct Pack<float, 1> {
    using bits = float;
    static __device__ void unpack(const float& q, float (&v)[1]) { v[0] = q; }
    static __device__ float pack(const float (&v)[1]) { return v[0]; }
};

template <typename T, int VEC, int GATE>
__global__ void __launch_bounds__(kBackThreads)
gated_backward_kernel(const T* __restrict__ dh, const T* __restrict__ gu, int64_t M, int64_t H, T* __restrict__ dgu, float* __restrict__ partial) {
    using P = Pack<T, VEC>;
    __shared__ float sums[2][kBackWarps][32 * VEC];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int64_t col = ((int64_t)blockIdx.x * 32 + lane) * VEC;
    float sg[VEC] = {}, su[VEC] = {};
    if (col < H) {
        for (int64_t r = (int64_t)blockIdx.y * kBackWarps + warp; r < M; r += (int64_t)gridDim.y * kBackWarps) {
            float d[VEC], a[VEC], u[VEC];
            P::unpack(*reinterpret_cast<const typename P::bits*>(dh + r * H + col), d);
            P::unpack(*reinterpret_cast<const typename P::bits*>(gu + r * 2 * H + col), a);
            P::unpack(*reinterpret_cast<const typename P::bits*>(gu + r * 2 * H + H + col), u);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                float value, slope;
                gate_value_and_slope<GATE, sizeof(T) == 2>(a[e], value, slope);
                a[e] = d[e] * u[e] * slope;
                u[e] = d[e] * value;
                sg[e] += a[e];
                su[e] += u[e];
            }
            *reinterpret_cast<typename P::bits*>(dgu + r * 2 * H + col) = P::pack(a);
            *reinterpret_cast<typename P::bits*>(dgu + r * 2 * H + H + col) = P::pack(u);
        }
    }
    if (!partial) return;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        sums[0][warp][lane * VEC + e] = sg[e];
        sums[1][warp][lane * VEC + e] = su[e];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * 32 * VEC; i += kBackThreads) {
        const int half = i / (32 * VEC), c = i % (32 * VEC);
        const int64_t at = (int64_t)blockIdx.x * 32 * VEC + c;
        if (at >= H) continue;
        float s = 0.f;
        for (int k = 0; k < kBackWarps; ++k) s += sums[half][k][c];
        partial[(int64_t)blockIdx.y * 2 * H + half * H + at] = s;
    }
}

// db from the blocks' partial sums: 32 columns a block, eight warps share out the partial sums, which meet in order.  The blocks behind those round the
// fp32 weight gradient to bf16.
constexpr int kFinishThreads = 256;
template <typename T>
__global__ void __launch_bounds__(kFinishThreads)
finish_kernel(const float* __restrict__ partial, int chunks, int64_t cols, T* __restrict__ db, int sum_blocks, const float* __restrict__ dw,
              uint16_t* __restrict__ dw_out, int64_t count) {
    ptx::grid_dependency_wait();
    ptx::launch_dependents();
    if ((int)blockIdx.x < sum_blocks) {
        __shared__ float sums[kFinishThreads / 32][32];
        const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
        const int64_t c = (int64_t)blockIdx.x * 32 + lane;
        float s = 0.f;
        if (c < cols)
            for (int k = warp; k < chunks; k += kFinishThreads / 32) s += partial[k * cols + c];
        sums[warp][lane] = s;
        __syncthreads();
        if (warp == 0 && c < cols) {
            s = 0.f;
            for (int k = 0; k < kFinishThreads / 32; ++k) s += sums[k][lane];
            put(db + c, s);
        }
        return;
    }
    const int64_t vecs = count / 8, stride = (int64_t)(gridDim.x - sum_blocks) * kFinishThreads, first = (int64_t)(blockIdx.x - sum_blocks) * kFinishThreads + threadIdx.x;
    const float4* from = reinterpret_cast<const float4*>(dw);
    for (int64_t i = first; i < vecs; i += stride) {
        const float4 a = __ldcs(from + 2 * i), b = __ldcs(from + 2 * i + 1);
        reinterpret_cast<uint4*>(dw_out)[i] = make_uint4(pack_bf16(a.x, a.y), pack_bf16(a.z, a.w), pack_bf16(b.x, b.y), pack_bf16(b.z, b.w));
    }
    for (int64_t e = vecs * 8 + first; e < count; e += stride) dw_out[e] = (uint16_t)pack_bf16(dw[e], 0.f);
}

int back_vec(int64_t H, dropit_dtype dtype) {
    const int wide = dtype == DROPIT_BF16 ? 8 : 4;
    return H % wide == 0 ? wide : 1;
}
// Blocks along the rows: about four blocks per SM in all.
int64_t back_chunks(int64_t M, int64_t H, dropit_dtype dtype) {
    const int64_t strips = (H + 32 * back_vec(H, dtype) - 1) / (32 * back_vec(H, dtype));
    const int64_t want = (4 * (int64_t)sm_count() + strips - 1) / strips;
    return std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(want, 65535), (M + kBackWarps - 1) / kBackWarps));
}

template <typename T, int VEC>
dropit_status launch_backward(const void* dh, const void* gu, int64_t M, int64_t H, dropit_gate gate, void* dgu, float* partial, int64_t chunks, cudaStream_t stream) {
    const dim3 grid((unsigned)((H + 32 * VEC - 1) / (32 * VEC)), (unsigned)chunks);
    auto kernel = gate == DROPIT_GATE_SILU ? gated_backward_kernel<T, VEC, DROPIT_GATE_SILU>
                  : gate == DROPIT_GATE_GELU ? gated_backward_kernel<T, VEC, DROPIT_GATE_GELU> : gated_backward_kernel<T, VEC, DROPIT_GATE_RELU>;
    // Not programmatically: blocks that come while the kernel in front still fills some of the SMs crowd on the others (12608 x 2048: 52 us, not 42).
    kernel<<<grid, kBackThreads, 0, stream>>>((const T*)dh, (const T*)gu, M, H, (T*)dgu, partial);
    return check_launch();
}

// Tiles of 32 rows x 32 columns, and for each as many CTAs as have the fullest SM do the fewest steps of the summed axis (joining costs about one).
template <typename... Params, typename... Args>
dropit_status launch_fma(void (*kernel)(Params...), int64_t rows, int64_t cols, int64_t K, cudaStream_t stream, Args... args) {
    const int64_t tiles = ((rows + kTile - 1) / kTile) * ((cols + kTile - 1) / kTile), steps = (K + kStep - 1) / kStep;
    unsigned parts = 1;
    int64_t least = 0;
    for (unsigned p = 1; p <= kMaxCluster && p <= steps; ++p) {
        const int64_t rounds = (tiles * p + sm_count() - 1) / sm_count(), time = rounds * ((steps + p - 1) / p) + (p > 1 ? 1 : 0);
        if (p == 1 || time < least) parts = p, least = time;
    }
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = parts;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((rows + kTile - 1) / kTile), (unsigned)((cols + kTile - 1) / kTile), parts);
    cfg.blockDim = dim3(kFmaThreads);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...) != cudaSuccess) {
        (void)cudaGetLastError();
        return DROPIT_ERR_CUDA;
    }
    return check_launch();
}
template <typename T>
dropit_status gated_fma(const void* x, const void* w, const void* bias, int64_t M, int64_t C, int64_t H, dropit_gate gate, void* h, void* gu, cudaStream_t stream) {
    auto kernel = gate == DROPIT_GATE_SILU ? gated_fma_kernel<T, DROPIT_GATE_SILU>
                  : gate == DROPIT_GATE_GELU ? gated_fma_kernel<T, DROPIT_GATE_GELU> : gated_fma_kernel<T, DROPIT_GATE_RELU>;
    return launch_fma(kernel, M, H, C, stream, (const T*)x, (const T*)w, (const T*)bias, M, C, H, (T*)h, (T*)gu);
}

bool gate_ok(dropit_gate g) { return g == DROPIT_GATE_SILU || g == DROPIT_GATE_GELU || g == DROPIT_GATE_RELU; }
dropit_status sizes_ok(int64_t M, int64_t C, int64_t H, dropit_dtype dtype) {
    const int64_t limit = (int64_t)1 << 31;
    if (M < 0 || C < 1 || H < 1 || (dtype != DROPIT_BF16 && dtype != DROPIT_F32)) return DROPIT_ERR_INVALID_ARG;
    if (C >= limit || 2 * H >= limit || M >= limit || M * C >= limit || M * 2 * H >= limit || 2 * H * C >= limit) return DROPIT_ERR_INVALID_ARG;
    return DROPIT_OK;
}
bool buffers_ok(std::initializer_list<const void*> needed) {
    for (const void* p : needed)
        if (!p || !is_aligned16(p)) return false;
    return true;
}

}  // namespace

int64_t gated_backward_chunks(int64_t M, int64_t H, dropit_dtype dtype) { return back_chunks(M, H, dtype); }

dropit_status gated_backward_sums(const void* dh, const void* gu, int64_t M, int64_t H, dropit_dtype dtype, dropit_gate gate, void* dgu, float* partial,
                                  void* cuda_stream) {
    cudaStream_t stream = as_stream(cuda_stream);
    const int64_t chunks = back_chunks(M, H, dtype);
    const int vec = back_vec(H, dtype);
    if (dtype == DROPIT_BF16)
        return vec == 8 ? launch_backward<uint16_t, 8>(dh, gu, M, H, gate, dgu, partial, chunks, stream)
                        : launch_backward<uint16_t, 1>(dh, gu, M, H, gate, dgu, partial, chunks, stream);
    return vec == 4 ? launch_backward<float, 4>(dh, gu, M, H, gate, dgu, partial, chunks, stream)
                    : launch_backward<float, 1>(dh, gu, M, H, gate, dgu, partial, chunks, stream);
}

dropit_status gated_finish(const float* partial, int64_t chunks, int64_t cols, dropit_dtype dtype, void* db, const float* dw, void* dw_out, int64_t count,
                           void* cuda_stream) {
    const int64_t sums = db ? (cols + 31) / 32 : 0;
    int64_t casts = (count / 8 + kFinishThreads - 1) / kFinishThreads;
    casts = std::min<int64_t>(std::max<int64_t>(casts, count ? 1 : 0), 8 * (int64_t)sm_count());
    if (sums + casts == 0) return DROPIT_OK;
    cudaStream_t stream = as_stream(cuda_stream);
    const dim3 grid((unsigned)(sums + casts));
    if (dtype == DROPIT_BF16)
        return launch_programmatic(finish_kernel<uint16_t>, grid, kFinishThreads, 0, stream, partial, (int)chunks, cols, (uint16_t*)db, (int)sums, dw,
                                   (uint16_t*)dw_out, count);
    return launch_programmatic(finish_kernel<float>, grid, kFinishThreads, 0, stream, partial, (int)chunks, cols, (float*)db, (int)sums, dw, (uint16_t*)dw_out, count);
}

}  // namespace dropit

using namespace dropit;

extern "C" dropit_status dropit_gated_linear(const void* x, const void* w, const void* bias, int64_t M, int64_t C, int64_t H, dropit_dtype dtype,
                                             dropit_gate gate, void* h, void* gu, int32_t* dev_status, void* cuda_stream) {
    const dropit_status sizes = sizes_ok(M, C, H, dtype);
    if (sizes != DROPIT_OK || !gate_ok(gate)) return DROPIT_ERR_INVALID_ARG;
    if (M == 0) return DROPIT_OK;
    if (!buffers_ok({x, w, h}) || !is_aligned16(bias) || !is_aligned16(gu)) return DROPIT_ERR_INVALID_ARG;
    if (dtype == DROPIT_BF16 && few_takes(M, C))
        return (gate == DROPIT_GATE_SILU ? launch_few<DROPIT_GATE_SILU> : gate == DROPIT_GATE_GELU ? launch_few<DROPIT_GATE_GELU> : launch_few<DROPIT_GATE_RELU>)(
            x, w, bias, (int)M, (int)C, (int)H, h, gu, as_stream(cuda_stream));
    if (dtype == DROPIT_BF16 && gated_tc_takes(M, C, H)) return gated_tc_forward(x, w, bias, M, C, H, gate, h, gu, dev_status, as_stream(cuda_stream));
    if (H > (int64_t)65535 * kTile) return DROPIT_ERR_UNSUPPORTED;
    return dtype == DROPIT_BF16 ? gated_fma<uint16_t>(x, w, bias, M, C, H, gate, h, gu, as_stream(cuda_stream))
                                : gated_fma<float>(x, w, bias, M, C, H, gate, h, gu, as_stream(cuda_stream));
}

extern "C" dropit_status dropit_gated_linear_backward_workspace(int64_t M, int64_t H, dropit_dtype dtype, size_t* workspace_bytes) {
    if (sizes_ok(M, 1, H, dtype) != DROPIT_OK || !workspace_bytes) return DROPIT_ERR_INVALID_ARG;
    *workspace_bytes = (size_t)back_chunks(M, H, dtype) * 2 * H * sizeof(float);
    return DROPIT_OK;
}

extern "C" dropit_status dropit_gated_linear_backward(const void* dh, const void* gu, int64_t M, int64_t H, dropit_dtype dtype, dropit_gate gate,
                                                      void* dgu, void* db, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (sizes_ok(M, 1, H, dtype) != DROPIT_OK || !gate_ok(gate)) return DROPIT_ERR_INVALID_ARG;
    if (M == 0 && !db) return DROPIT_OK;
    if ((M && !buffers_ok({dh, gu, dgu})) || !is_aligned16(db)) return DROPIT_ERR_INVALID_ARG;
    const int64_t chunks = back_chunks(M, H, dtype);
    if (db && (!workspace || !is_aligned16(workspace))) return DROPIT_ERR_INVALID_ARG;
    if (db && workspace_bytes < (size_t)chunks * 2 * H * sizeof(float)) return DROPIT_ERR_WORKSPACE;
    float* partial = db ? reinterpret_cast<float*>(workspace) : nullptr;
    const dropit_status s = gated_backward_sums(dh, gu, M, H, dtype, gate, dgu, partial, cuda_stream);
    return s != DROPIT_OK || !db ? s : gated_finish(partial, chunks, 2 * H, dtype, db, nullptr, nullptr, 0, cuda_stream);
}

extern "C" dropit_status dropit_gated_input_grad(const void* dgu, const void* w, int64_t M, int64_t C, int64_t H, dropit_dtype dtype, void* dx,
                                                 int32_t* dev_status, void* cuda_stream) {
    if (sizes_ok(M, C, H, dtype) != DROPIT_OK) return DROPIT_ERR_INVALID_ARG;
    if (M == 0) return DROPIT_OK;
    if (!buffers_ok({dgu, w, dx})) return DROPIT_ERR_INVALID_ARG;
    if (dtype == DROPIT_BF16 && gated_tc_takes(M, C, H)) return gated_tc_input_grad(dgu, w, M, C, H, dx, dev_status, as_stream(cuda_stream));
    if (C > (int64_t)65535 * kTile) return DROPIT_ERR_UNSUPPORTED;
    cudaStream_t stream = as_stream(cuda_stream);
    return dtype == DROPIT_BF16 ? launch_fma(input_grad_fma_kernel<uint16_t>, M, C, 2 * H, stream, (const uint16_t*)dgu, (const uint16_t*)w, M, C, 2 * H, (uint16_t*)dx)
                                : launch_fma(input_grad_fma_kernel<float>, M, C, 2 * H, stream, (const float*)dgu, (const float*)w, M, C, 2 * H, (float*)dx);
}
