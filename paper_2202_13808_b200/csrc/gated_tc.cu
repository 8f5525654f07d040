// The gated linear's products on the tensor cores: h = f(x Wg^T + bg) * (x Wu^T + bu), and dx = dgu W.
//
// A persistent pair of CTAs (cta_group::2) walks over tiles of 256 rows x BN columns.  A stage of the pipeline is 128 values of the summed axis: each
// CTA brings its own 128 rows of the left operand and half of the right one's BN by TMA (x and W lie K-major; W for dx lies MN-major, as it
// is stored), one copy an operand.  In the forward pass the even CTA's half are rows of the gate's weights and the odd one's the same rows of the other
// half, so that a CTA's accumulator holds a and u of the same 128 x BN / 2 values of h side by side, and the gate is a matter of the registers of one
// thread.  Two accumulators in tensor memory: while eight warps turn one into h, a and u, the MMAs of the next tile run into the other.
//
// Few rows: narrower tiles, so that more SMs take part, and for dx, whose summed axis is 2H long, two or four pairs of a cluster share a tile's
// summed axis and add their accumulators through the cluster's shared memory, in order (see plan()).
//
// Bound by the tensor cores for many rows, 2 M C 2H flops, as long as the sum is longer than the epilogue of a tile.  12608 x 768 -> 2048 (79 GFLOP, 48 us
// at the measured rate): forward 57 us (ReLU 56, GELU 61), 71 where a and u are kept, 73 with a bias; there the epilogue is the limit: at 128 channels, with 8 us of MMAs, it takes
// 36 and 49 (SiLU).  dx 65 in bursts, 73 for long under the power cap (a library product of its size 58 and 66).
//
// Rounded to bf16: h, a, u and dx, each once from its fp32 sum.  a and u in fp32 would double what the layer keeps (103 MB at this size) and
// the stores that bound it; the gradients carry 0.3 % (rms) instead of 0.17 % for it and for dgu, which the tensor cores take in bf16.
#include "gated.h"

#include <algorithm>

#include "weight_grad_common.cuh"

namespace dropit {

namespace {

constexpr int kRows = 256;                   // of a pair's tile
constexpr int kStep = 128;                   // summed values of a stage
constexpr int kProducers = 3;                // threads that issue copies, in warps of their own
constexpr int kEpiWarps = 8;
constexpr int kFirstEpiWarp = 1 + kProducers;        // warp 0: MMA
constexpr int kThreads = 32 * (kFirstEpiWarp + kEpiWarps);
constexpr int kSquareBytes = 32 * 32 * 2;            // through which a warp's results leave, two of them in turn
constexpr int kSquares = 2;
enum { kForward = 0, kInputGrad = 1 };

constexpr int kLeftBytes = 128 * kStep * 2;
// A CTA's half of the right operand; MN-major it comes in groups of 64 columns, of which narrow tiles use half a one.
__host__ __device__ constexpr int right_bytes(int mode, int bn) { return (mode == kForward ? bn / 2 : (bn / 2 + 63) / 64 * 64) * kStep * 2; }
__host__ __device__ constexpr int stages(int bn) { return bn >= 192 ? 3 : 4; }

struct Control {
    uint64_t full[4];
    uint64_t empty[4];
    uint64_t ready[2];                       // accumulator b is final
    uint64_t drained[2];                     // leader: both CTAs' epilogues have read accumulator b
    uint64_t done;                           // no MMA is in flight any more
    uint32_t tmem_base;
    int abort_flag;
    int consumed;                            // leader: stages whose operands the MMA thread has seen arrive
    int issued[4];                           // per slot: rounds this CTA's producers have issued
    int peer_issued[4];                      // the other CTA's
    int peer_abort;
};

constexpr size_t smem_bytes(int mode, int bn) {
    return 1024 + (size_t)stages(bn) * (kLeftBytes + right_bytes(mode, bn)) + (size_t)kEpiWarps * kSquares * kSquareBytes + sizeof(Control);
}
static_assert(smem_bytes(kForward, 256) <= 227 * 1024 && smem_bytes(kForward, 128) <= 227 * 1024, "shared memory of a CTA");

struct Maps {
    CUtensorMap left, right, out[3];         // out: h, a, u for the TMA stores
};
struct Shape {
    int M, N;                                // N: hidden width (forward) or columns of dx
    int tiles_n, tiles, steps;               // steps: stages of a tile's summed axis
    int splits;                              // pairs that share a tile's summed axis (the cluster has twice as many CTAs)
    int keep;                                // a and u are stored
    uint16_t* out;                           // dx
    int grouped_left, grouped_right;         // one copy brings both 64-wide halves of a stage
    const uint16_t* bias;
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// A lane's 32 values of one row into a square of 32 x 32, as the TMA store's 64-byte swizzle wants them.
__device__ __forceinline__ void stage_row(uint32_t square, int lane, const float (&v)[32]) {
#pragma unroll
    for (int c = 0; c < 4; ++c)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(square + lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4)), "r"(pack_bf16(v[8 * c], v[8 * c + 1])),
                     "r"(pack_bf16(v[8 * c + 2], v[8 * c + 3])), "r"(pack_bf16(v[8 * c + 4], v[8 * c + 5])), "r"(pack_bf16(v[8 * c + 6], v[8 * c + 7]))
                     : "memory");
}
// The same square to rows of `pitch` elements from `to` on without TMA; `rows` and `cols` (a multiple of 8) are what there is of them.  The lanes change
// places in shared memory, so that a store instruction covers 64 bytes of eight rows and not 16 of 32.
__device__ __forceinline__ void store_square(uint16_t* to, size_t pitch, uint8_t* square, int lane, const float (&v)[32], int rows, int cols) {
    stage_row(ptx::smem_u32(square), lane, v);
    __syncwarp();
    const int c = lane & 3;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + (lane >> 2);
        const uint4 q = *reinterpret_cast<const uint4*>(square + r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
        if (r < rows && 8 * c < cols) *reinterpret_cast<uint4*>(to + r * pitch + 8 * c) = q;
    }
    __syncwarp();
}
// 32 values of the bias from column c on (limit, a multiple of 8 and at least that: its end; behind it anything).  All loads go out at once, in front of the
// accumulator's: one after the other 12608 x 768 -> 2048 with a and u took 80 us instead of 74, 591 rows 16.6 instead of 15.8.
__device__ __forceinline__ void load_bias(uint4 (&q)[4], const uint16_t* bias, int c, int limit) {
#pragma unroll
    for (int e = 0; e < 4; ++e) q[e] = __ldg(reinterpret_cast<const uint4*>(bias + min(c + 8 * e, limit - 8)));
}
__device__ __forceinline__ void add_bias(float (&acc)[32], const uint4 (&q)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t w[4] = {q[e].x, q[e].y, q[e].z, q[e].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            acc[8 * e + 2 * i] += __uint_as_float(w[i] << 16);
            acc[8 * e + 2 * i + 1] += __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
}

template <int MODE, int BN, int GATE>
__global__ void __launch_bounds__(kThreads, 1)
gated_tc_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Shape shape, int32_t* dev_status, uint32_t wait_limit) {
    extern __shared__ uint8_t smem_raw[];
    // the same offsets in both CTAs: the MMA addresses the operands of both with one descriptor
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    constexpr int kStages = stages(BN), kRightBytes = right_bytes(MODE, BN), kHidden = BN / 2;
    constexpr uint32_t kStageTx = kLeftBytes + kRightBytes;
    constexpr int kTmemPitch = BN <= 64 ? 64 : BN <= 128 ? 128 : 256, kColumns = 2 * kTmemPitch;
    uint8_t* left = smem;
    uint8_t* right = left + kStages * kLeftBytes;
    uint8_t* squares = right + kStages * kRightBytes;
    Control* ctl = reinterpret_cast<Control*>(squares + kEpiWarps * kSquares * kSquareBytes);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = ptx::cluster_ctarank(), leader = rank & ~1u;
    const int member = (int)(rank & 1u), split = (int)(rank >> 1);                // member 0: the pair's leader
    const uint16_t both = (uint16_t)(3u << leader);
    const int first_tile = (int)(blockIdx.x / (2 * shape.splits)), stride = (int)(gridDim.x / (2 * shape.splits));
    const int step0 = split * shape.steps / shape.splits, steps = (split + 1) * shape.steps / shape.splits - step0;
    volatile int* abort_flag = &ctl->abort_flag;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            ptx::mbar_init(&ctl->full[s], 1);
            ptx::mbar_init(&ctl->empty[s], 1);
            ctl->issued[s] = ctl->peer_issued[s] = 0;
        }
        for (int b = 0; b < 2; ++b) {
            ptx::mbar_init(&ctl->ready[b], 1);
            ptx::mbar_init(&ctl->drained[b], 2 * kEpiWarps);
        }
        ptx::mbar_init(&ctl->done, 1);
        ctl->abort_flag = ctl->consumed = ctl->peer_abort = 0;
        ptx::fence_mbar_init();
        ptx::prefetch_tensormap(&maps.left);
        ptx::prefetch_tensormap(&maps.right);
    }
    if (warp == 0) {
        ptx::tmem_alloc_pair(&ctl->tmem_base, kColumns);
        ptx::tmem_relinquish_pair();
    }
    ptx::tc_fence_before();
    ptx::cluster_sync_all();             // all CTAs' barriers exist before any CTA signals another
    ptx::tc_fence_after();
    const uint32_t tmem_base = ctl->tmem_base;
    ptx::grid_dependency_wait();         // set up while the kernel in front was ending; from here on memory is read and written
    ptx::launch_dependents();
    const int quarter = warp & 3, half = (warp - kFirstEpiWarp) >> 2;
    uint8_t* square = squares + (warp - kFirstEpiWarp) * kSquares * kSquareBytes;     // epilogue warps
    bool final_ok = false;               // splits: this warp's accumulator is there

    if (warp == 0) {
        // ---------------- MMA issuer (leader only) ----------------
        if (lane == 0 && member == 0) {
            constexpr uint32_t idesc = ptx::make_idesc_bf16(kRows, BN, false, MODE == kInputGrad);
            int s = 0, consumed = 0, turn = 0;
            uint32_t parity = 0;
            bool go = true;
            for (int tile = first_tile; tile < shape.tiles && go; tile += stride, ++turn) {
                const int b = turn & 1;
                if (turn >= 2 && !ptx::mbar_wait_poll(&ctl->drained[b], (uint32_t)((turn >> 1) - 1) & 1u, wait_limit)) {
                    *abort_flag = 1;
                    break;
                }
                ptx::tc_fence_after();
                const uint32_t tmem_d = tmem_base + b * kTmemPitch;
                for (int k = 0; k < steps; ++k) {
                    if (*abort_flag || !ptx::mbar_wait_poll(&ctl->full[s], parity, wait_limit)) {
                        *abort_flag = 1;
                        go = false;
                        break;
                    }
                    ++consumed;
                    ptx::tc_fence_after();
                    const uint32_t a_addr = ptx::smem_u32(left + s * kLeftBytes), b_addr = ptx::smem_u32(right + s * kRightBytes);
#pragma unroll
                    for (int kk = 0; kk < kStep / 16; ++kk) {
                        // K-major: 64-wide halves of the stage behind one another, 32 bytes further for every 16 values
                        const uint64_t ad = ptx::make_smem_desc_sw128(a_addr + (kk / 4) * (128 * 128) + (kk % 4) * 32, 16, 1024);
                        const uint64_t bd = MODE == kForward ? ptx::make_smem_desc_sw128(b_addr + (kk / 4) * (kHidden * 128) + (kk % 4) * 32, 16, 1024)
                                                             : ptx::make_smem_desc_sw128(b_addr + kk * 2048, 64 * kStep * 2, 1024);
                        ptx::umma_bf16_pair(tmem_d, ad, bd, idesc, (k | kk) ? 1u : 0u);
                    }
                    ptx::umma_commit_pair(&ctl->empty[s], both);
                    if (++s == kStages) { s = 0; parity ^= 1u; }
                }
                if (go) ptx::umma_commit_pair(&ctl->ready[b], both);
            }
            ctl->consumed = consumed;
            ptx::umma_commit_pair(&ctl->done, both);
        }
    } else if (warp < kFirstEpiWarp) {
        // ---------------- TMA producers (both CTAs): every third stage each ----------------
        if (lane == 0) {
            const uint32_t full0 = ptx::map_shared_to_cta(ptx::smem_u32(&ctl->full[0]), leader);
            int k = warp - 1;
            bool go = true;
            uint32_t i = (uint32_t)k;                                    // stages of this CTA's tiles, counted through
            for (int tile = first_tile; tile < shape.tiles && go; tile += stride) {
                const int row = (tile / shape.tiles_n) * kRows + member * 128;
                const int n0 = (tile % shape.tiles_n) * (MODE == kForward ? kHidden : BN);
                for (; k < steps; k += kProducers, i += kProducers) {
                    const uint32_t s = i % kStages, round = i / kStages;
                    if (*abort_flag || (round > 0 && !ptx::mbar_wait_poll(&ctl->empty[s], (round - 1) & 1u, wait_limit))) {
                        *abort_flag = 1;
                        go = false;
                        break;
                    }
                    const uint32_t bar = full0 + 8u * s;
                    // in front of the copies: the slot's next round is another thread's, which waits for what these bring
                    reinterpret_cast<volatile int*>(ctl->issued)[s] = (int)round + 1;
                    if (!member) ptx::mbar_arrive_expect_tx(&ctl->full[s], 2u * kStageTx);
                    uint8_t* a = left + s * kLeftBytes;
                    uint8_t* b = right + s * kRightBytes;
                    const int k0 = (step0 + k) * kStep;
                    if (shape.grouped_left) {
                        ptx::tma_load_3d_pair(a, &maps.left, 0, row, k0 / 64, bar);
                    } else {
                        ptx::tma_load_2d_pair(a, &maps.left, k0, row, bar);
                        ptx::tma_load_2d_pair(a + 128 * 128, &maps.left, k0 + 64, row, bar);
                    }
                    if constexpr (MODE == kForward) {
                        if (shape.grouped_right) {
                            ptx::tma_load_3d_pair(b, &maps.right, 0, n0 + member * shape.N, k0 / 64, bar);
                        } else {
                            ptx::tma_load_2d_pair(b, &maps.right, k0, n0 + member * shape.N, bar);
                            ptx::tma_load_2d_pair(b + kHidden * 128, &maps.right, k0 + 64, n0 + member * shape.N, bar);
                        }
                    } else {
                        if (shape.grouped_right) {
                            ptx::tma_load_3d_pair(b, &maps.right, 0, k0, (n0 + member * kHidden) / 64, bar);
                        } else {
#pragma unroll
                            for (int g = 0; g < kRightBytes / (64 * kStep * 2); ++g)
                                ptx::tma_load_2d_pair(b + g * (64 * kStep * 2), &maps.right, n0 + member * kHidden + 64 * g, k0, bar);
                        }
                    }
                }
                k -= steps;
            }
        }
    } else {
        // ---------------- epilogue: accumulator -> h, a, u or dx (both CTAs, each its own 128 rows) ----------------
        const uint32_t drained0 = ptx::map_shared_to_cta(ptx::smem_u32(&ctl->drained[0]), leader);
        int turn = 0, which = 0;
        // 32 rows x 32 columns through the next of the warp's squares, once its last store has read it
        auto store = [&](const CUtensorMap* map, const float (&v)[32], int col, int row) {
            if (lane == 0) ptx::bulk_wait_read<kSquares - 1>();
            __syncwarp();
            stage_row(ptx::smem_u32(square) + which * kSquareBytes, lane, v);
            ptx::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
                ptx::tma_store_2d(map, square + which * kSquareBytes, col, row);
                ptx::bulk_commit();
            }
            which ^= 1;
        };
        for (int tile = first_tile; tile < shape.tiles; tile += stride, ++turn) {
            const int b = turn & 1;
            if (MODE == kForward && shape.bias) {       // the tile's part of the bias on its way while the accumulator is not there yet
                const int n = (tile % shape.tiles_n) * kHidden + (lane & 15) * 8;
                if (n < shape.N) ptx::prefetch_l1(shape.bias + (lane < 16 ? 0 : shape.N) + n);
            }
            bool ok = ptx::mbar_wait_warp(&ctl->ready[b], (uint32_t)(turn >> 1) & 1u, wait_limit);
            ok = __all_sync(kFullMask, ok && !*abort_flag);
            if (!ok) { *abort_flag = 1; break; }
            ptx::tc_fence_after();
            if (MODE == kInputGrad && shape.splits > 1) { final_ok = true; break; }
            const int row = (tile / shape.tiles_n) * kRows + member * 128 + quarter * 32;
            const uint32_t tmem = tmem_base + ((uint32_t)(32 * quarter) << 16) + b * kTmemPitch;
            constexpr int kChunks = (MODE == kForward ? kHidden : BN) / 32;
            const int n0 = (tile % shape.tiles_n) * (MODE == kForward ? kHidden : BN);
#pragma unroll 1
            for (int ch = half; ch < kChunks; ch += 2) {
                const int c = ch * 32;
                float v[32], u[MODE == kForward ? 32 : 1];
                uint4 bias_v[4], bias_u[4];
                if (MODE == kForward && shape.bias) {
                    load_bias(bias_v, shape.bias, n0 + c, shape.N);
                    load_bias(bias_u, shape.bias + shape.N, n0 + c, shape.N);
                }
                {
                    uint32_t r[32];
                    ptx::tmem_ld_32x32(tmem + c, r);
                    if constexpr (MODE == kForward) {
                        uint32_t q[32];
                        ptx::tmem_ld_32x32(tmem + kHidden + c, q);
                        ptx::tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 32; ++e) u[e] = __uint_as_float(q[e]);
                    } else {
                        ptx::tmem_ld_wait();
                    }
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = __uint_as_float(r[e]);
                }
                if (row >= shape.M || n0 + c >= shape.N) continue;
                if constexpr (MODE == kForward) {
                    if (shape.bias) {
                        add_bias(v, bias_v);
                        add_bias(u, bias_u);
                    }
                    if (shape.keep) {
                        store(&maps.out[1], v, n0 + c, row);
                        store(&maps.out[2], u, n0 + c, row);
                    }
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = gate_value<GATE, true>(v[e]) * u[e];
                    store(&maps.out[0], v, n0 + c, row);
                } else {
                    store_square(shape.out + (size_t)row * shape.N + n0 + c, (size_t)shape.N, square, lane, v, shape.M - row, shape.N - (n0 + c));
                }
            }
            // the accumulator has been read: the next tile but one may have it
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive_cluster(drained0 + 8u * b);
        }
        if (MODE == kForward && lane == 0) ptx::bulk_wait_read<0>();     // the squares have been read; what they hold arrives before the kernel counts as ended
    }

    if constexpr (MODE == kInputGrad) {
        // The pairs that share a tile's summed axis each hold all of its sums over their part.  Rows 32 q .. 32 q + 31 of a CTA are finished by the pair
        // q * splits / 4: the others send it theirs, and it adds them in the pairs' order.
        if (shape.splits > 1) {
            const int S = shape.splits, quarters = 4 / S;            // of 32 rows that a pair finishes
            constexpr int kChunks = BN / 32;
            __syncthreads();
            ptx::cluster_sync_all();         // every pair's MMAs are done: the pipeline's buffers are free
            const int owner = quarter / quarters;
            const uint32_t tmem = tmem_base + ((uint32_t)(32 * quarter) << 16);
            auto place = [&](int slot, int ch) { return (uint32_t)(((slot * quarters + quarter % quarters) * kChunks + ch) * 4096 + lane * 16); };
            if (final_ok && owner != split) {
                const uint32_t base = ptx::map_shared_to_cta(ptx::smem_u32(smem), (uint32_t)(2 * owner + member));
#pragma unroll 1
                for (int ch = half; ch < kChunks; ch += 2) {
                    uint32_t r[32];
                    ptx::tmem_ld_32x32(tmem + ch * 32, r);
                    ptx::tmem_ld_wait();
                    const uint32_t to = base + place(split < owner ? split : split - 1, ch);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        ptx::st_cluster_v4(to + e * 512, __uint_as_float(r[4 * e]), __uint_as_float(r[4 * e + 1]), __uint_as_float(r[4 * e + 2]),
                                           __uint_as_float(r[4 * e + 3]));
                }
            }
            ptx::cluster_sync_all();
            if (final_ok && owner == split) {
                const int row = (first_tile / shape.tiles_n) * kRows + member * 128 + quarter * 32, n0 = (first_tile % shape.tiles_n) * BN;
#pragma unroll 1
                for (int ch = half; ch < kChunks; ch += 2) {
                    uint32_t r[32];
                    ptx::tmem_ld_32x32(tmem + ch * 32, r);
                    ptx::tmem_ld_wait();
                    if (row >= shape.M || n0 + ch * 32 >= shape.N) continue;
                    float v[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = 0.f;
                    for (int s = 0; s < S; ++s) {
                        if (s == split) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) v[e] += __uint_as_float(r[e]);
                        } else {
                            const uint8_t* from = smem + place(s < split ? s : s - 1, ch);
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const float4 q = *reinterpret_cast<const float4*>(from + e * 512);
                                v[4 * e] += q.x; v[4 * e + 1] += q.y; v[4 * e + 2] += q.z; v[4 * e + 3] += q.w;
                            }
                        }
                    }
                    store_square(shape.out + (size_t)row * shape.N + n0 + ch * 32, (size_t)shape.N, square, lane, v, shape.M - row, shape.N - (n0 + ch * 32));
                }
            }
        }
    }

    // Neither CTA leaves while another may still signal its barriers or read its shared memory.
    __syncthreads();
    if (threadIdx.x == 0) {
        const uint32_t other = rank ^ 1u;
        ptx::st_cluster_u32(ptx::map_shared_to_cta(ptx::smem_u32(&ctl->peer_abort), other), (uint32_t)*abort_flag);
        for (int s = 0; s < kStages; ++s)
            ptx::st_cluster_u32(ptx::map_shared_to_cta(ptx::smem_u32(&ctl->peer_issued[s]), other), (uint32_t)ctl->issued[s]);
    }
    ptx::tc_fence_before();
    ptx::cluster_sync_all();
    if (*abort_flag || *reinterpret_cast<volatile int*>(&ctl->peer_abort)) {
        // After a wait was given up, copies may be in flight whose stage the MMA thread never took, and one CTA may have issued a stage that the
        // other did not: the leader squares the accounts of those barriers by hand (bytes that were announced but never sent are counted as
        // arrived; bytes that were sent unannounced get their arrival) and waits for the rest, while the other CTA stays.
        if (!member && threadIdx.x == 0) {
            const int consumed = ctl->consumed;
            for (int s = 0; s < kStages; ++s) {
                const int taken = consumed > s ? (consumed - s + kStages - 1) / kStages : 0;      // rounds of slot s that the MMAs took
                const int ours = ctl->issued[s], theirs = *reinterpret_cast<volatile int*>(&ctl->peer_issued[s]);
                if (ours <= taken && theirs <= taken) continue;
                uint64_t* bar = &ctl->full[s];
                if (ours <= taken) ptx::mbar_arrive_expect_tx(bar, kStageTx);
                else if (theirs <= taken) ptx::mbar_complete_tx(bar, kStageTx);
                ptx::mbar_wait(bar, (uint32_t)taken & 1u, kWaitLimit);
            }
            if (dev_status) atomicExch(dev_status, (int)DROPIT_ERR_TIMEOUT);
        }
        __syncthreads();
        ptx::cluster_sync_all();         // both CTAs of the pair come here (others of the cluster may have left)
    }
    if (warp == 0) {
        // tensor memory is given back by both CTAs, and only once no MMA can still write to it
        ptx::mbar_wait_warp(&ctl->done, 0, kWaitLimit);
        ptx::tc_fence_after();
        ptx::tmem_dealloc_pair(tmem_base, kColumns);
    }
}

using Kernel = void (*)(Maps, Shape, int32_t*, uint32_t);
template <int BN>
Kernel forward_kernel(dropit_gate gate) {
    return gate == DROPIT_GATE_SILU ? gated_tc_kernel<kForward, BN, DROPIT_GATE_SILU>
           : gate == DROPIT_GATE_GELU ? gated_tc_kernel<kForward, BN, DROPIT_GATE_GELU> : gated_tc_kernel<kForward, BN, DROPIT_GATE_RELU>;
}
constexpr int kWidths[] = {256, 192, 128, 64};
Kernel kernel_of(int mode, int width, dropit_gate gate) {
    if (mode == kForward)
        return width == 256 ? forward_kernel<256>(gate) : width == 192 ? forward_kernel<192>(gate) : width == 128 ? forward_kernel<128>(gate) : forward_kernel<64>(gate);
    return width == 256 ? gated_tc_kernel<kInputGrad, 256, 0> : width == 128 ? gated_tc_kernel<kInputGrad, 128, 0> : gated_tc_kernel<kInputGrad, 64, 0>;
}

// How many clusters of 2 * splits CTAs run at the same time (some SMs have no partner), once the kernel may use its shared memory.
int resident_clusters(Kernel kernel, size_t smem, int splits) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2 * splits;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * splits);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int v = 0;
    if (cudaOccupancyMaxActiveClusters(&v, kernel, &cfg) != cudaSuccess || v <= 0) v = std::max(1, sm_count() / (2 * splits));
    (void)cudaGetLastError();
    return v;
}

struct Plan {
    int width, splits, clusters;             // clusters: that run at the same time
    int tiles_n, tiles, steps;
    float us;
};
// Time of a tile's stage in a pair, in us: measured 0.75 at the full width, where it is the MMAs' (64 KB of copies a CTA), and about as the copies' bytes
// below it.
float step_us(int mode, int width) { return 1.14e-5f * (float)(kLeftBytes + right_bytes(mode, width)); }

// Width of the tiles and, for dx, pairs per tile: whatever is done first.  A wave costs its stages, the last tile's epilogue 2.6 us at the full width; pairs
// that join their sums 1 us for the cluster's barriers and 9 at the full width for sending and adding (measured with %globaltimer).
Plan plan(int mode, int64_t M, int64_t N, int64_t K) {
    static std::atomic<int> pairs_of[64][3];                // [device][log2 splits]
    const int dev = current_device();
    int resident[3];
    for (int l = 0; l < 3; ++l) {
        resident[l] = dev >= 0 && dev < 64 ? pairs_of[dev][l].load(std::memory_order_acquire) : 0;
        if (resident[l]) continue;
        for (int m = 0; m < 2; ++m)
            for (int w : kWidths)
                for (int g = 0; g < (m == kForward ? 3 : w == 192 ? 0 : 1); ++g)
                    (void)cudaFuncSetAttribute(kernel_of(m, w, (dropit_gate)g), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes(m, w));
        resident[l] = resident_clusters(kernel_of(kInputGrad, 256, DROPIT_GATE_SILU), smem_bytes(kInputGrad, 256), 1 << l);
        if (dev >= 0 && dev < 64) pairs_of[dev][l].store(resident[l], std::memory_order_release);
    }
    Plan best = {};
    for (int w : kWidths) {
        if (mode == kInputGrad && w == 192) continue;       // three groups of 64 columns are not two halves
        const int columns = mode == kForward ? w / 2 : w;
        Plan p = {};
        p.width = w;
        p.tiles_n = (int)((N + columns - 1) / columns);
        p.tiles = (int)((M + kRows - 1) / kRows) * p.tiles_n;
        p.steps = (int)((K + kStep - 1) / kStep);
        for (int l = 0; l < (mode == kForward ? 1 : 3); ++l) {
            p.splits = 1 << l;
            p.clusters = resident[l];
            if (l && (p.tiles > p.clusters || p.steps < 4 * p.splits)) break;       // one tile a cluster, and enough to share
            const int waves = (p.tiles + p.clusters - 1) / p.clusters;
            p.us = (float)(waves * ((p.steps + p.splits - 1) / p.splits)) * step_us(mode, w) + (l ? 1.f + 0.035f * (float)w : 0.01f * (float)w);
            if (!best.width || p.us < best.us * 0.98f) best = p;
        }
    }
    return best;
}

dropit_status launch(int mode, Kernel kernel, const Plan& p, const Maps& maps, const Shape& shape, int32_t* dev_status, cudaStream_t stream) {
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2 * p.splits;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * p.splits * (p.splits > 1 ? p.tiles : std::min(p.clusters, p.tiles))));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem_bytes(mode, p.width);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, kernel, maps, shape, dev_status, spin_limit(kWaitLimit)) != cudaSuccess) {
        (void)cudaGetLastError();
        return DROPIT_ERR_CUDA;
    }
    return check_launch();
}

// [rows x cols] in pieces of 64 columns x box_rows: as [cols / 64][rows][64] with two (or `groups`) of them a copy, where 64 divides the columns.
bool operand_map(CUtensorMap* map, const void* base, int64_t rows, int64_t cols, int groups, int box_rows, int* grouped) {
    *grouped = cols % 64 == 0;
    return *grouped ? make_map_grouped_bf16(map, base, rows, cols, groups, box_rows) : make_map_2d_bf16(map, base, rows, cols, box_rows);
}

}  // namespace

bool gated_tc_takes(int64_t M, int64_t C, int64_t H) { return M >= 1 && C % 8 == 0 && H % 8 == 0; }

dropit_status gated_tc_forward(const void* x, const void* w, const void* bias, int64_t M, int64_t C, int64_t H, dropit_gate gate, void* h, void* gu,
                               int32_t* dev_status, cudaStream_t stream) {
    const Plan p = plan(kForward, M, H, C);
    Maps maps = {};
    Shape s = {};
    if (!operand_map(&maps.left, x, M, C, kStep / 64, 128, &s.grouped_left) ||
        !operand_map(&maps.right, w, 2 * H, C, kStep / 64, p.width / 2, &s.grouped_right))
        return DROPIT_ERR_CUDA;
    s.M = (int)M;
    s.N = (int)H;
    s.tiles_n = p.tiles_n;
    s.tiles = p.tiles;
    s.steps = p.steps;
    s.splits = 1;
    uint16_t* kept = reinterpret_cast<uint16_t*>(gu);
    if (!make_map_out_bf16(&maps.out[0], h, M, H, H)) return DROPIT_ERR_CUDA;
    if (gu && (!make_map_out_bf16(&maps.out[1], kept, M, H, 2 * H) || !make_map_out_bf16(&maps.out[2], kept + H, M, H, 2 * H))) return DROPIT_ERR_CUDA;
    s.keep = gu != nullptr;
    s.bias = reinterpret_cast<const uint16_t*>(bias);
    return launch(kForward, kernel_of(kForward, p.width, gate), p, maps, s, dev_status, stream);
}

static dropit_status input_grad_rows(const Plan& p, const uint16_t* dgu, const void* w, int64_t M, int64_t C, int64_t H, uint16_t* dx, int32_t* dev_status,
                                     cudaStream_t stream) {
    Maps maps = {};
    Shape s = {};
    if (!operand_map(&maps.left, dgu, M, 2 * H, kStep / 64, 128, &s.grouped_left)) return DROPIT_ERR_CUDA;
    if (p.width == 64 ? !make_map_2d_bf16(&maps.right, w, 2 * H, C, kStep)       // halves of a group start between two
                      : !operand_map(&maps.right, w, 2 * H, C, p.width / 128, kStep, &s.grouped_right))
        return DROPIT_ERR_CUDA;
    s.M = (int)M;
    s.N = (int)C;
    s.tiles_n = p.tiles_n;
    s.tiles = p.tiles;
    s.steps = p.steps;
    s.splits = p.splits;
    s.out = dx;
    return launch(kInputGrad, kernel_of(kInputGrad, p.width, DROPIT_GATE_SILU), p, maps, s, dev_status, stream);
}

// A last wave of a few tiles takes as long as their whole summed axis.  Where it is a sixteenth of the pairs or less, the rows of the full waves are one
// launch and the rest, whose pairs share the axis, another (us in bursts, one launch in brackets): 12608 x 4096 -> 768 (150 tiles on 74 pairs) 65 (71),
// 19200 x 4096 -> 256 (75 tiles) 48 (55); with half the sum the second launch costs what it saves, 19000 x 2048 -> 768 (225 tiles) 52 (51).  With more tiles in
// the last wave it costs more (32768 rows, 14 tiles: 154 and 151; 25000 x 2048 -> 384, 48 tiles: 61 and 53).
dropit_status gated_tc_input_grad(const void* dgu, const void* w, int64_t M, int64_t C, int64_t H, void* dx, int32_t* dev_status, cudaStream_t stream) {
    const Plan whole = plan(kInputGrad, M, C, 2 * H);
    const uint16_t* from = reinterpret_cast<const uint16_t*>(dgu);
    uint16_t* to = reinterpret_cast<uint16_t*>(dx);
    const int last = whole.tiles % whole.clusters;
    if (whole.splits == 1 && whole.tiles > whole.clusters && last && 16 * last <= whole.clusters) {
        const int64_t rows = (int64_t)kRows * ((whole.tiles - last) / whole.tiles_n);
        if (rows > 0 && rows < M) {
            const dropit_status s = input_grad_rows(plan(kInputGrad, rows, C, 2 * H), from, w, rows, C, H, to, dev_status, stream);
            if (s != DROPIT_OK) return s;
            return input_grad_rows(plan(kInputGrad, M - rows, C, 2 * H), from + rows * 2 * H, w, M - rows, C, H, to + rows * C, dev_status, stream);
        }
    }
    return input_grad_rows(whole, from, w, M, C, H, to, dev_status, stream);
}

}  // namespace dropit
