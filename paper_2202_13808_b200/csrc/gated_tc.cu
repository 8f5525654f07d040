// The gated linear's products on the tensor cores: h = f(x Wg^T + bg) * (x Wu^T + bu), and dx = dgu W.
//
// A persistent pair of CTAs (cta_group::2) walks over tiles of 256 rows.  A stage of the pipeline is 64 values of the summed axis: each CTA brings its
// own 128 rows of the left operand and half of the right one by TMA (x and W lie K-major; W for dx lies MN-major, as it is stored).
// In the forward pass the even CTA's half are rows of the gate's weights and the odd one's the same rows of the other half, so that
// a CTA's accumulator holds a and u of the same 128 x 128 values of h side by side, and the gate is a matter of the registers of one thread.
// Two accumulators in tensor memory: while eight warps turn one into h, a and u, the MMAs of the next tile run into the other.
// Results leave through shared memory as TMA stores, which also drop what lies behind the last row or column.
//
// Bound by the tensor cores for many rows: 2 M C 2H flops.
#include "gated.h"

#include <algorithm>

#include "weight_grad_common.cuh"

namespace dropit {

namespace {

constexpr int kRows = 256;                   // of a pair's tile
constexpr int kStages = 5;
constexpr int kEpiWarps = 8;
constexpr int kThreads = 64 + 32 * kEpiWarps;        // TMA warp, MMA warp, epilogue warps
constexpr int kStoreBytes = 32 * 32 * 2;             // what a warp stages for one store: 32 rows x 32 columns
enum { kForward = 0, kInputGrad = 1 };

constexpr int kLeftBytes = 128 * kBK * 2;
__host__ __device__ constexpr int right_bytes(int bn) { return bn / 2 * kBK * 2; }
__host__ __device__ constexpr int stores_per_warp(int mode) { return mode == kForward ? 3 : 2; }

struct Control {
    uint64_t full[kStages];
    uint64_t empty[kStages];
    uint64_t ready[2];                       // accumulator b is final
    uint64_t drained[2];                     // leader: both CTAs' epilogues have read accumulator b
    uint64_t done;                           // no MMA is in flight any more
    uint32_t tmem_base;
    int abort_flag;
    int consumed;                            // leader: stages whose operands the MMA thread has seen arrive
    int issued[kStages];                     // per slot: rounds this CTA's producer has issued
    int peer_issued[kStages];                // leader: the other CTA's
    int peer_abort;
};

constexpr size_t smem_bytes(int mode, int bn) {
    return 1024 + (size_t)kStages * (kLeftBytes + right_bytes(bn)) + (size_t)kEpiWarps * stores_per_warp(mode) * kStoreBytes + sizeof(Control);
}
static_assert(smem_bytes(kForward, 256) <= 227 * 1024, "shared memory of a CTA");

struct Maps {
    CUtensorMap left, right, out[3];         // out: h, a, u, or dx
};
struct Shape {
    int M, K, N;                             // K: summed axis; N: hidden width (forward) or columns of dx
    int tiles_n, tiles, steps;               // steps: stages per tile
    int keep;                                // a and u are stored
    const uint16_t* bias;
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// A lane's 32 values of one row into the warp's staging square, as the store's 64-byte swizzle wants them.
__device__ __forceinline__ void stage_row(uint32_t square, int lane, const float (&v)[32]) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const uint32_t at = square + lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4);
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(pack_bf16(v[8 * c], v[8 * c + 1])),
                     "r"(pack_bf16(v[8 * c + 2], v[8 * c + 3])), "r"(pack_bf16(v[8 * c + 4], v[8 * c + 5])), "r"(pack_bf16(v[8 * c + 6], v[8 * c + 7]))
                     : "memory");
    }
}
// acc += 32 values of the bias from column c on (limit: its end)
__device__ __forceinline__ void add_bias(float (&acc)[32], const uint16_t* bias, int c, int limit) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (c + 8 * e >= limit) break;
        const uint4 q = __ldg(reinterpret_cast<const uint4*>(bias + c + 8 * e));
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            acc[8 * e + 2 * i] += __uint_as_float(w[i] << 16);
            acc[8 * e + 2 * i + 1] += __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
}

template <int MODE, int BN, int GATE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
gated_tc_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Shape shape, int32_t* dev_status, uint32_t wait_limit) {
    extern __shared__ uint8_t smem_raw[];
    // the same offsets in both CTAs: the MMA addresses the operands of both with one descriptor
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    constexpr int kRightBytes = right_bytes(BN);
    constexpr uint32_t kStageTx = kLeftBytes + kRightBytes;
    uint8_t* left = smem;
    uint8_t* right = left + kStages * kLeftBytes;
    uint8_t* squares = right + kStages * kRightBytes;
    Control* ctl = reinterpret_cast<Control*>(squares + kEpiWarps * stores_per_warp(MODE) * kStoreBytes);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int member = (int)(ptx::cluster_ctarank() & 1u);       // 0: leader
    const int first_tile = blockIdx.x >> 1, stride = gridDim.x >> 1;
    constexpr uint32_t kColumns = 2 * BN;
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
    if (warp == 1) {
        ptx::tmem_alloc_pair(&ctl->tmem_base, kColumns);
        ptx::tmem_relinquish_pair();
    }
    ptx::tc_fence_before();
    ptx::cluster_sync_all();             // both CTAs' barriers exist before either CTA signals the other
    ptx::tc_fence_after();
    const uint32_t tmem_base = ctl->tmem_base;

    if (warp == 0) {
        // ---------------- TMA producer (both CTAs) ----------------
        if (lane == 0) {
            const uint32_t full0 = ptx::map_shared_to_cta(ptx::smem_u32(&ctl->full[0]), 0);
            int s = 0, round = 0;
            bool go = true;
            for (int tile = first_tile; tile < shape.tiles && go; tile += stride) {
                const int row = (tile / shape.tiles_n) * kRows + member * 128;
                const int n0 = (tile % shape.tiles_n) * (MODE == kForward ? BN / 2 : BN);
                for (int k = 0; k < shape.steps; ++k) {
                    if (*abort_flag || (round > 0 && !ptx::mbar_wait_spin(&ctl->empty[s], (uint32_t)(round - 1) & 1u, wait_limit))) {
                        *abort_flag = 1;
                        go = false;
                        break;
                    }
                    const uint32_t bar = full0 + 8u * (uint32_t)s;
                    if (!member) ptx::mbar_arrive_expect_tx(&ctl->full[s], 2u * kStageTx);
                    uint8_t* a = left + s * kLeftBytes;
                    uint8_t* b = right + s * kRightBytes;
                    ptx::tma_load_2d_pair(a, &maps.left, k * kBK, row, bar);
                    if constexpr (MODE == kForward) {
                        ptx::tma_load_2d_pair(b, &maps.right, k * kBK, n0 + member * shape.N, bar);
                    } else {
#pragma unroll
                        for (int g = 0; g < BN / 128; ++g)
                            ptx::tma_load_2d_pair(b + g * (64 * kBK * 2), &maps.right, n0 + member * (BN / 2) + 64 * g, k * kBK, bar);
                    }
                    ctl->issued[s] = round + 1;
                    if (++s == kStages) { s = 0; ++round; }
                }
            }
            if (member)
                for (int i = 0; i < kStages; ++i)
                    ptx::st_cluster_u32(ptx::map_shared_to_cta(ptx::smem_u32(&ctl->peer_issued[i]), 0), (uint32_t)ctl->issued[i]);
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer (leader only) ----------------
        if (lane == 0 && member == 0) {
            constexpr uint32_t idesc = ptx::make_idesc_bf16(kRows, BN, false, MODE == kInputGrad);
            int s = 0, consumed = 0, turn = 0;
            uint32_t parity = 0;
            bool go = true;
            for (int tile = first_tile; tile < shape.tiles && go; tile += stride, ++turn) {
                const int b = turn & 1;
                if (turn >= 2 && !ptx::mbar_wait_spin(&ctl->drained[b], (uint32_t)((turn >> 1) - 1) & 1u, wait_limit)) {
                    *abort_flag = 1;
                    break;
                }
                ptx::tc_fence_after();
                const uint32_t tmem_d = tmem_base + b * BN;
                for (int k = 0; k < shape.steps; ++k) {
                    if (*abort_flag || !ptx::mbar_wait_spin(&ctl->full[s], parity, wait_limit)) {
                        *abort_flag = 1;
                        go = false;
                        break;
                    }
                    ++consumed;
                    ptx::tc_fence_after();
                    const uint32_t a_addr = ptx::smem_u32(left + s * kLeftBytes), b_addr = ptx::smem_u32(right + s * kRightBytes);
#pragma unroll
                    for (int kk = 0; kk < kBK / 16; ++kk) {
                        const uint64_t ad = ptx::make_smem_desc_sw128(a_addr + kk * 32, 16, 1024);
                        const uint64_t bd = MODE == kForward ? ptx::make_smem_desc_sw128(b_addr + kk * 32, 16, 1024)
                                                             : ptx::make_smem_desc_sw128(b_addr + kk * 2048, 64 * kBK * 2, 1024);
                        ptx::umma_bf16_pair(tmem_d, ad, bd, idesc, (k | kk) ? 1u : 0u);
                    }
                    ptx::umma_commit_pair(&ctl->empty[s], 3);
                    if (++s == kStages) { s = 0; parity ^= 1u; }
                }
                if (go) ptx::umma_commit_pair(&ctl->ready[b], 3);
            }
            ctl->consumed = consumed;
            ptx::umma_commit_pair(&ctl->done, 3);
        }
    } else {
        // ---------------- epilogue: accumulator -> h, a, u or dx (both CTAs, each its own 128 rows) ----------------
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        constexpr int kStores = stores_per_warp(MODE);
        uint8_t* mine = squares + (warp - 2) * kStores * kStoreBytes;
        const uint32_t mine_addr = ptx::smem_u32(mine);
        const uint32_t drained0 = ptx::map_shared_to_cta(ptx::smem_u32(&ctl->drained[0]), 0);
        int turn = 0, square = 0;
        for (int tile = first_tile; tile < shape.tiles; tile += stride, ++turn) {
            const int b = turn & 1;
            bool ok = ptx::mbar_wait_warp(&ctl->ready[b], (uint32_t)(turn >> 1) & 1u, wait_limit);
            ok = __all_sync(kFullMask, ok && !*abort_flag);
            if (!ok) { *abort_flag = 1; break; }
            ptx::tc_fence_after();
            const int row = (tile / shape.tiles_n) * kRows + member * 128 + quarter * 32;
            const uint32_t tmem = tmem_base + ((uint32_t)(32 * quarter) << 16) + b * BN;
            if constexpr (MODE == kForward) {
                constexpr int kHidden = BN / 2, kChunks = kHidden / 64;
                const int n0 = (tile % shape.tiles_n) * kHidden;
#pragma unroll 1
                for (int ch = 0; ch < kChunks; ++ch) {
                    const int c = half * (kHidden / 2) + ch * 32;
                    uint32_t ra[32], ru[32];
                    ptx::tmem_ld_32x32(tmem + c, ra);
                    ptx::tmem_ld_32x32(tmem + kHidden + c, ru);
                    ptx::tmem_ld_wait();
                    if (ch == kChunks - 1) {        // the accumulator is in registers: the next tile but one may have it
                        ptx::tc_fence_before();
                        __syncwarp();
                        if (lane == 0) ptx::mbar_arrive_cluster(drained0 + 8u * b);
                    }
                    if (row >= shape.M || n0 + c >= shape.N) continue;
                    float a[32], u[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) a[e] = __uint_as_float(ra[e]), u[e] = __uint_as_float(ru[e]);
                    if (shape.bias) {
                        add_bias(a, shape.bias, n0 + c, shape.N);
                        add_bias(u, shape.bias + shape.N, n0 + c, shape.N);
                    }
                    if (lane == 0) ptx::bulk_wait_read<0>();         // the squares of the chunk before have been read
                    __syncwarp();
                    if (shape.keep) {
                        stage_row(mine_addr + kStoreBytes, lane, a);
                        stage_row(mine_addr + 2 * kStoreBytes, lane, u);
                    }
#pragma unroll
                    for (int e = 0; e < 32; ++e) a[e] = gate_value<GATE, true>(a[e]) * u[e];
                    stage_row(mine_addr, lane, a);
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        ptx::tma_store_2d(&maps.out[0], mine, n0 + c, row);
                        if (shape.keep) {
                            ptx::tma_store_2d(&maps.out[1], mine + kStoreBytes, n0 + c, row);
                            ptx::tma_store_2d(&maps.out[2], mine + 2 * kStoreBytes, n0 + c, row);
                        }
                        ptx::bulk_commit();
                    }
                }
            } else {
                constexpr int kChunks = BN / 64;
                const int n0 = (tile % shape.tiles_n) * BN;
#pragma unroll 1
                for (int ch = 0; ch < kChunks; ++ch) {
                    const int c = half * (BN / 2) + ch * 32;
                    uint32_t r[32];
                    ptx::tmem_ld_32x32(tmem + c, r);
                    ptx::tmem_ld_wait();
                    if (ch == kChunks - 1) {
                        ptx::tc_fence_before();
                        __syncwarp();
                        if (lane == 0) ptx::mbar_arrive_cluster(drained0 + 8u * b);
                    }
                    if (row >= shape.M || n0 + c >= shape.N) continue;
                    float v[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = __uint_as_float(r[e]);
                    if (lane == 0) ptx::bulk_wait_read<1>();         // two squares in turn
                    __syncwarp();
                    stage_row(mine_addr + square * kStoreBytes, lane, v);
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        ptx::tma_store_2d(&maps.out[0], mine + square * kStoreBytes, n0 + c, row);
                        ptx::bulk_commit();
                    }
                    square ^= 1;
                }
            }
        }
        if (lane == 0) ptx::bulk_wait<0>();
    }

    // Neither CTA leaves while the other may still signal its barriers or read its shared memory.  After a wait was given up, copies may be in
    // flight whose stage the MMA thread never took, and one CTA may have issued a stage that the other did not: the leader squares the accounts
    // of those barriers by hand (bytes that were announced but never sent are counted as arrived; bytes that were sent unannounced get
    // their arrival) and waits for the rest, between two cluster barriers that keep the other CTA alive.
    __syncthreads();
    if (member && threadIdx.x == 0 && *abort_flag)
        ptx::st_cluster_u32(ptx::map_shared_to_cta(ptx::smem_u32(&ctl->peer_abort), 0), 1u);
    ptx::cluster_sync_all();
    if (!member && threadIdx.x == 0 && (*abort_flag || *reinterpret_cast<volatile int*>(&ctl->peer_abort))) {
        *abort_flag = 1;
        const int consumed = ctl->consumed;
        for (int s = 0; s < kStages; ++s) {
            const int taken = consumed > s ? (consumed - s + kStages - 1) / kStages : 0;      // rounds of slot s that the MMAs took
            const int mine = ctl->issued[s], theirs = *reinterpret_cast<volatile int*>(&ctl->peer_issued[s]);
            if (mine <= taken && theirs <= taken) continue;
            uint64_t* bar = &ctl->full[s];
            if (mine <= taken) ptx::mbar_arrive_expect_tx(bar, kStageTx);
            else if (theirs <= taken) ptx::mbar_complete_tx(bar, kStageTx);
            ptx::mbar_wait(bar, (uint32_t)taken & 1u, kWaitLimit);
        }
    }
    ptx::tc_fence_before();
    ptx::cluster_sync_all();
    if (warp == 1) {
        // tensor memory is given back by both CTAs, and only once no MMA can still write to it
        ptx::mbar_wait_warp(&ctl->done, 0, kWaitLimit);
        ptx::tc_fence_after();
        ptx::tmem_dealloc_pair(tmem_base, kColumns);
    }
    if (*abort_flag && threadIdx.x == 0 && dev_status) atomicExch(dev_status, (int)DROPIT_ERR_TIMEOUT);
}

using Kernel = void (*)(Maps, Shape, int32_t*, uint32_t);
Kernel forward_kernel(dropit_gate gate) {
    return gate == DROPIT_GATE_SILU ? gated_tc_kernel<kForward, 256, DROPIT_GATE_SILU>
           : gate == DROPIT_GATE_GELU ? gated_tc_kernel<kForward, 256, DROPIT_GATE_GELU> : gated_tc_kernel<kForward, 256, DROPIT_GATE_RELU>;
}

// How many pairs run at the same time (some SMs may have no partner).
int resident_pairs(Kernel kernel, size_t smem) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int v = 0;
    if (cudaOccupancyMaxActiveClusters(&v, kernel, &cfg) != cudaSuccess || v <= 0) v = sm_count() / 2;
    (void)cudaGetLastError();
    return v;
}

// What a kernel needs once per device: its shared memory allowed, and the number of pairs.
struct PerDevice {
    std::atomic<int> pairs[64];
    int get(Kernel kernel, size_t smem) {
        const int dev = current_device();
        int v = dev >= 0 && dev < 64 ? pairs[dev].load(std::memory_order_acquire) : 0;
        if (v) return v;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) {
            (void)cudaGetLastError();
            return 0;
        }
        v = resident_pairs(kernel, smem);
        if (dev >= 0 && dev < 64) pairs[dev].store(v, std::memory_order_release);
        return v;
    }
};

dropit_status launch(Kernel kernel, size_t smem, PerDevice& device, const Maps& maps, const Shape& shape, int32_t* dev_status, cudaStream_t stream) {
    const int pairs = device.get(kernel, smem);
    if (!pairs) return DROPIT_ERR_CUDA;
    kernel<<<2 * std::min(pairs, shape.tiles), kThreads, smem, stream>>>(maps, shape, dev_status, spin_limit(kWaitLimit));
    return check_launch();
}

}  // namespace

bool gated_tc_takes(int64_t M, int64_t C, int64_t H) { return M >= 1 && C % 8 == 0 && H % 8 == 0; }

dropit_status gated_tc_forward(const void* x, const void* w, const void* bias, int64_t M, int64_t C, int64_t H, dropit_gate gate, void* h, void* gu,
                               int32_t* dev_status, cudaStream_t stream) {
    constexpr int BN = 256;
    Maps maps = {};
    uint16_t* kept = reinterpret_cast<uint16_t*>(gu);
    if (!make_map_2d_bf16(&maps.left, x, M, C, 128) || !make_map_2d_bf16(&maps.right, w, 2 * H, C, BN / 2) || !make_map_out_bf16(&maps.out[0], h, M, H, H))
        return DROPIT_ERR_CUDA;
    if (gu && (!make_map_out_bf16(&maps.out[1], kept, M, H, 2 * H) || !make_map_out_bf16(&maps.out[2], kept + H, M, H, 2 * H))) return DROPIT_ERR_CUDA;
    Shape s = {};
    s.M = (int)M;
    s.K = (int)C;
    s.N = (int)H;
    s.tiles_n = (int)((H + BN / 2 - 1) / (BN / 2));
    s.tiles = (int)((M + kRows - 1) / kRows) * s.tiles_n;
    s.steps = (int)((C + kBK - 1) / kBK);
    s.keep = gu != nullptr;
    s.bias = reinterpret_cast<const uint16_t*>(bias);
    static PerDevice device[3];
    return launch(forward_kernel(gate), smem_bytes(kForward, BN), device[gate], maps, s, dev_status, stream);
}

dropit_status gated_tc_input_grad(const void* dgu, const void* w, int64_t M, int64_t C, int64_t H, void* dx, int32_t* dev_status, cudaStream_t stream) {
    constexpr int BN = 256;
    Maps maps = {};
    if (!make_map_2d_bf16(&maps.left, dgu, M, 2 * H, 128) || !make_map_2d_bf16(&maps.right, w, 2 * H, C, kBK) || !make_map_out_bf16(&maps.out[0], dx, M, C, C))
        return DROPIT_ERR_CUDA;
    Shape s = {};
    s.M = (int)M;
    s.K = (int)(2 * H);
    s.N = (int)C;
    s.tiles_n = (int)((C + BN - 1) / BN);
    s.tiles = (int)((M + kRows - 1) / kRows) * s.tiles_n;
    s.steps = (int)((2 * H + kBK - 1) / kBK);
    static PerDevice device;
    return launch(gated_tc_kernel<kInputGrad, BN, 0>, smem_bytes(kInputGrad, BN), device, maps, s, dev_status, stream);
}

}  // namespace dropit
