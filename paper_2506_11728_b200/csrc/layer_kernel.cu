// Dense kernel of the 8-bit transformer layer: exact int8 sums on the tensor cores, and behind them, in the
// same kernel, the scales, bias, activation, residual, gating or the gradient of the gating.
//
// Main loop.  As in the plain integer product: persistent CTAs (or CTA pairs, cta_group::2) walk 128 x block_n
// (256 x block_n) tiles; one TMA producer warp per operand fills 128-byte-swizzled shared-memory stages of 128
// bytes of K, one warp issues tcgen05.mma.kind::i8 into one of two accumulators in tensor memory, so that the
// epilogue of a tile runs beside the next tile's main loop.
//
// Gated forms.  One accumulator of block_n columns holds both projections of block_n / 2 output columns: the B
// tile of a stage is made of block_n / 2 rows of the gate weights followed by as many rows of the other
// projection's, so one MMA (N = block_n) advances both and the tokens are staged once for the two.  In the pair
// form each CTA stages one projection whole: the tile's halves are the halves cta_group::2 asks for.
//
// Epilogue: layer_epilogue.cuh.
//
// What bounds it.  Long K: the tensor cores, and over more than a few calls the power limit (gated 16384 x 14336 x 4096
// bf16: 3440 TOPS in a short burst, 2870 sustained at 1.26 GHz; linear 16384 x 4096 x 11008 with residual 2630 sustained).
// Short K: the epilogue's arithmetic.  Few tiles: the chain launch - first copies - last epilogue, 8 to 11 us from 128
// to 1024 tokens of 4096 outputs.  Both projections in one accumulator make the gated block one pass over the tokens and
// write H alone: G and U never leave the SM.
//
// Every wait is bounded.  A kernel that gives one up unwinds: all roles of both CTAs stop, copies (unwind.cuh) and MMAs in
// flight are awaited, tensor memory is released, bit 0 of *status is set.
#include <algorithm>

#include "layer_epilogue.cuh"
#include "unwind.cuh"

namespace mip {

namespace {

template <bool kPair, int kOp, bool kWide, int kEpiWarps>
__global__ void __launch_bounds__(32 * (3 + kEpiWarps), 1)
mip_layer_kernel(const __grid_constant__ LayerParams p) {
    constexpr int kGroup = kPair ? 2 : 1;
    constexpr bool kGatedForm = kOp == kOpGated || kOp == kOpGatedGrad || kOp == kOpRawGated;
    constexpr bool kRaw = kOp == kOpRaw || kOp == kOpRawGated;
    constexpr int kRowsPerTile = kPair ? 2 * kBlockM : kBlockM;
    constexpr int kBuffers = slot_count(kOp);
    constexpr int kSlotBytesPerWarp = slot_bytes_per_warp(kOp, kWide);
    const uint32_t cta_rank = kPair ? cluster_ctarank() : 0u;
    const bool leader = cta_rank == 0;
    const int first_unit = kPair ? static_cast<int>(blockIdx.x >> 1) : static_cast<int>(blockIdx.x);
    const int unit_stride = kPair ? static_cast<int>(gridDim.x >> 1) : static_cast<int>(gridDim.x);
    const int b_rows = kPair ? (p.block_n >> 1) : p.block_n;       // rows of B staged by this CTA
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    const uint32_t pad = ((raw_addr + 1023u) & ~1023u) - raw_addr;
    uint8_t* smem = smem_raw + pad;
    const uint32_t smem_base = raw_addr + pad;
    constexpr uint32_t a_bytes = kBlockM * 128;
    const uint32_t b_bytes = b_rows * 128;
    const uint32_t stage_bytes = a_bytes + b_bytes;
    // shared memory: [stages x (A | B)] [slots of the epilogue warps] [their column vectors] [control block]
    const uint32_t slots = smem_base + p.stages * stage_bytes;
    const uint32_t colvec = slots + kEpiWarps * kSlotBytesPerWarp;
    const uint32_t ctrl = colvec + kEpiWarps * kColBytes;
    const uint32_t bar_full = ctrl;
    const uint32_t bar_empty = bar_full + 8u * p.stages;
    const uint32_t bar_tfull = bar_empty + 8u * p.stages;
    const uint32_t bar_tempty = bar_tfull + 16u;
    const uint32_t bar_drain = bar_tempty + 16u;
    const uint32_t bar_in = ctrl + 256u;                           // kEpiWarps x kBuffers: a slot's tile has arrived
    uint8_t* ctrl_ptr = smem + (ctrl - smem_base);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ctrl_ptr + 16 * p.stages + 40);
    volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(tmem_slot + 1);
    const UnwindWords unwind = {ctrl + 16u * p.stages + 48u};
    static_assert(16 * kMaxLayerStages + 48 + UnwindWords::kBytes <= 256, "control block");

    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(bar_full + 8u * s, 2);                       // two producers
            mbar_init(bar_empty + 8u * s, 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(bar_tfull + 8u * a, 1);
            mbar_init(bar_tempty + 8u * a, kPair ? 2 * kEpiWarps : kEpiWarps);
        }
        mbar_init(bar_drain, 1);
        for (int i = 0; i < kEpiWarps * kBuffers; ++i) mbar_init(bar_in + 8u * i, 1);
        *abort_flag = 0;
        fence_mbar_init();
        tma_prefetch_desc(&p.tmap_a);
        tma_prefetch_desc(&p.tmap_b0);
        if (kGatedForm) tma_prefetch_desc(&p.tmap_b1);
        if (p.r_tma) tma_prefetch_desc(&p.tmap_r);
        if (p.c_tma) tma_prefetch_desc(&p.tmap_c);
    }
    if (kPair) {   // the peer runs (see tmem_alloc), and its barriers are initialised before anything remote touches them
        __syncwarp();
        cluster_arrive();
        cluster_wait();
    }
    if (warp == 1) {
        tmem_alloc<kGroup>(smem_u32(tmem_slot), p.tmem_cols);
        tmem_relinquish<kGroup>();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait();          // from here on global memory is touched
    pdl_launch_dependents();      // (only now: one kernel at a time waits for another)
    const uint32_t tmem_base = *tmem_slot;
    const int total_units = layer_units(p);
    const uint64_t budget = p.wait_budget_ns;
    uint32_t issued = 0;

    if (warp == 0 || warp == 2 + kEpiWarps) {
        // ------------------------------------------------------------ TMA producers: A (warp 0), B (last warp)
        uint32_t s = 0, phase = 0;
        bool ok = true;
        const bool side_a = warp == 0;
        // (fewer than 128 rows in all: only those are copied -- rows a TMA copy has to fill with zeros cost it several
        // times those it reads -- and the accumulator rows behind them, never stored, add up what lies there)
        const uint32_t tx_bytes = kGroup * (side_a ? static_cast<uint32_t>(p.a_rows) * 128u : b_bytes);
        for (int unit = first_unit; unit < total_units && ok; unit += unit_stride) {
            const LayerTile tc = decode_tile(p, unit, kRowsPerTile);
            const int m_cta = tc.m0 + static_cast<int>(cta_rank) * kBlockM;
            const int half = p.block_n >> 1;
            for (int kb = tc.kb0; kb < tc.kb1; ++kb) {
                if (!mbar_wait_warp(bar_empty + 8u * s, phase ^ 1u, abort_flag, budget)) { ok = false; break; }
                const uint32_t full_local = bar_full + 8u * s;
                const uint32_t full = kPair ? mapa_u32(full_local, 0) : full_local;
                const uint32_t a_dst = smem_base + s * stage_bytes;
                const uint32_t b_dst = a_dst + a_bytes;
                if (elect_one()) {
                    if (leader) mbar_arrive_expect_tx(full_local, tx_bytes);
                    if (side_a) {
                        if (kPair) tma_load_2d_pair(a_dst, &p.tmap_a, full, kb * 128, m_cta);
                        else tma_load_2d(a_dst, &p.tmap_a, full, kb * 128, m_cta);
                    } else if (!kGatedForm) {
                        if (kPair) tma_load_2d_pair(b_dst, &p.tmap_b0, full, kb * 128, tc.n0 + static_cast<int>(cta_rank) * b_rows);
                        else tma_load_2d(b_dst, &p.tmap_b0, full, kb * 128, tc.n0);
                    } else if (kPair) {          // one projection per CTA of the pair
                        tma_load_2d_pair(b_dst, leader ? &p.tmap_b0 : &p.tmap_b1, full, kb * 128, tc.n0);
                    } else {
                        tma_load_2d(b_dst, &p.tmap_b0, full, kb * 128, tc.n0);
                        tma_load_2d(b_dst + half * 128, &p.tmap_b1, full, kb * 128, tc.n0);
                    }
                }
                ++issued;
                if (++s == static_cast<uint32_t>(p.stages)) { s = 0; phase ^= 1u; }
            }
        }
        if (lane == 0) unwind.put(side_a ? 0 : 1, issued);
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer
        if (leader) {
            uint32_t s = 0, phase = 0;
            bool ok = true;
            int t = 0;
            for (int unit = first_unit; unit < total_units && ok; unit += unit_stride, ++t) {
                const LayerTile tc = decode_tile(p, unit, kRowsPerTile);
                const uint32_t acc = t & 1, acc_phase = (t >> 1) & 1;
                if (!mbar_wait_warp<kPair>(bar_tempty + 8u * acc, acc_phase ^ 1u, abort_flag, budget)) { ok = false; break; }
                tc_fence_after();
                const uint32_t d_tmem = tmem_base + acc * p.block_n;
                for (int kb = tc.kb0; kb < tc.kb1; ++kb) {
                    if (!mbar_wait_warp(bar_full + 8u * s, phase, abort_flag, budget)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t a_addr = smem_base + s * stage_bytes;
                    const uint64_t a_desc = make_kmajor_desc(a_addr, 128);
                    const uint64_t b_desc = make_kmajor_desc(a_addr + a_bytes, 128);
                    const uint32_t empty_local = bar_empty + 8u * s;
                    const uint32_t empty_peer = kPair ? mapa_u32(empty_local, 1) : 0u;
                    if (elect_one()) {
#pragma unroll
                        for (uint32_t k = 0; k < 4; ++k)
                            mma_i8<kGroup>(d_tmem, a_desc + 2ull * k, b_desc + 2ull * k, p.idesc, (kb > tc.kb0 || k > 0) ? 1u : 0u);
                        if (kPair) {
                            mma_commit_pair(empty_local);
                            mma_commit_pair(empty_peer);
                        } else {
                            mma_commit(empty_local);
                        }
                    }
                    if (++s == static_cast<uint32_t>(p.stages)) { s = 0; phase ^= 1u; }
                }
                if (ok && !(p.debug_flags & 1)) {   // (test hook, bit 0: the "accumulator ready" signal is withheld)
                    const uint32_t tfull_local = bar_tfull + 8u * acc;
                    const uint32_t tfull_peer = kPair ? mapa_u32(tfull_local, 1) : 0u;
                    if (elect_one()) {
                        if (kPair) {
                            mma_commit_pair(tfull_local);
                            mma_commit_pair(tfull_peer);
                        } else {
                            mma_commit(tfull_local);
                        }
                    }
                }
            }
        }
    } else {
        if constexpr (kRaw)
            raw_epilogue<kPair, kGatedForm, kEpiWarps / 4>(p, (warp - 2) >> 2, bar_tfull, bar_tempty, abort_flag, tmem_base, warp & 3, lane,
                                                           cta_rank, first_unit, unit_stride);
        else
            layer_epilogue<kPair, kOp, kWide, kEpiWarps>(p, slots, colvec, bar_in, bar_tfull, bar_tempty, abort_flag, tmem_base, warp - 2, warp & 3,
                                              lane, cta_rank, first_unit, unit_stride);
    }

    __syncwarp();
    tc_fence_before();
    __syncthreads();
    bool unwinding = *abort_flag != 0;
    if (kPair) {   // both CTAs have stopped, and know it of each other
        if (threadIdx.x == 0) unwind.tell(cta_rank ^ 1u, *abort_flag);
        __syncwarp();
        cluster_arrive();
        cluster_wait();
        unwinding = unwinding || unwind.get(0) != 0;
    }
    if (unwinding) {
        if (warp == 0 && leader)
            drain_copies<kPair, 2>(unwind, bar_full, static_cast<uint32_t>(p.stages), static_cast<uint32_t>(p.a_rows) * 128u, b_bytes, lane, budget);
        if (warp == 1 && leader) {
            if (elect_one()) {
                if (kPair) mma_commit_pair(bar_drain); else mma_commit(bar_drain);
            }
            __syncwarp();
            const uint64_t t0 = globaltimer_ns();
            while (!mbar_try_wait(bar_drain, 0)) {
                if (globaltimer_ns() - t0 > budget) break;
            }
            __syncwarp();
            tc_fence_before();
        }
        __syncthreads();
        if (kPair) {   // (the peer's shared memory is still being written or read until here)
            cluster_arrive();
            cluster_wait();
        }
    }
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc<kGroup>(tmem_base, p.tmem_cols);
    }
    if (threadIdx.x == 0 && *abort_flag != 0) atomicOr(p.status, 1u);
}

template <bool kPair, int kOp, bool kWide, int kEpiWarps>
cudaError_t launch_t(const LayerParams& p, const cudaLaunchConfig_t& cfg) {
    return cudaLaunchKernelEx(&cfg, mip_layer_kernel<kPair, kOp, kWide, kEpiWarps>, p);
}
template <bool kPair, int kOp, bool kWide, int kEpiWarps>
cudaError_t init_t() {
    return cudaFuncSetAttribute(mip_layer_kernel<kPair, kOp, kWide, kEpiWarps>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBudget);
}
template <bool kPair, int kOp>
cudaError_t init_op() {
    for (cudaError_t e : {init_t<kPair, kOp, false, kFewEpiWarps>(), init_t<kPair, kOp, false, kManyEpiWarps>(), init_t<kPair, kOp, true, kFewEpiWarps>()})
        if (e != cudaSuccess) return e;
    return cudaSuccess;
}
template <bool kPair, int kOp>
cudaError_t launch_op(const LayerParams& p, const cudaLaunchConfig_t& cfg) {
    if (p.type == kF32) return launch_t<kPair, kOp, true, kFewEpiWarps>(p, cfg);
    return p.epi_warps == kManyEpiWarps ? launch_t<kPair, kOp, false, kManyEpiWarps>(p, cfg) : launch_t<kPair, kOp, false, kFewEpiWarps>(p, cfg);
}

}  // namespace

// (partial sums are words: the float32 form's slots)
int layer_fixed_smem(int op, bool wide, int epi_warps) {
    return epi_warps * (slot_bytes_per_warp(op, wide) + kColBytes) + kCtrlBytes + 1024;
}

cudaError_t layer_init() {
    for (cudaError_t e : {init_op<false, kOpLinear>(), init_op<true, kOpLinear>(), init_op<false, kOpGated>(), init_op<true, kOpGated>(),
                          init_op<false, kOpGatedGrad>(), init_op<true, kOpGatedGrad>(), init_t<false, kOpRaw, true, kFewEpiWarps>(),
                          init_t<true, kOpRaw, true, kFewEpiWarps>(), init_t<false, kOpRawGated, true, kFewEpiWarps>(),
                          init_t<true, kOpRawGated, true, kFewEpiWarps>()})
        if (e != cudaSuccess) return e;
    return cudaSuccess;
}

cudaError_t launch_layer(const LayerParams& p, int op, int pair, int grid, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(grid), 1, 1);
    cfg.blockDim = dim3(static_cast<unsigned>(32 * (3 + p.epi_warps)), 1, 1);
    cfg.dynamicSmemBytes = std::max(kSmemFloor, static_cast<size_t>(p.stages) * (kBlockM + (pair ? p.block_n / 2 : p.block_n)) * 128 +
                                                    layer_fixed_smem(op, p.type == kF32, p.epi_warps));
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_allowed();
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pair ? 2 : 1;
    switch (op) {
        case kOpRaw: return pair ? launch_t<true, kOpRaw, true, kFewEpiWarps>(p, cfg) : launch_t<false, kOpRaw, true, kFewEpiWarps>(p, cfg);
        case kOpRawGated: return pair ? launch_t<true, kOpRawGated, true, kFewEpiWarps>(p, cfg) : launch_t<false, kOpRawGated, true, kFewEpiWarps>(p, cfg);
        case kOpLinear: return pair ? launch_op<true, kOpLinear>(p, cfg) : launch_op<false, kOpLinear>(p, cfg);
        case kOpGated: return pair ? launch_op<true, kOpGated>(p, cfg) : launch_op<false, kOpGated>(p, cfg);
        default: return pair ? launch_op<true, kOpGatedGrad>(p, cfg) : launch_op<false, kOpGatedGrad>(p, cfg);
    }
}

}  // namespace mip
