// C = A diag(s) B with A bfloat16 and B 8-bit codes [K][N]: the products of a backward pass through 8-bit weights
// (dX, scales of the weights' rows) and 8-bit activations (dW, scales of the tokens).
//
// The scales lie along the summed axis, so they cannot be applied behind the sum: each code times its row's scale is
// rounded to bfloat16 on its way to the tensor core (codes alone are exact in bfloat16), and tcgen05.mma.kind::f16
// multiplies it with A into binary32.  The codes cross HBM and L2 as bytes; nothing is written back in 16 bits.
//
// Roles.  Warp 0 loads A (TMA, 128-byte swizzle, K-major or M-major as it lies), warp 1 issues the MMAs, then four or eight
// (16-bit results) epilogue warps (layer_epilogue.cuh), one that loads B's codes (TMA, 64 rows x 128 bytes, plain rows),
// and eight that convert, two groups by turns: a lane takes 16 codes of a row (one 16-byte read, eight lanes a row), scales them and writes the two
// 16-byte pieces of the N-major 128-byte-swizzled tile the tensor core reads.  Lanes of the row's second half write
// their pieces in the other order, so that eight lanes cover all banks.  A stage is 64 k: 16 KB of A, 8 KB of codes,
// 16 KB of converted B per CTA.  In the pair form (256 x 256 tile, cta_group::2) each CTA converts its half of B, so
// the conversion -- 16 codes per clock and SM at the tensor core's pace, against 32 for a CTA of its own -- hides.
//
// What bounds it: shared memory.  A stage writes 16 KB of A, 8 KB of codes and 16 KB of converted B, and reads the codes
// and both operands once more: 80 KB at 128 bytes a clock are 640 clocks against the 512 of its products, 670 measured.
// 22016 x 4096 x 8192: 1360 TFLOP/s in a short burst, 1120 sustained under the power limit (the library's bf16 product
// 1620 and 1360).
//
// Every wait is bounded, with the unwinding of the dense layer kernel.
#include <algorithm>

#include "layer_epilogue.cuh"
#include "stage_waits.h"
#include "unwind.cuh"

namespace mip {

namespace {

constexpr int kConvWarps = 8;
constexpr int product_threads(bool wide) { return 32 * (3 + product_epi_warps(wide) + kConvWarps); }
constexpr uint32_t kABytes = kBlockM * kProductK * 2;          // 16 KB
constexpr uint32_t kBBytes = kProductN * kProductK * 2;        // 16 KB, two blocks of 64 columns
constexpr uint32_t kRawBytes = kProductN * kProductK;          // 8 KB
constexpr uint32_t kProductStage = kABytes + kBBytes + kRawBytes;
constexpr uint32_t kScaleBytes = kProductK * 4;                // the rows' scales, behind the stages
constexpr int kProductSlots = 4 * slot_bytes_per_warp(kOpProduct, true);       // (as much as 8 warps' 16-bit slots)
static_assert(product_epi_warps(false) * slot_bytes_per_warp(kOpProduct, false) <= kProductSlots && product_epi_warps(true) == 4, "slots");
constexpr int kProductFixed = kProductSlots + kCtrlBytes + 1024;

// Four codes (the bytes of w) times s (twice, packed), rounded to bfloat16.  A byte with its sign bit flipped, put
// behind the exponent of 2^23, is the float 2^23 + 128 + code: one byte permutation per code and one exact packed
// subtraction per two instead of conversion instructions, which run at a quarter of their rate or less.
__device__ __forceinline__ void scale_codes(uint32_t w, uint64_t ss, uint32_t& lo, uint32_t& hi) {
    constexpr uint64_t kBias = 0xCB000080CB000080ull;              // -(2^23 + 128), twice
    w ^= 0x80808080u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint64_t v;
        asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "r"(__byte_perm(w, 0x4B000000u, 0x7540u + 2 * h)),
            "r"(__byte_perm(w, 0x4B000000u, 0x7541u + 2 * h)));
        asm("add.rn.f32x2 %0, %0, %1;" : "+l"(v) : "l"(kBias));
        asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(v) : "l"(ss));
        float a, b;
        asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
        (h ? hi : lo) = pack2(a, b, false);
    }
}

template <bool kPair, bool kAMajorM, bool kWide, bool kRaw>
__global__ void __launch_bounds__(product_threads(kWide), 1)
mip_product_kernel(const __grid_constant__ LayerParams p) {
    constexpr int kGroup = kPair ? 2 : 1;
    constexpr int kEpiWarps = product_epi_warps(kWide);
    constexpr int kFirstConvWarp = 3 + kEpiWarps;
    constexpr int kRowsPerTile = kGroup * kBlockM;
    const uint32_t cta_rank = kPair ? cluster_ctarank() : 0u;
    const bool leader = cta_rank == 0;
    const int first_unit = kPair ? static_cast<int>(blockIdx.x >> 1) : static_cast<int>(blockIdx.x);
    const int unit_stride = kPair ? static_cast<int>(gridDim.x >> 1) : static_cast<int>(gridDim.x);
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    const uint32_t pad = ((raw_addr + 1023u) & ~1023u) - raw_addr;
    uint8_t* smem = smem_raw + pad;
    const uint32_t smem_base = raw_addr + pad;
    const uint32_t stages = static_cast<uint32_t>(p.stages);
    const uint32_t slots = smem_base + stages * kProductStage;
    const uint32_t scales = slots + kProductSlots;
    const uint32_t ctrl = scales + stages * kScaleBytes;
    // control block, 8 bytes each: A has arrived | B is converted | A and B have been read | codes have arrived | codes
    // have been read (`stages` of each), accumulators full and empty, drain, arrivals in the slots
    const uint32_t bar_a = ctrl;
    const uint32_t bar_b = ctrl + 64u;
    const uint32_t bar_empty = ctrl + 128u;
    const uint32_t bar_raw = ctrl + 192u;
    const uint32_t bar_rawfree = ctrl + 256u;
    const uint32_t bar_tfull = ctrl + 320u;
    const uint32_t bar_tempty = ctrl + 336u;
    const uint32_t bar_drain = ctrl + 352u;
    const uint32_t bar_in = ctrl + 384u;
    uint8_t* ctrl_ptr = smem + (ctrl - smem_base);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ctrl_ptr + 360);
    volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(ctrl_ptr + 364);
    const UnwindWords unwind = {bar_in + 8u * kEpiWarps * slot_count(kOpProduct)};
    static_assert(384 + 8 * kEpiWarps * slot_count(kOpProduct) + UnwindWords::kBytes <= kCtrlBytes, "control block");

    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < stages; ++s) {
            mbar_init(bar_a + 8u * s, 1);
            mbar_init(bar_b + 8u * s, kGroup * kConvWarps / 2);
            mbar_init(bar_empty + 8u * s, 1);
            mbar_init(bar_raw + 8u * s, 33);     // the copy of the codes, and every lane's copy of two scales
            mbar_init(bar_rawfree + 8u * s, kConvWarps / 2);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(bar_tfull + 8u * a, 1);
            mbar_init(bar_tempty + 8u * a, kGroup * kEpiWarps);
        }
        mbar_init(bar_drain, 1);
        for (int i = 0; i < kEpiWarps * slot_count(kOpProduct); ++i) mbar_init(bar_in + 8u * i, 1);
        *abort_flag = 0;
        fence_mbar_init();
        tma_prefetch_desc(&p.tmap_a);
        tma_prefetch_desc(&p.tmap_b0);
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
    uint32_t issued = 0;       // stages whose copies this warp (0: A, 6: codes) has asked for
    uint32_t s = 0, phase = 0;
    const auto advance = [&] { if (++s == stages) { s = 0; phase ^= 1u; } };

    if (warp == 0) {
        // ------------------------------------------------------------ A
        bool ok = true;
        for (int unit = first_unit; unit < total_units && ok; unit += unit_stride) {
            const LayerTile tc = decode_tile(p, unit, kRowsPerTile);
            const int m_cta = tc.m0 + static_cast<int>(cta_rank) * kBlockM;
            for (int kb = tc.kb0; kb < tc.kb1; ++kb) {
                if (!mbar_wait_warp(bar_empty + 8u * s, phase ^ 1u, abort_flag, budget)) { ok = false; break; }
                const uint32_t local = bar_a + 8u * s;
                const uint32_t full = kPair ? mapa_u32(local, 0) : local;     // both CTAs' bytes complete on the leader's
                const uint32_t dst = smem_base + s * kProductStage;
                if (elect_one()) {
                    if (leader) mbar_arrive_expect_tx(local, kGroup * kABytes);
                    if (kAMajorM) {          // two blocks of 64 rows of the tile
                        for (int i = 0; i < 2; ++i) {
                            if (kPair) tma_load_2d_pair(dst + i * (kABytes / 2), &p.tmap_a, full, m_cta + 64 * i, kb * kProductK);
                            else tma_load_2d(dst + i * (kABytes / 2), &p.tmap_a, full, m_cta + 64 * i, kb * kProductK);
                        }
                    } else {
                        if (kPair) tma_load_2d_pair(dst, &p.tmap_a, full, kb * kProductK, m_cta);
                        else tma_load_2d(dst, &p.tmap_a, full, kb * kProductK, m_cta);
                    }
                }
                ++issued;
                advance();
            }
        }
        if (lane == 0) unwind.put(0, issued);
    } else if (warp == 2 + kEpiWarps) {
        // ------------------------------------------------------------ codes of B
        bool ok = true;
        if (!p.b0_scale)         // no scales: ones, written once
            for (uint32_t i = lane; i < stages * kProductK; i += 32) sts_f32(scales + i * 4u, 1.0f);
        for (int unit = first_unit; unit < total_units && ok; unit += unit_stride) {
            const LayerTile tc = decode_tile(p, unit, kRowsPerTile);
            const int n_cta = tc.n0 + static_cast<int>(cta_rank) * kProductN;
            for (int kb = tc.kb0; kb < tc.kb1; ++kb) {
                if (!mbar_wait_warp(bar_rawfree + 8u * s, phase ^ 1u, abort_flag, budget)) { ok = false; break; }
                if (elect_one()) {
                    mbar_arrive_expect_tx(bar_raw + 8u * s, kRawBytes);
                    tma_load_2d(smem_base + s * kProductStage + kABytes + kBBytes, &p.tmap_b0, bar_raw + 8u * s, n_cta, kb * kProductK);
                }
                // the rows' scales: 4-byte asynchronous copies (the vector has no alignment beyond that), two per lane,
                // rows beyond K zero; every lane's arrival follows its copies
                if (p.b0_scale) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int k = kb * kProductK + h * 32 + lane;
                        const uint32_t bytes = k < p.K ? 4u : 0u;
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;"
                                     ::"r"(scales + s * kScaleBytes + static_cast<uint32_t>(h * 32 + lane) * 4u),
                                       "l"(__cvta_generic_to_global(p.b0_scale + (k < p.K ? k : 0))), "r"(bytes) : "memory");
                    }
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar_raw + 8u * s) : "memory");
                } else {
                    mbar_arrive(bar_raw + 8u * s);
                }
                ++issued;
                advance();
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer
        if (leader) {
            bool ok = true;
            int t = 0;
            for (int unit = first_unit; unit < total_units && ok; unit += unit_stride, ++t) {
                const LayerTile tc = decode_tile(p, unit, kRowsPerTile);
                const uint32_t acc = t & 1, acc_phase = (t >> 1) & 1;
                if (!mbar_wait_warp<kPair>(bar_tempty + 8u * acc, acc_phase ^ 1u, abort_flag, budget)) { ok = false; break; }
                tc_fence_after();
                const uint32_t d_tmem = tmem_base + acc * p.block_n;
                for (int kb = tc.kb0; kb < tc.kb1; ++kb) {
                    if (!mbar_wait_warp(bar_a + 8u * s, phase, abort_flag, budget) ||
                        !mbar_wait_warp<kPair>(bar_b + 8u * s, phase, abort_flag, budget)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t a_addr = smem_base + s * kProductStage;
                    const uint64_t a_desc = kAMajorM ? make_mnmajor_desc(a_addr, kABytes / 2) : make_kmajor_desc(a_addr, 128);
                    const uint64_t b_desc = make_mnmajor_desc(a_addr + kABytes, kBBytes / 2);
                    // 16 k per instruction: 32 bytes of a K-major row, 16 rows of 128 bytes of an M- or N-major block
                    constexpr uint64_t a_step = kAMajorM ? 128ull : 2ull, b_step = 128ull;
                    const uint32_t empty_local = bar_empty + 8u * s;
                    const uint32_t empty_peer = kPair ? mapa_u32(empty_local, 1) : 0u;
                    if (elect_one()) {
#pragma unroll
                        for (uint32_t k = 0; k < kProductK / 16; ++k)
                            mma_f16<kGroup>(d_tmem, a_desc + a_step * k, b_desc + b_step * k, p.idesc, (kb > tc.kb0 || k > 0) ? 1u : 0u);
                        if (kPair) {
                            mma_commit_pair(empty_local);
                            mma_commit_pair(empty_peer);
                        } else {
                            mma_commit(empty_local);
                        }
                    }
                    advance();
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
    } else if (warp >= kFirstConvWarp) {
        // ------------------------------------------------------------ codes -> bfloat16
        // Two groups of four warps take the stages in turn: the chain of one stage -- wait, read, convert, write, proxy
        // fence, arrive -- may then last as long as two of the tensor core's stages.
        const int cw = warp - kFirstConvWarp;
        const int j = lane & 7;                                    // 16 columns of the CTA's 128
        const int r0 = (cw & 3) * 16 + (lane >> 3);                // this lane's rows of a stage: r0 + 4 i, i < 4
        // its two 16-byte pieces inside the block of 64 columns; the second half of a row writes the odd one first
        const uint32_t flip = static_cast<uint32_t>(j >> 2);
        const uint32_t block = kABytes + flip * (kBBytes / 2);
        const uint32_t piece = static_cast<uint32_t>(j & 3) * 2u;
        uint32_t total = 0;                                        // stages this CTA converts
        for (int unit = first_unit; unit < total_units; unit += unit_stride) {
            const LayerTile tc = decode_tile(p, unit, kRowsPerTile);
            total += static_cast<uint32_t>(tc.kb1 - tc.kb0);
        }
        for (uint32_t it = static_cast<uint32_t>(cw >> 2); it < total; it += 2) {
            const uint32_t st = it % stages, ph = (it / stages) & 1u;
            const uint32_t stage = smem_base + st * kProductStage;
            // the tensor core has read what the buffer held; codes and scales are in place.  (Lanes decide together.)
            const auto wait = [&](StageWait what) {
                return what == kStageFree ? mbar_wait(bar_empty + 8u * st, ph ^ 1u, abort_flag, budget)
                                          : mbar_wait(bar_raw + 8u * st, ph, abort_flag, budget);
            };
            const bool ready = wait(kConverterFirst) && wait(kConverterSecond);
            if (!__all_sync(~0u, ready)) break;
            // (the second half of a row reads its two halves in the other order too, so no register is chosen by lane)
            uint32_t w[4][4];
            uint64_t ss[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t src = stage + kABytes + kBBytes + static_cast<uint32_t>(r0 + 4 * i) * 128u + static_cast<uint32_t>(j) * 16u;
                asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[i][0]), "=r"(w[i][1]) : "r"(src + flip * 8u) : "memory");
                asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[i][2]), "=r"(w[i][3]) : "r"(src + (flip ^ 1u) * 8u) : "memory");
                uint32_t sc;
                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(sc) : "r"(scales + st * kScaleBytes + static_cast<uint32_t>(r0 + 4 * i) * 4u) : "memory");
                asm("mov.b64 %0, {%1, %1};" : "=l"(ss[i]) : "r"(sc));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t r = static_cast<uint32_t>(r0 + 4 * i);
                uint32_t first[4], second[4];                      // eight columns each
                scale_codes(w[i][0], ss[i], first[0], first[1]);
                scale_codes(w[i][1], ss[i], first[2], first[3]);
                const uint32_t row = stage + block + r * 128u;
                st_shared_v4(row + (((piece + flip) ^ (r & 7u)) << 4), first);
                scale_codes(w[i][2], ss[i], second[0], second[1]);
                scale_codes(w[i][3], ss[i], second[2], second[3]);
                st_shared_v4(row + (((piece + (flip ^ 1u)) ^ (r & 7u)) << 4), second);
            }
            // the writes become visible to the tensor core, and the codes' bytes may be overwritten by the TMA
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
                if (kPair && !leader) mbar_arrive_remote_fenced(bar_b + 8u * st, 0);
                else mbar_arrive(bar_b + 8u * st);
                mbar_arrive(bar_rawfree + 8u * st);
            }
        }
    } else {
        if constexpr (kRaw)
            raw_epilogue<kPair, false, kEpiWarps / 4>(p, (warp - 2) >> 2, bar_tfull, bar_tempty, abort_flag, tmem_base, warp & 3, lane, cta_rank,
                                                      first_unit, unit_stride);
        else
            layer_epilogue<kPair, kOpProduct, kWide, kEpiWarps>(p, slots, 0, bar_in, bar_tfull, bar_tempty, abort_flag, tmem_base, warp - 2, warp & 3,
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
        // A's copies complete on the leader's barriers, the codes', of one producer alone, on each CTA's own
        if (warp == 0 && leader) drain_copies<kPair, 1>(unwind, bar_a, stages, kABytes, 0, lane, budget);
        if (warp == 2 + kEpiWarps) {
            const uint32_t n = min(issued, stages);
            for (uint32_t i = 1; i <= n; ++i) {
                const uint32_t idx = issued - i;
                const uint64_t t0 = globaltimer_ns();
                while (!mbar_try_wait(bar_raw + 8u * (idx % stages), (idx / stages) & 1u)) {
                    if (globaltimer_ns() - t0 > budget) break;
                }
            }
            __syncwarp();
        }
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

template <bool kPair, bool kAMajorM, bool kWide, bool kRaw>
cudaError_t product_init_t() {
    return cudaFuncSetAttribute(mip_product_kernel<kPair, kAMajorM, kWide, kRaw>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBudget);
}
template <bool kPair, bool kAMajorM>
cudaError_t product_init_form() {
    for (cudaError_t e : {product_init_t<kPair, kAMajorM, false, false>(), product_init_t<kPair, kAMajorM, true, false>(),
                          product_init_t<kPair, kAMajorM, true, true>()})
        if (e != cudaSuccess) return e;
    return cudaSuccess;
}
template <bool kPair, bool kAMajorM>
cudaError_t product_launch_form(const LayerParams& p, int raw, const cudaLaunchConfig_t& cfg) {
    if (raw) return cudaLaunchKernelEx(&cfg, mip_product_kernel<kPair, kAMajorM, true, true>, p);
    if (p.type == kF32) return cudaLaunchKernelEx(&cfg, mip_product_kernel<kPair, kAMajorM, true, false>, p);
    return cudaLaunchKernelEx(&cfg, mip_product_kernel<kPair, kAMajorM, false, false>, p);
}

}  // namespace

int product_stages() { return (kSmemBudget - kProductFixed) / static_cast<int>(kProductStage + kScaleBytes); }

cudaError_t product_init() {
    for (cudaError_t e : {product_init_form<false, false>(), product_init_form<false, true>(), product_init_form<true, false>(),
                          product_init_form<true, true>()})
        if (e != cudaSuccess) return e;
    return cudaSuccess;
}

cudaError_t launch_product(const LayerParams& p, int a_order, int pair, int raw, int grid, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(grid), 1, 1);
    cfg.blockDim = dim3(product_threads(raw || p.type == kF32), 1, 1);
    cfg.dynamicSmemBytes = std::max(kSmemFloor, static_cast<size_t>(p.stages) * (kProductStage + kScaleBytes) + kProductFixed);
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
    if (pair) return a_order ? product_launch_form<true, true>(p, raw, cfg) : product_launch_form<true, false>(p, raw, cfg);
    return a_order ? product_launch_form<false, true>(p, raw, cfg) : product_launch_form<false, false>(p, raw, cfg);
}

}  // namespace mip
