// Few-token form of the 8-bit floating-point product (M <= 32, tokens K-contiguous): every weight byte is read once, whatever M
// is, so the time is that of streaming the weights.
//
// As in the few-token kernel of the 8-bit layer, the operands change places: 128 columns of C (rows of the weights, or
// columns where they lie N-contiguous) are the accumulator's lanes, the tokens its columns, and K is split over the CTAs of a
// cluster.  The scales change from one block of 128 k to the next, so each block's products get columns of tensor
// memory of their own (as many blocks as 256 columns hold; then by turns), and four warps add them, a thread one column
// of C for all tokens, behind the product of the token's and the weights' scale.  The tokens' scales of all the CTA's blocks
// lie in shared memory.  At the end each thread sends its sums to the CTA that owns its columns; owners add them in the
// order of K and finish.
//
// What bounds it: the weights' bytes, and for small ones the launch, the first copies and the exchange.  Measured in a graph:
// 4096 x 4096 at one token 6.6 us, 14336 x 4096 at 16 11.4 us (5.2 TB/s of weights), 11008 x 4096 at 32, N-contiguous, 13.8 us.
//
// Weights under the constant-weights promise are fetched before the previous kernel in the stream has completed;
// without it the L2 is asked for them.  Every wait is bounded.
#include <algorithm>

#include "internal.h"
#include "layer_math.cuh"
#include "ptx.cuh"

namespace mip {

namespace {

constexpr int kFewThreads = 192, kFewSums = 128;             // copies, MMAs, and four warps that sum
constexpr int kFewColumns = 256;                             // of tensor memory
constexpr int kMaxFewStages = 6;
constexpr uint32_t kWeightTile = 128 * 128;
// No more than two CTAs of this kernel share an SM, nor one with a kernel that takes more than the other half of tensor memory:
// what two take, and one beside two of the 8-bit layer's few-token kernel, is there (see kSmemFloor).
constexpr size_t kFewSmemFloor = 100 * 1024, kFewSmemMost = 113 * 1024;
static_assert(3 * (kFewSmemFloor + kSmemReserved) > kSmemPerSm && kSmemFloor + kFewSmemFloor + 2 * kSmemReserved > kSmemPerSm, "CTAs on an SM");
static_assert(2 * (kFewSmemMost + kSmemReserved) <= kSmemPerSm, "two CTAs on an SM");

__device__ __forceinline__ float4 lds_float4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void mma_f8_one(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}

// kTokens: 16 or 32 columns of the accumulator.  kVec: a scale for each column of C, else for each 128.
template <int kTokens, bool kVec>
__global__ void __launch_bounds__(kFewThreads)
mip_f8_stream_kernel(const __grid_constant__ F8ProductParams p) {
    constexpr int kDepth = kFewColumns / kTokens;            // blocks of products in tensor memory
    const int split = p.split;
    const uint32_t rank = split > 1 ? cluster_ctarank() : 0u;
    const int n0 = static_cast<int>(blockIdx.x) / split * 128;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    const uint32_t pad = ((raw_addr + 1023u) & ~1023u) - raw_addr;
    uint8_t* smem = smem_raw + pad;
    const uint32_t smem_base = raw_addr + pad;
    constexpr uint32_t stage_bytes = kWeightTile + kTokens * 128u;
    // (exactly M token rows are copied; the accumulator's columns behind them add up whatever lies there and are never read)
    const uint32_t tx_bytes = kWeightTile + static_cast<uint32_t>(p.M) * 128u;
    // shared memory: [stages x (weights | tokens)] [sums received] [tokens' scales by block] [control block]
    const uint32_t xbuf = smem_base + p.stages * stage_bytes;
    constexpr uint32_t pitch = (kTokens + 4) * 4u;           // bytes per column of C: 16-byte reads of 8 of them hit all banks
    const uint32_t scales = xbuf + 128u * pitch;
    const uint32_t ctrl = scales + static_cast<uint32_t>(p.kb_share) * kTokens * 4u;
    const uint32_t bar_full = ctrl, bar_empty = bar_full + 8u * kMaxFewStages;
    const uint32_t bar_tfull = bar_empty + 8u * kMaxFewStages, bar_tempty = bar_tfull + 8u * kDepth, bar_drain = bar_tempty + 8u * kDepth;
    uint8_t* ctrl_ptr = smem + (bar_drain + 8u - smem_base);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ctrl_ptr);
    volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(tmem_slot + 1);

    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(bar_full + 8u * s, 1);
            mbar_init(bar_empty + 8u * s, 1);
        }
        for (int s = 0; s < kDepth; ++s) {
            mbar_init(bar_tfull + 8u * s, 1);
            mbar_init(bar_tempty + 8u * s, 4);
        }
        mbar_init(bar_drain, 1);
        *abort_flag = 0;
        fence_mbar_init();
        tma_prefetch_desc(&p.tmap_a);
        tma_prefetch_desc(&p.tmap_b0);
    }
    if (warp == 1) {
        tmem_alloc<1>(smem_u32(tmem_slot), kFewColumns);
        tmem_relinquish<1>();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (split > 1) cluster_arrive();       // "this CTA has started": awaited before anything is sent to it
    const uint32_t tmem_base = *tmem_slot;
    const uint64_t budget = p.wait_budget_ns;
    const int kb0 = static_cast<int>(rank) * p.kb_share;
    const int n_kb = max(0, min(p.k_blocks, kb0 + p.kb_share) - kb0);
    uint32_t issued = 0;

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer
        const auto x_of = [&](int kb) { return p.b_mn ? n0 : kb * 128; };
        const auto y_of = [&](int kb) { return p.b_mn ? kb * 128 : n0; };
        const int early = min(n_kb, p.stages);
        if (elect_one()) {
            for (int i = 0; i < early; ++i) {
                if (p.b_constant) {
                    mbar_arrive_expect_tx(bar_full + 8u * i, tx_bytes);
                    tma_load_2d(smem_base + i * stage_bytes, &p.tmap_b0, bar_full + 8u * i, x_of(kb0 + i), y_of(kb0 + i));
                } else {
                    tma_prefetch_l2_2d(&p.tmap_b0, x_of(kb0 + i), y_of(kb0 + i));
                }
            }
        }
        __syncwarp();
        pdl_wait();
        pdl_launch_dependents();      // (only now: one kernel at a time waits for another)
        uint32_t s = 0, phase = 0;
        for (int i = 0; i < n_kb; ++i) {
            if (i >= p.stages && !mbar_wait_warp(bar_empty + 8u * s, phase ^ 1u, abort_flag, budget)) break;
            if (elect_one()) {
                const uint32_t dst = smem_base + s * stage_bytes, bar = bar_full + 8u * s;
                if (!(p.b_constant && i < early)) {
                    mbar_arrive_expect_tx(bar, tx_bytes);
                    tma_load_2d(dst, &p.tmap_b0, bar, x_of(kb0 + i), y_of(kb0 + i));
                }
                tma_load_2d(dst + kWeightTile, &p.tmap_a, bar, (kb0 + i) * 128, 0);
            }
            ++issued;
            if (++s == static_cast<uint32_t>(p.stages)) { s = 0; phase ^= 1u; }
        }
    } else {
        pdl_wait();
        pdl_launch_dependents();
    }
    __syncwarp();
    if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer
        uint32_t s = 0, phase = 0, acc = 0, acc_phase = 0;
        const uint64_t a_step = p.b_mn ? 256ull : 2ull;
        for (int i = 0; i < n_kb; ++i) {
            if (i >= kDepth && !mbar_wait_warp(bar_tempty + 8u * acc, acc_phase ^ 1u, abort_flag, budget)) break;
            if (!mbar_wait_warp(bar_full + 8u * s, phase, abort_flag, budget)) break;
            tc_fence_after();
            const uint32_t addr = smem_base + s * stage_bytes;
            const uint64_t a_desc = p.b_mn ? make_mnmajor_desc(addr, kWeightTile) : make_kmajor_desc(addr, 128);
            const uint64_t b_desc = make_kmajor_desc(addr + kWeightTile, 128);
            if (elect_one()) {
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k)
                    mma_f8_one(tmem_base + acc * kTokens, a_desc + a_step * k, b_desc + 2ull * k, p.idesc, k > 0 ? 1u : 0u);
                if (!(p.debug_flags & 1)) mma_commit(bar_tfull + 8u * acc);      // (test hook, bit 0: the signal is withheld)
                mma_commit(bar_empty + 8u * s);
            }
            __syncwarp();
            if (++s == static_cast<uint32_t>(p.stages)) { s = 0; phase ^= 1u; }
            if (++acc == kDepth) { acc = 0; acc_phase ^= 1u; }
        }
    }
    __syncwarp();

    const int me = static_cast<int>(threadIdx.x) - 64;         // of the summing threads
    const int q = warp & 3, lane_col = q * 32 + lane;          // the accumulator's lane
    uint64_t sum[kTokens / 2];
    bool ok = true;
    if (warp >= 2) {
        // ------------------------------------------------------------ sums
        // the tokens' scales of this CTA's blocks (0 behind the last token), block by block
        for (int i = me; i < n_kb * kTokens; i += kFewSums) {
            const int kb = kb0 + i / kTokens, t = i % kTokens;
            const float s = t < p.M ? (p.sa ? __ldg(p.sa + static_cast<long long>(kb) * p.lds_a + t) : 1.0f) : 0.0f;
            asm volatile("st.shared.f32 [%0], %1;" ::"r"(scales + i * 4u), "f"(s) : "memory");
        }
        const float* pb = nullptr;
        if (p.sb) pb = p.sb + static_cast<long long>(kb0) * p.sb_k + (kVec ? min(n0 + lane_col, p.N - 1) : (n0 >> 7) * p.sb_n);
        float next = pb && n_kb > 0 ? __ldg(pb) : 1.0f;
        asm volatile("bar.sync 1, 128;" ::: "memory");
#pragma unroll
        for (int j = 0; j < kTokens / 2; ++j) sum[j] = 0ull;
        uint32_t acc = 0, acc_phase = 0;
        for (int i = 0; i < n_kb; ++i) {
            const float sb = next;
            if (pb && i + 1 < n_kb) next = __ldg(pb += p.sb_k);
            if (!mbar_wait_warp(bar_tfull + 8u * acc, acc_phase, abort_flag, budget)) { ok = false; break; }
            tc_fence_after();
            const uint32_t t_at = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + acc * kTokens;
            const uint32_t s_at = scales + static_cast<uint32_t>(i) * kTokens * 4u;
            const uint64_t sb2 = pack_f2(sb, sb);
#pragma unroll
            for (int c = 0; c < kTokens; c += 16) {
                uint32_t v[16];
                tmem_ld_32x16(t_at + c, v);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 16; j += 4) {
                    const float4 s = lds_float4(s_at + static_cast<uint32_t>(c + j) * 4u);
                    uint64_t* to = &sum[(c + j) / 2];
                    to[0] = fma_f2(pack_f2(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), mul_f2(pack_f2(s.x, s.y), sb2), to[0]);
                    to[1] = fma_f2(pack_f2(__uint_as_float(v[j + 2]), __uint_as_float(v[j + 3])), mul_f2(pack_f2(s.z, s.w), sb2), to[1]);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_tempty + 8u * acc);
            if (++acc == kDepth) { acc = 0; acc_phase ^= 1u; }
        }
    }
    __syncwarp();

    // ---------------------------------------------------------------- sums to their owners
    const int cols_own = 128 / split;                          // columns of C this CTA finishes
    if (split > 1) cluster_wait();
    if (warp >= 2 && ok) {
        const int owner = lane_col / cols_own, local = lane_col - owner * cols_own;
        const uint32_t mine = xbuf + static_cast<uint32_t>(static_cast<int>(rank) * cols_own + local) * pitch;
        const uint32_t dst = split > 1 ? mapa_u32(mine, static_cast<uint32_t>(owner)) : mine;
#pragma unroll
        for (int j = 0; j < kTokens; j += 4) {
            float a, b, c, d;
            unpack_f2(sum[j / 2], a, b);
            unpack_f2(sum[j / 2 + 1], c, d);
            asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(dst + j * 4u), "f"(a), "f"(b), "f"(c), "f"(d) : "memory");
        }
    }
    tc_fence_before();
    __syncwarp();
    if (split > 1) {
        cluster_arrive();
        cluster_wait();
    }
    __syncthreads();

    // ---------------------------------------------------------------- owners finish their columns, four tokens at a time
    if (*abort_flag == 0) {
        if (warp >= 2) {
            const int t_first = me / cols_own, t_step = kFewSums / cols_own, lc = me - t_first * cols_own;
            const int n = n0 + static_cast<int>(rank) * cols_own + lc;
            if (n < p.N) {
                const float bias = p.bias ? __ldg(p.bias + n) : 0.0f;
                const int groups = (p.M + 3) >> 2;
                for (int t4 = t_first; t4 < groups; t4 += t_step) {
                    float r[4], y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int j = 0; j < 4; ++j) r[j] = p.R && 4 * t4 + j < p.M ? load_element(p.R, (4ll * t4 + j) * p.ldr + n, p.type) : 0.0f;
                    for (int sl = 0; sl < split; ++sl) {
                        const float4 s = lds_float4(xbuf + static_cast<uint32_t>(sl * cols_own + lc) * pitch + static_cast<uint32_t>(t4) * 16u);
                        y[0] += s.x; y[1] += s.y; y[2] += s.z; y[3] += s.w;
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (4 * t4 + j < p.M) store_element(p.C, (4ll * t4 + j) * p.ldc + n, p.type, y[j] + bias + r[j]);
                }
            }
        }
    } else {
        // unwinding: what was asked for must have landed, and MMAs must have retired, before the memory is given back
        if (warp == 0) {
            // (the first `stages` copies are always all asked for: nothing stops the producer before)
            const uint32_t stages = p.stages, first = issued > stages ? issued - stages : 0u;
            for (uint32_t i = first; i < issued; ++i) {
                const uint64_t t0 = globaltimer_ns();
                while (!mbar_try_wait(bar_full + 8u * (i % p.stages), (i / p.stages) & 1u)) {
                    if (globaltimer_ns() - t0 > budget) break;
                }
            }
        }
        if (warp == 1) {
            if (elect_one()) mma_commit(bar_drain);
            __syncwarp();
            const uint64_t t0 = globaltimer_ns();
            while (!mbar_try_wait(bar_drain, 0)) {
                if (globaltimer_ns() - t0 > budget) break;
            }
        }
        if (threadIdx.x == 0) atomicOr(p.status, 1u);
    }
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc<1>(tmem_base, kFewColumns);
    }
}

size_t few_smem(int tokens, int kb_share, int stages) {
    const int depth = kFewColumns / tokens;
    return static_cast<size_t>(stages) * (kWeightTile + tokens * 128) + 128 * (tokens + 4) * 4 + static_cast<size_t>(kb_share) * tokens * 4 +
           16 * kMaxFewStages + 16 * depth + 32 + 1024;
}
template <int kTokens>
cudaError_t few_init() {
    for (cudaError_t e : {cudaFuncSetAttribute(mip_f8_stream_kernel<kTokens, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBudget),
                          cudaFuncSetAttribute(mip_f8_stream_kernel<kTokens, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBudget)})
        if (e != cudaSuccess) return e;
    return cudaSuccess;
}
template <int kTokens>
cudaError_t few_launch(const F8ProductParams& p, bool vec, const cudaLaunchConfig_t& cfg) {
    return vec ? cudaLaunchKernelEx(&cfg, mip_f8_stream_kernel<kTokens, true>, p) : cudaLaunchKernelEx(&cfg, mip_f8_stream_kernel<kTokens, false>, p);
}

}  // namespace

// Stages that leave room for a second CTA on the SM; 0: not even two fit (a long share of K for many tokens).
int f8_stream_stages(int tokens, int kb_share) {
    int stages = std::min(kMaxFewStages, std::max(2, kb_share));
    while (stages >= 2 && few_smem(tokens, kb_share, stages) > kFewSmemMost) --stages;
    return stages >= 2 ? stages : 0;
}

cudaError_t f8_stream_init() {
    for (cudaError_t e : {few_init<16>(), few_init<32>()})
        if (e != cudaSuccess) return e;
    return cudaSuccess;
}

cudaError_t launch_f8_stream(const F8ProductParams& p, bool vec, int grid, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(grid), 1, 1);
    cfg.blockDim = dim3(kFewThreads, 1, 1);
    cfg.dynamicSmemBytes = std::max(kFewSmemFloor, few_smem(p.block_n, p.kb_share, p.stages));
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_allowed();
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(p.split);
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.split > 1 ? 2 : 1;
    return p.block_n == 16 ? few_launch<16>(p, vec, cfg) : few_launch<32>(p, vec, cfg);
}

}  // namespace mip
