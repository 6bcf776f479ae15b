// Few-token form of the 8-bit layer's operators (M <= 64): every weight byte is read once, whatever M is, so the time
// is that of streaming the weights.
//
// The operands change places: 128 weight rows lie on the accumulator's lanes (gated forms: 64 rows of each
// projection), the tokens are its columns (16, 32, 48 or 64), so tcgen05.mma.kind::i8 wastes nothing on absent tokens
// but a few columns, and a CTA is four warps that hardly issue anything: warp 0 asks the TMA for 16 KB weight tiles
// (128-byte swizzle) and the tokens' slice beside them, warp 1 issues MMAs.
//
// K is split over the CTAs of a cluster (1, 2, 4 or 8), so that matrices of a few thousand rows fill the machine too;
// two CTAs share an SM when their stages fit, one streams while the other finishes.  At the end each thread (= weight
// row) sends its partial sums to the CTA that owns its output columns, through distributed shared memory; integer
// sums do not depend on the order.  Owners add the partials and finish 4 tokens of a column per thread: neighbouring
// lanes hold neighbouring columns, so rows of C are written in whole segments.
//
// Measured: gated 11008 x 4096 at 16 tokens 20.5 us a call (4.4 TB/s of weights; what is not streaming is the launch, the
// first copies' latency and the exchange, 5 to 6 us), linear 4096 x 4096 at one token 6.7 us.
//
// Weights under the constant-weights promise are fetched before the previous kernel in the stream has completed;
// without it the L2 is asked for them (a prefetch brings nothing into the SM).  Every wait is bounded.
#include "internal.h"
#include "layer_math.cuh"
#include "ptx.cuh"

namespace mip {

namespace {

constexpr int kStreamThreads = 128;
constexpr uint32_t kWeightTile = kStreamRows * 128;

__device__ __forceinline__ int4 lds_int4(uint32_t addr) {
    int4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}

template <int kOp, bool kWide>
__global__ void __launch_bounds__(kStreamThreads)
mip_layer_stream_kernel(const __grid_constant__ LayerParams p) {
    constexpr bool kGatedForm = kOp != kOpLinear;
    const int split = p.split;
    const uint32_t rank = split > 1 ? cluster_ctarank() : 0u;
    const int tile = static_cast<int>(blockIdx.x) / split;
    const int n0 = tile * p.out_n;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    const uint32_t pad = ((raw_addr + 1023u) & ~1023u) - raw_addr;
    uint8_t* smem = smem_raw + pad;
    const uint32_t smem_base = raw_addr + pad;
    const uint32_t stage_bytes = kWeightTile + static_cast<uint32_t>(p.block_n) * 128u;
    // (exactly M token rows are copied: rows a TMA copy has to fill with zeros cost it several times those it reads.
    // The accumulator's columns behind them add up whatever lies there and are never read.)
    const uint32_t tx_bytes = kWeightTile + static_cast<uint32_t>(p.M) * 128u;
    // shared memory: [stages x (weights | tokens)] [partial sums received] [control block]
    const uint32_t xbuf = smem_base + p.stages * stage_bytes;
    const uint32_t pitch = static_cast<uint32_t>(p.block_n + 4) * 4u;      // bytes per row: 16-byte reads of 8 rows hit all banks
    const uint32_t ctrl = xbuf + kStreamRows * pitch;
    const uint32_t bar_full = ctrl, bar_empty = ctrl + 8u * kMaxStages, bar_done = ctrl + 16u * kMaxStages, bar_drain = bar_done + 8u;
    uint8_t* ctrl_ptr = smem + (ctrl - smem_base);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ctrl_ptr + 16 * kMaxStages + 16);
    volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(tmem_slot + 1);

    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(bar_full + 8u * s, 1);
            mbar_init(bar_empty + 8u * s, 1);
        }
        mbar_init(bar_done, 1);
        mbar_init(bar_drain, 1);
        *abort_flag = 0;
        fence_mbar_init();
        tma_prefetch_desc(&p.tmap_a);
        tma_prefetch_desc(&p.tmap_b0);
        if (kGatedForm) tma_prefetch_desc(&p.tmap_b1);
    }
    if (warp == 1) {
        tmem_alloc<1>(smem_u32(tmem_slot), p.tmem_cols);
        tmem_relinquish<1>();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (split > 1) cluster_arrive();       // "this CTA has started": awaited before anything is sent to it
    const uint32_t tmem_base = *tmem_slot;
    const uint64_t budget = p.wait_budget_ns;
    const int share = (p.k_blocks + split - 1) / split;
    const int kb0 = static_cast<int>(rank) * share;
    const int n_kb = max(0, min(p.k_blocks, kb0 + share) - kb0);
    uint32_t issued = 0;

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer
        const auto load_weights = [&](uint32_t dst, uint32_t bar, int kb) {
            tma_load_2d(dst, &p.tmap_b0, bar, kb * 128, n0);
            if (kGatedForm) tma_load_2d(dst + kWeightTile / 2, &p.tmap_b1, bar, kb * 128, n0);
        };
        const int early = min(n_kb, p.stages);
        if (elect_one()) {
            for (int i = 0; i < early; ++i) {
                if (p.b_constant) {
                    mbar_arrive_expect_tx(bar_full + 8u * i, tx_bytes);
                    load_weights(smem_base + i * stage_bytes, bar_full + 8u * i, kb0 + i);
                } else {
                    tma_prefetch_l2_2d(&p.tmap_b0, (kb0 + i) * 128, n0);
                    if (kGatedForm) tma_prefetch_l2_2d(&p.tmap_b1, (kb0 + i) * 128, n0);
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
                    load_weights(dst, bar, kb0 + i);
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
    if (warp == 1 && n_kb > 0) {
        // ------------------------------------------------------------ MMA issuer
        uint32_t s = 0, phase = 0;
        bool ok = true;
        for (int i = 0; i < n_kb; ++i) {
            if (!mbar_wait_warp(bar_full + 8u * s, phase, abort_flag, budget)) { ok = false; break; }
            tc_fence_after();
            const uint32_t addr = smem_base + s * stage_bytes;
            const uint64_t a_desc = make_kmajor_desc(addr, 128), b_desc = make_kmajor_desc(addr + kWeightTile, 128);
            if (elect_one()) {
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k)
                    mma_i8<1>(tmem_base, a_desc + 2ull * k, b_desc + 2ull * k, p.idesc, (i > 0 || k > 0) ? 1u : 0u);
                mma_commit(bar_empty + 8u * s);
            }
            if (++s == static_cast<uint32_t>(p.stages)) { s = 0; phase ^= 1u; }
        }
        if (ok && !(p.debug_flags & 1) && elect_one()) mma_commit(bar_done);   // (test hook, bit 0: the signal is withheld)
    }
    __syncwarp();

    // An owner finishes items of 4 tokens of one column; a thread's items all lie in the same column.  What an item
    // needs besides its sums is asked for in batches of kBatch items, all loads together and ahead of the stores they
    // could alias, the first batch before the sums are ready: a thread waits for memory once per 16 / split tokens x
    // columns of its own instead of once per item (16 tokens, 4096 x 4096, split 1: 16.8 -> 11 us).
    const int cols_own = p.out_n / split;                  // output columns this CTA finishes (divides 128)
    const int rows_own = kStreamRows / split;              // weight rows behind them
    const int groups = (p.M + 3) >> 2;                     // of 4 tokens
    const int t_first = static_cast<int>(threadIdx.x) / cols_own, t_step = kStreamThreads / cols_own;
    const int lc = static_cast<int>(threadIdx.x) - t_first * cols_own;
    const int n = n0 + static_cast<int>(rank) * cols_own + lc;
    constexpr int kBatch = 4;
    float b0 = 1.0f, b1 = kGatedForm ? 1.0f : 0.0f;        // scales of the column; b1 is the bias of a linear layer
    // (the elements are kept as they come: converting one where it is loaded would wait for it there)
    using Raw = std::conditional_t<kWide, uint32_t, uint16_t>;
    float as[kBatch][4];
    Raw r[kBatch][4];
    const bool f16 = p.type == kF16;
    const auto value_of = [&](Raw x) { return kWide ? __uint_as_float(x) : (f16 ? __half2float(__ushort_as_half(x)) : __uint_as_float(static_cast<uint32_t>(x) << 16)); };
    const auto put = [&](void* base, long long i, float v) {
        if (kWide) static_cast<float*>(base)[i] = v;
        else if (f16) static_cast<__half*>(base)[i] = __float2half_rn(v);
        else static_cast<__nv_bfloat16*>(base)[i] = __float2bfloat16_rn(v);
    };
    const auto fetch = [&](int t) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const long long tok = 4ll * (t + i * t_step) + q;
                const bool in = n < p.N && tok < p.M;
                as[i][q] = in ? scale_at(p.a_scale, tok) : 0.0f;
                r[i][q] = (kOp != kOpGated && in && p.R) ? static_cast<const Raw*>(p.R)[tok * p.ldr + n] : Raw(0);
            }
        }
    };
    if (n < p.N) {
        b0 = scale_at(p.b0_scale, n);
        if (kGatedForm) b1 = scale_at(p.b1_scale, n);
        else if (p.bias) b1 = __ldg(p.bias + n);
    }
    fetch(t_first);

    // ---------------------------------------------------------------- partial sums to their owners
    bool ok = n_kb == 0 || mbar_wait(bar_done, 0u, abort_flag, budget);
    ok = __all_sync(~0u, ok);
    tc_fence_after();
    if (split > 1) cluster_wait();
    if (ok) {
        const int row = warp * 32 + lane;
        const int col = kGatedForm ? row & 63 : row;
        const int owner = col / cols_own;
        const int local = col - owner * cols_own + (kGatedForm && row >= 64 ? cols_own : 0);
        const uint32_t mine = xbuf + static_cast<uint32_t>(static_cast<int>(rank) * rows_own + local) * pitch;
        const uint32_t dst = split > 1 ? mapa_u32(mine, static_cast<uint32_t>(owner)) : mine;
        for (int c = 0; c < p.block_n; c += 16) {
            uint32_t v[16];
            if (n_kb > 0) {
                tmem_ld_32x16(tmem_base + (static_cast<uint32_t>(warp * 32) << 16) + c, v);
                tmem_ld_wait();
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] = 0u;
            }
#pragma unroll
            for (int j = 0; j < 16; j += 4)
                asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};"
                             ::"r"(dst + static_cast<uint32_t>(c + j) * 4u), "r"(v[j]), "r"(v[j + 1]), "r"(v[j + 2]), "r"(v[j + 3]) : "memory");
        }
    }
    tc_fence_before();
    if (split > 1) {
        cluster_arrive();
        cluster_wait();
    }
    __syncthreads();

    // ---------------------------------------------------------------- owners finish their columns
    if (*abort_flag == 0) {
        for (int t = t_first; t < groups && n < p.N; t += kBatch * t_step) {
            if (t != t_first) fetch(t);
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const int t4 = t + i * t_step;
                if (t4 >= groups) break;
                int s0[4] = {0, 0, 0, 0}, s1[4] = {0, 0, 0, 0};
                for (int sl = 0; sl < split; ++sl) {
                    const uint32_t at = xbuf + static_cast<uint32_t>(sl * rows_own + lc) * pitch + static_cast<uint32_t>(t4) * 16u;
                    const int4 a = lds_int4(at);
                    s0[0] += a.x; s0[1] += a.y; s0[2] += a.z; s0[3] += a.w;
                    if (kGatedForm) {
                        const int4 b = lds_int4(at + static_cast<uint32_t>(cols_own) * pitch);
                        s1[0] += b.x; s1[1] += b.y; s1[2] += b.z; s1[3] += b.w;
                    }
                }
                float y[4], y2[4];
                with_activation(p.act, [&](auto act) {
                    constexpr int kAct = decltype(act)::value;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float z0 = __int2float_rn(s0[q]) * as[i][q] * b0;
                        if (kOp == kOpLinear) {
                            y[q] = activation<kAct>(z0 + b1) + value_of(r[i][q]);
                        } else {
                            const float z1 = __int2float_rn(s1[q]) * as[i][q] * b1;
                            if (kOp == kOpGated) {
                                y[q] = activation<kAct>(z0) * z1;
                            } else {
                                float value, slope;
                                activation_slope<kAct>(z0, value, slope);
                                y[q] = value_of(r[i][q]) * z1 * slope;
                                y2[q] = value_of(r[i][q]) * value;
                            }
                        }
                    }
                });
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const long long tok = 4ll * t4 + q;
                    if (tok >= p.M) break;
                    put(p.C, tok * p.ldc + n, y[q]);
                    if (kOp == kOpGatedGrad) put(p.C2, tok * p.ldc2 + n, y2[q]);
                }
            }
        }
    } else {
        // unwinding: what was asked for must have landed, and MMAs must have retired, before the memory is given back
        if (warp == 0) {
            const uint32_t n = min(issued, static_cast<uint32_t>(p.stages));
            for (uint32_t i = 1; i <= n; ++i) {
                const uint32_t idx = issued - i;
                const uint64_t t0 = globaltimer_ns();
                while (!mbar_try_wait(bar_full + 8u * (idx % p.stages), (idx / p.stages) & 1u)) {
                    if (globaltimer_ns() - t0 > budget) break;
                }
            }
        }
        if (warp == 1) {
            if (elect_one()) mma_commit(bar_drain);
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
        tmem_dealloc<1>(tmem_base, p.tmem_cols);
    }
}

template <int kOp>
cudaError_t stream_init_t() {
    const cudaError_t e = cudaFuncSetAttribute(mip_layer_stream_kernel<kOp, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBudget);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(mip_layer_stream_kernel<kOp, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBudget);
}
template <int kOp>
cudaError_t stream_launch_t(const LayerParams& p, const cudaLaunchConfig_t& cfg) {
    return p.type == kF32 ? cudaLaunchKernelEx(&cfg, mip_layer_stream_kernel<kOp, true>, p)
                          : cudaLaunchKernelEx(&cfg, mip_layer_stream_kernel<kOp, false>, p);
}

}  // namespace

static constexpr int stream_smem_of(int tokens, int stages) {
    return stages * (static_cast<int>(kWeightTile) + tokens * 128) + kStreamRows * (tokens + 4) * 4 + 256 + 1024;
}
static_assert(kSmemFloor + stream_smem_of(16, 2) + 2 * kSmemReserved > kSmemPerSm, "a CTA beside one of a dense kernel's");
int stream_smem(int tokens, int stages) { return stream_smem_of(tokens, stages); }

cudaError_t stream_init() {
    for (cudaError_t e : {stream_init_t<kOpLinear>(), stream_init_t<kOpGated>(), stream_init_t<kOpGatedGrad>()})
        if (e != cudaSuccess) return e;
    return cudaSuccess;
}

cudaError_t launch_layer_stream(const LayerParams& p, int op, int grid, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(grid), 1, 1);
    cfg.blockDim = dim3(kStreamThreads, 1, 1);
    cfg.dynamicSmemBytes = stream_smem(p.block_n, p.stages);
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
    if (op == kOpLinear) return stream_launch_t<kOpLinear>(p, cfg);
    return op == kOpGated ? stream_launch_t<kOpGated>(p, cfg) : stream_launch_t<kOpGatedGrad>(p, cfg);
}

}  // namespace mip
