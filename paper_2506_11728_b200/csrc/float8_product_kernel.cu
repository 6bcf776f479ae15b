// C = sum over blocks of 128 k of  sa[kb][i] sb[kb][j] (A B)_kb  + bias + residual, A and B 8-bit floating point: the products of a
// layer and of its backward pass (operands K- or M/N-contiguous, as they lie).
//
// The scales change along the summed axis, so a block's products are summed by the tensor core on their own
// (tcgen05.mma.kind::f8f6f4, binary32 in tensor memory) and added to the tile's sums, which live in
// registers, behind their two scales.  Eight warps do that: a thread has one row and 128 (CTA pairs, 256 x 256 tiles) or 64
// (single CTAs, 128 x 128) columns.  A block's products wait for a signal, are read, and free their buffer by another
// signal: some 300 clocks of latency beside the reading.  A pair's tile is therefore computed by halves of 128 columns, each
// with two buffers in tensor memory and four warps of its own: a buffer has the time of a whole block and a half for that.  With squares of 128 x 128 on B's side both scales are one number per thread and block: one packed
// multiply-add for two elements.  With a scale for each column they come through shared memory, and it is one multiplication
// more.
//
// Outputs go through swizzled slots in shared memory as in the layer's kernels (layer_epilogue.cuh).
//
// What bounds it.  Squares: 8192 x 4096 x 4096 bf16 131 to 136 us (2060 TFLOP/s); without a tile's outputs, which nothing hides as the
// sums' registers are taken until then, 111, without the sums 92.  16384 x 4096 x 11008: 717 us after a pause, 773 in a row of calls
// (power).  A scale for each column: two packed operations for two elements make a block 512 clocks of the summing warps' pipes at
// least, 1200 with their waits (11008 x 4096 x 8192 float32, added to: 568 us).  Few blocks of K: a tile's
// outputs (16384 x 4096 x 64 bf16 70 us, float32 57, their bytes 21 and 41).
//
// Every wait is bounded, with the unwinding of the dense layer kernel.
#include <algorithm>

#include "layer_epilogue.cuh"
#include "unwind.cuh"

namespace mip {

namespace {

constexpr int kSumWarps = 8;
constexpr int kF8Threads = 32 * (4 + kSumWarps);
constexpr int kMaxF8Stages = 8;
constexpr int slot_buffers(bool wide) { return wide ? 2 : 3; }           // per summing warp
constexpr int all_slot_bytes(bool wide) { return kSumWarps * slot_buffers(wide) * slot_bytes(wide); }
// Scales of a k-block: of the tile's 128 rows times those of its squares (each half's two), or of the rows and of the columns.
// As many blocks as there are buffers of products for a half, twice: a block's place is written when the products of one
// `depth` blocks before are ready, which says that the buffers of another `depth` blocks before have been given back; nothing
// reads a block's scales behind that.
constexpr int scale_bytes(bool pair, bool vec) { return vec ? (pair ? 1536 : 1024) : (pair ? 1024 : 512); }
constexpr int scale_places(bool pair) { return pair ? 4 : 8; }
constexpr int kBiasBytes = kSumWarps * 128;                              // 32 columns for each summing warp
// Where the last tiles lie, from the scales' warp to the summing warps, which look behind a tile's last block.  A tile's position is
// written before any wait for the tile: with the wait for the block in front of it the buffers up to 2 * depth blocks before that one
// had been given back, and where a tile is one block, the tile behind those is still to be looked up.
constexpr int tile_places(bool pair) { return pair ? 8 : 16; }
constexpr int tile_bytes(bool pair) { return 16 * tile_places(pair); }
// Registers per thread: the sums take 128 of those of a pair's summing warps.  The block is launched with kLaunchRegs a thread; the
// four other warps give theirs up (checked against the compiled kernel before its first launch).
constexpr int kLaunchRegs = 168, kFewRegs = 120, kManyRegs = 192;
static_assert(4 * kFewRegs + kSumWarps * kManyRegs <= (4 + kSumWarps) * kLaunchRegs, "register split");

template <int kRegs>
__device__ __forceinline__ void regs_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegs)); }
template <int kRegs>
__device__ __forceinline__ void regs_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegs)); }

template <int kCtaGroup>
__device__ __forceinline__ void mma_f8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    if (kCtaGroup == 1)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
            ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
            ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}

// Signals this barrier, in both CTAs of a pair, when all MMAs issued so far are done.
template <bool kPair>
__device__ __forceinline__ void commit_all(uint32_t bar) {
    if (kPair)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"(static_cast<uint16_t>(3)) : "memory");
    else
        mma_commit(bar);
}
__device__ __forceinline__ void tmem_ld_wait_for_16(uint32_t (&v)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
          "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]) :: "memory");
}
// Arrives on a barrier of the cluster (see mbar_arrive_remote_fenced).
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cta.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool wait_fast(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, uint64_t budget) {
    if (__all_sync(~0u, mbar_try_wait(bar, parity))) return true;
    return mbar_wait_warp(bar, parity, abort_flag, budget);
}
__device__ __forceinline__ uint64_t words_f2(uint32_t a, uint32_t b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(a), "r"(b));
    return r;
}

// kPair: 256 x 256 tiles of CTA pairs, else 128 x 128.  kVec: a scale for each column of B, else for each 128.
// kWide: 32-bit outputs.  kRaw: the sums go to planes of partial sums.
template <bool kPair, bool kVec, bool kWide, bool kRaw>
__global__ void __launch_bounds__(kF8Threads, 1)
mip_f8_product_kernel(const __grid_constant__ F8ProductParams p) {
    constexpr int kCtas = kPair ? 2 : 1;
    // The tile's columns by halves (pair): 64 of each CTA's B tile, so that a half's 128 columns are two runs of 64.
    constexpr int kHalves = kPair ? 2 : 1;
    constexpr int kN = 128;                              // accumulator columns of an instruction
    constexpr int kDepth = 4 / kHalves;                  // blocks of products in tensor memory, for each half
    constexpr int kCols = kPair ? 128 : 64;              // columns per thread
    constexpr int kRowsPerTile = kCtas * kBlockM;
    constexpr uint32_t a_bytes = kBlockM * 128, b_bytes = 128 * 128, stage_bytes = a_bytes + b_bytes;
    constexpr int kSlot = slot_bytes(kWide), kSlotBuffers = slot_buffers(kWide);
    const uint32_t cta_rank = kPair ? cluster_ctarank() : 0u;
    const bool leader = cta_rank == 0;
    const int first_unit = kPair ? static_cast<int>(blockIdx.x >> 1) : static_cast<int>(blockIdx.x);
    const int unit_stride = kPair ? static_cast<int>(gridDim.x >> 1) : static_cast<int>(gridDim.x);
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    const uint32_t pad = ((raw_addr + 1023u) & ~1023u) - raw_addr;
    uint8_t* smem = smem_raw + pad;
    const uint32_t smem_base = raw_addr + pad;
    // shared memory: [stages x (A | B)] [slots of the summing warps] [scales] [bias] [control block] [tile positions]
    const uint32_t slots = smem_base + p.stages * stage_bytes;
    const uint32_t scales = slots + (kRaw ? 0u : all_slot_bytes(kWide));
    constexpr uint32_t kScaleBytes = scale_bytes(kPair, kVec), kPlaces = scale_places(kPair);
    const uint32_t bias_at = scales + kPlaces * kScaleBytes;
    const uint32_t ctrl = bias_at + kBiasBytes;
    const uint32_t tile_at = ctrl + kCtrlBytes;          // m0, n0 and first plane row
    constexpr uint32_t kTilePlaces = tile_places(kPair);
    static_assert(kTilePlaces >= 2 * kDepth + 2 && (kTilePlaces & (kTilePlaces - 1)) == 0, "tile positions");
    const uint32_t bar_full = ctrl, bar_empty = ctrl + 8u * kMaxF8Stages;
    const uint32_t bar_tfull = ctrl + 16u * kMaxF8Stages, bar_tempty = bar_tfull + 32u, bar_drain = bar_tempty + 32u;
    const uint32_t bar_in = bar_drain + 8u;              // kSumWarps x kSlotBuffers: a slot's tile has arrived
    uint8_t* ctrl_ptr = smem + (bar_in + 8u * kSumWarps * kSlotBuffers - smem_base);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ctrl_ptr);
    volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(tmem_slot + 1);
    const UnwindWords unwind = {bar_in + 8u * kSumWarps * kSlotBuffers + 8u};
    static_assert(16 * kMaxF8Stages + 72 + 8 * kSumWarps * slot_buffers(false) + 8 + UnwindWords::kBytes <= kCtrlBytes, "control block");

    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(bar_full + 8u * s, 2);                       // two producers
            mbar_init(bar_empty + 8u * s, 1);
        }
        for (int a = 0; a < 4; ++a) {
            mbar_init(bar_tfull + 8u * a, 2);       // the products, and the scales
            mbar_init(bar_tempty + 8u * a, kSumWarps);      // warps that read it: four of each CTA's, or all eight
        }
        mbar_init(bar_drain, 1);
        for (int i = 0; i < kSumWarps * kSlotBuffers; ++i) mbar_init(bar_in + 8u * i, 1);
        *abort_flag = 0;
        fence_mbar_init();
        tma_prefetch_desc(&p.tmap_a);
        tma_prefetch_desc(&p.tmap_b0);
        if (p.r_tma) tma_prefetch_desc(&p.tmap_r);
        if (p.c_tma) tma_prefetch_desc(&p.tmap_c);
    }
    if (kPair) {   // the peer runs (see tmem_alloc), and its barriers are initialised before anything remote touches them
        __syncwarp();
        cluster_arrive();
        cluster_wait();
    }
    if (warp == 1) {
        tmem_alloc<kCtas>(smem_u32(tmem_slot), 512);
        tmem_relinquish<kCtas>();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait();          // from here on global memory is touched
    pdl_launch_dependents();      // (only now: one kernel at a time waits for another)
    const uint32_t tmem_base = *tmem_slot;
    const int total_units = layer_units(p);
    const uint64_t budget = p.wait_budget_ns;
    // k-blocks of a unit (without a split, all: no division)
    const auto unit_blocks = [&](int unit) {
        if (p.split <= 1) return p.k_blocks;
        const int kb0 = unit % p.split * p.kb_share;
        return min(p.k_blocks, kb0 + p.kb_share) - kb0;
    };

    if (warp < 4) {
        if constexpr (kPair) regs_dec<kFewRegs>();
        if (warp == 0 || warp == 2) {
            // -------------------------------------------------------- TMA producers: A (warp 0), B (warp 2)
            uint32_t s = 0, phase = 0, issued = 0;
            bool ok = true;
            const bool side_a = warp == 0;
            const int mn = side_a ? p.a_mn : p.b_mn;
            // (fewer than 128 K-contiguous rows of A in all: only those are copied, as in the dense layer kernel)
            const uint32_t tx_bytes = kCtas * (side_a ? static_cast<uint32_t>(p.a_rows) * 128u : b_bytes);
            for (int unit = first_unit; unit < total_units && ok; unit += unit_stride) {
                const LayerTile tc = decode_tile(p, unit, kRowsPerTile);
                const int at = side_a ? tc.m0 + static_cast<int>(cta_rank) * kBlockM : tc.n0 + static_cast<int>(cta_rank) * 128;
                for (int kb = tc.kb0; kb < tc.kb1; ++kb) {
                    if (!mbar_wait_warp(bar_empty + 8u * s, phase ^ 1u, abort_flag, budget)) { ok = false; break; }
                    const uint32_t full_local = bar_full + 8u * s;
                    const uint32_t full = kPair ? mapa_u32(full_local, 0) : full_local;
                    const uint32_t dst = smem_base + s * stage_bytes + (side_a ? 0u : a_bytes);
                    if (elect_one()) {
                        if (leader) mbar_arrive_expect_tx(full_local, tx_bytes);
                        const CUtensorMap* map = side_a ? &p.tmap_a : &p.tmap_b0;
                        const int x = mn ? at : kb * 128, y = mn ? kb * 128 : at;
                        if (kPair) tma_load_2d_pair(dst, map, full, x, y);
                        else tma_load_2d(dst, map, full, x, y);
                    }
                    ++issued;
                    if (++s == static_cast<uint32_t>(p.stages)) { s = 0; phase ^= 1u; }
                }
            }
            if (lane == 0) unwind.put(side_a ? 0 : 1, issued);
        } else if (warp == 1 && leader) {
            // -------------------------------------------------------- MMA issuer
            uint32_t s = 0, phase = 0, acc = 0, acc_phase = 0;
            // 32 k per instruction: 32 bytes of a K-contiguous row, 32 rows of 128 bytes of an M/N-contiguous block.  The
            // second half's columns: 64 rows further, or 64 bytes.
            const uint64_t a_step = p.a_mn ? 256ull : 2ull, b_step = p.b_mn ? 256ull : 2ull, b_half = p.b_mn ? 4ull : 512ull;
            const uint64_t a_first = p.a_mn ? make_mnmajor_desc(smem_base, a_bytes) : make_kmajor_desc(smem_base, 128);
            const uint64_t b_first = p.b_mn ? make_mnmajor_desc(smem_base + a_bytes, b_bytes) : make_kmajor_desc(smem_base + a_bytes, 128);
            const uint32_t stages = p.stages, idesc = p.idesc;
            const bool signal = !(p.debug_flags & 1);          // (test hook, bit 0: the "products ready" signal is withheld)
            bool ok = true;
            for (int unit = first_unit; unit < total_units && ok; unit += unit_stride) {
                for (int left = unit_blocks(unit); left > 0; --left) {
                    if (!wait_fast(bar_full + 8u * s, phase, abort_flag, budget)) { ok = false; break; }
                    const uint64_t a_desc = a_first + static_cast<uint64_t>(s * (stage_bytes >> 4));
                    const uint64_t b_desc = b_first + static_cast<uint64_t>(s * (stage_bytes >> 4));
#pragma unroll
                    for (int h = 0; h < kHalves; ++h) {
                        const uint32_t buf = h * kDepth + acc;
                        if (!wait_fast(bar_tempty + 8u * buf, acc_phase ^ 1u, abort_flag, budget)) { ok = false; break; }
                        tc_fence_after();
                        if (elect_one()) {
#pragma unroll
                            for (uint32_t k = 0; k < 4; ++k)
                                mma_f8<kCtas>(tmem_base + buf * kN, a_desc + a_step * k, b_desc + b_half * h + b_step * k, idesc, k > 0 ? 1u : 0u);
                            if (signal) commit_all<kPair>(bar_tfull + 8u * buf);
                            if (h == kHalves - 1) commit_all<kPair>(bar_empty + 8u * s);
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                    if (++s == stages) { s = 0; phase ^= 1u; }
                    if (++acc == kDepth) { acc = 0; acc_phase ^= 1u; }
                }
            }
        } else if (warp == 3) {
            // -------------------------------------------------------- scales, and where the tiles lie
            // (The summing warps go from block to block in the time of two or three hundred instructions: what does not have to be
            // there is here.)  Loads are two blocks ahead.  Rows, columns and blocks behind the last read the last one's: nothing of
            // what they give is stored.
            constexpr int kB = kVec ? kCtas * 4 : kHalves;
            uint32_t acc = 0, uses = 0, place = 0, tile_no = 0;
            bool ok = true;
            for (int unit = first_unit; unit < total_units && ok; unit += unit_stride, ++tile_no) {
                const LayerTile tc = decode_tile(p, unit, kRowsPerTile);
                if (lane == 0)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %3};"
                                 ::"r"(tile_at + (tile_no & (kTilePlaces - 1)) * 16u), "r"(tc.m0), "r"(tc.n0), "r"(tc.plane) : "memory");
                int row[4];
                long long col[kB];
#pragma unroll
                for (int i = 0; i < 4; ++i) row[i] = min(tc.m0 + static_cast<int>(cta_rank) * kBlockM + lane + 32 * i, p.M - 1);
#pragma unroll
                for (int i = 0; i < kB; ++i) {
                    const int c = min(tc.n0 + (kVec ? lane + 32 * i : 128 * i), p.N - 1);
                    col[i] = kVec ? c : (c >> 7) * p.sb_n;
                }
                float a_s[3][4], b_s[3][kB];
                const auto fetch = [&](int to, int kb) {
                    const long long k = min(kb, tc.kb1 - 1);
#pragma unroll
                    for (int i = 0; i < 4; ++i) a_s[to][i] = p.sa ? __ldg(p.sa + k * p.lds_a + row[i]) : 1.0f;
#pragma unroll
                    for (int i = 0; i < kB; ++i) b_s[to][i] = p.sb ? __ldg(p.sb + k * p.sb_k + col[i]) : 1.0f;
                };
                fetch(0, tc.kb0);
                fetch(1, tc.kb0 + 1);
                for (int kb = tc.kb0; kb < tc.kb1; ++kb) {
                    fetch(2, kb + 2);
#pragma unroll
                    for (int h = 0; h < kHalves; ++h)
                        if (uses > 0 && ok) ok = wait_fast(bar_tfull + 8u * (h * kDepth + acc), (uses - 1) & 1u, abort_flag, budget);
                    if (!ok) break;
                    const uint32_t at = scales + place * kScaleBytes;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t r = static_cast<uint32_t>(lane + 32 * i);
                        if constexpr (kVec) sts_f32(at + r * 4u, a_s[0][i]);
                        else if constexpr (kPair)
                            asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(at + r * 8u), "f"(a_s[0][i] * b_s[0][0]), "f"(a_s[0][i] * b_s[0][kB - 1]) : "memory");
                        else sts_f32(at + r * 4u, a_s[0][i] * b_s[0][0]);
                    }
                    if constexpr (kVec) {
#pragma unroll
                        for (int i = 0; i < kB; ++i) {             // (pair: by halves, in the order of their columns)
                            const uint32_t c = static_cast<uint32_t>(lane + 32 * i);
                            sts_f32(at + 512u + 4u * (kPair ? (c >> 6 & 1u) * 128u + (c & 63u) + (c >> 7) * 64u : c), b_s[0][i]);
                        }
                    }
                    __syncwarp();
                    if (lane == 0) {
#pragma unroll
                        for (int h = 0; h < kHalves; ++h) mbar_arrive(bar_tfull + 8u * (h * kDepth + acc));
                    }
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) a_s[j][i] = a_s[j + 1][i];
#pragma unroll
                        for (int i = 0; i < kB; ++i) b_s[j][i] = b_s[j + 1][i];
                    }
                    if (++acc == kDepth) { acc = 0; ++uses; }
                    if (++place == kPlaces) place = 0;
                }
            }
        }
    } else {
        // ------------------------------------------------------------ sums and outputs
        if constexpr (kPair) regs_inc<kManyRegs>();
        const int e = warp - 4, q = warp & 3, half = e >> 2;
        const uint32_t my_slots = slots + static_cast<uint32_t>(e) * kSlotBuffers * kSlot;
        const uint32_t my_bias = bias_at + static_cast<uint32_t>(e) * 128u;
        const uint32_t my_bar = bar_in + 8u * static_cast<uint32_t>(e * kSlotBuffers);
        // (pair: this half's buffers, 128 columns each; else half the columns of all)
        const uint32_t t_base = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + static_cast<uint32_t>(kPair ? half * kDepth * kN : half * kCols);
        const uint32_t my_tfull = bar_tfull + (kPair ? 8u * half * kDepth : 0u);
        uint32_t my_tempty = bar_tempty + (kPair ? 8u * half * kDepth : 0u);
        if (kPair) my_tempty = mapa_u32(my_tempty, 0);             // the leader's
        constexpr int kRuns = kCols / 32;
        // columns of the tile that a thread's c-th run of 32 is
        const auto run_col = [&](int c) { return kPair ? 64 * half + 32 * (c & 1) + 128 * (c >> 1) : half * kCols + 32 * c; };
        // where this row's scales lie in a block's place, and those of this warp's columns
        const uint32_t my_scale = scales + static_cast<uint32_t>(q * 32 + lane) * (kVec || !kPair ? 4u : 8u);
        const uint32_t my_cols = scales + 512u + static_cast<uint32_t>(half * kCols) * 4u;
        const bool f16 = p.type == kF16, has_r = p.R != nullptr, r_tma = !kRaw && p.r_tma != 0, c_tma = p.c_tma != 0;
        uint32_t acc = 0, acc_phase = 0, place = 0, tile_no = 0, loads = 0, taken = 0;     // tile loads asked for, and waited for
        bool ok = true;
        for (int unit = first_unit; unit < total_units && ok; unit += unit_stride, ++tile_no) {
            struct { int m0, n0, plane; } tc = {};
            int row0 = 0;
            const auto read_tile = [&] {
                int none;
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(tc.m0), "=r"(tc.n0), "=r"(tc.plane), "=r"(none) : "r"(tile_at + (tile_no & (kTilePlaces - 1)) * 16u) : "memory");
                row0 = tc.m0 + static_cast<int>(cta_rank) * kBlockM + q * 32;
            };
            const auto run_ok = [&](int c) { return row0 < p.M && tc.n0 + run_col(c) < p.N; };       // (warp-uniform)
            // what the slots hold in the end: the first of it is asked for beside the first block
            int asked = 0;                                         // runs
            const auto ask_round = [&] {
                fence_proxy_async_smem();
                __syncwarp();
                for (int i = 0; i < kSlotBuffers && asked < kRuns && run_ok(asked); ++i) {
                    const uint32_t b = loads % kSlotBuffers;
                    if (elect_one()) {
                        mbar_arrive_expect_tx(my_bar + 8u * b, kSlot);
                        tma_load_2d(my_slots + b * kSlot, &p.tmap_r, my_bar + 8u * b, tc.n0 + run_col(asked), row0);
                    }
                    __syncwarp();
                    ++asked;
                    ++loads;
                }
            };
            uint64_t sum[kCols / 2];
#pragma unroll
            for (int j = 0; j < kCols / 2; ++j) sum[j] = 0ull;
            const int blocks = unit_blocks(unit);
            for (int i = 0; i < blocks; ++i) {
                if (!wait_fast(my_tfull + 8u * acc, acc_phase, abort_flag, budget)) { ok = false; break; }
                tc_fence_after();
                const uint32_t t_at = t_base + acc * kN, at = place * kScaleBytes;
                uint32_t v[2][16];
                tmem_ld_32x16(t_at, v[0]);
                uint64_t s2[2];
                if constexpr (kVec || !kPair) {
                    float s;
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(s) : "r"(my_scale + at) : "memory");
                    s2[0] = s2[1] = pack_f2(s, s);
                } else {
                    float s0, s1;
                    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(s0), "=f"(s1) : "r"(my_scale + at) : "memory");
                    s2[0] = pack_f2(s0, s0);
                    s2[1] = pack_f2(s1, s1);
                }
#pragma unroll
                for (int c = 0; c < kCols / 16; ++c) {
                    const uint32_t cols_at = my_cols + at + static_cast<uint32_t>(16 * c) * 4u;
                    const bool last = c + 1 == kCols / 16;
                    float b_s[4][4];                               // (of the last run; before it there are no registers for all of a run's)
                    if (kVec && last) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) lds_f4(cols_at + 16u * j, b_s[j]);
                    }
                    tmem_ld_wait_for_16(v[c & 1]);
                    if (!last) {
                        tmem_ld_32x16(t_at + 16 * (c + 1), v[(c + 1) & 1]);
                    } else {
                        // the buffer is the tensor core's again, and the scales' place the scales' warp's: what is left of both is
                        // in registers
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) {
                            if (kPair) mbar_arrive_cluster(my_tempty + 8u * acc);
                            else mbar_arrive(my_tempty + 8u * acc);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 16; j += 4) {
                        const uint64_t x0 = words_f2(v[c & 1][j], v[c & 1][j + 1]), x1 = words_f2(v[c & 1][j + 2], v[c & 1][j + 3]);
                        uint64_t* to = &sum[8 * c + j / 2];
                        if constexpr (kVec) {
                            float (&b)[4] = b_s[j / 4];
                            if (!last) lds_f4(cols_at + 4u * j, b);
                            to[0] = fma_f2(mul_f2(x0, pack_f2(b[0], b[1])), s2[0], to[0]);
                            to[1] = fma_f2(mul_f2(x1, pack_f2(b[2], b[3])), s2[0], to[1]);
                        } else {
                            to[0] = fma_f2(x0, s2[c / (kRuns)], to[0]);
                            to[1] = fma_f2(x1, s2[c / (kRuns)], to[1]);
                        }
                    }
                }
                if (++acc == kDepth) { acc = 0; acc_phase ^= 1u; }
                if (++place == kPlaces) place = 0;
                if (r_tma && i == 0) {
                    read_tile();
                    if (run_ok(0)) {
                        if (elect_one()) tma_store_wait_read<0>();
                        __syncwarp();
                        ask_round();
                    }
                }
            }
            if (!ok) break;
            read_tile();
            if constexpr (kRaw) {
                // (planes have whole blocks of 32 rows and columns)
                float* out = static_cast<float*>(p.C) + static_cast<long long>(tc.plane + row0 + lane) * p.ldc + tc.n0;
#pragma unroll
                for (int c = 0; c < kRuns; ++c) {
                    if (!run_ok(c)) continue;
                    uint32_t w[32];
#pragma unroll
                    for (int j = 0; j < 16; ++j) asm("mov.b64 {%0, %1}, %2;" : "=r"(w[2 * j]), "=r"(w[2 * j + 1]) : "l"(sum[16 * c + j]));
#pragma unroll
                    for (int j = 0; j < 4; ++j) st_global_v8(reinterpret_cast<int32_t*>(out) + run_col(c) + 8 * j, &w[8 * j]);
                }
            } else {
                // by rounds of as many slots as there are: one fence and one wait for a round
#pragma unroll
                for (int c0 = 0; c0 < kRuns; c0 += kSlotBuffers) {
                    if (!run_ok(c0) || !ok) continue;
                    if (!r_tma || c0 > 0) {
                        if (c_tma && elect_one()) tma_store_wait_read<0>();
                        __syncwarp();
                        if (r_tma) ask_round();
                    }
#pragma unroll
                    for (int c = c0; c < c0 + kSlotBuffers && c < kRuns; ++c) {
                        if (!run_ok(c) || !ok) continue;
                        const int col = tc.n0 + run_col(c);
                        // (buffers by turns: a round that asks for tiles begins where the last one ended)
                        const uint32_t b = r_tma ? taken % kSlotBuffers : static_cast<uint32_t>(c - c0), at = my_slots + b * kSlot;
                        if (r_tma) {
                            ok = mbar_wait_warp(my_bar + 8u * b, (taken / kSlotBuffers) & 1u, abort_flag, budget);
                            if (!ok) continue;
                            ++taken;
                        } else if (has_r) {
                            slot_rows_in<kWide>(at, p.R, p.ldr, row0, col, p.M, p.N, lane);
                        }
                        if (p.bias) {
                            __syncwarp();
                            sts_f32(my_bias + lane * 4, col + lane < p.N ? __ldg(p.bias + col + lane) : 0.0f);
                            __syncwarp();
                        }
                        constexpr int kPer = kWide ? 4 : 8;        // columns per 16-byte piece
#pragma unroll
                        for (int g = 0; g < 32 / kPer; ++g) {
                            float y[kPer];
#pragma unroll
                            for (int j = 0; j < kPer; j += 2) unpack_f2(sum[16 * c + (g * kPer + j) / 2], y[j], y[j + 1]);
                            if (p.bias) {
#pragma unroll
                                for (int j = 0; j < kPer; j += 4) {
                                    float bv[4];
                                    lds_f4(my_bias + static_cast<uint32_t>(g * kPer + j) * 4u, bv);
#pragma unroll
                                    for (int i = 0; i < 4; ++i) y[j + i] += bv[i];
                                }
                            }
                            uint32_t o[4];
                            if (has_r) {
                                lds_v4(slot_piece<kWide>(at, lane, g), o);
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    if constexpr (kWide) {
                                        y[j] += __uint_as_float(o[j]);
                                    } else {
                                        float lo, hi;
                                        unpack2(o[j], f16, lo, hi);
                                        y[2 * j] += lo;
                                        y[2 * j + 1] += hi;
                                    }
                                }
                            }
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                if constexpr (kWide) o[j] = __float_as_uint(y[j]);
                                else o[j] = pack2(y[2 * j], y[2 * j + 1], f16);
                            }
                            st_shared_v4(slot_piece<kWide>(at, lane, g), o);
                        }
                        if (!c_tma) slot_rows_out<kWide>(at, p.C, p.ldc, row0, col, p.M, p.N, lane);
                    }
                    if (c_tma && ok) {
                        fence_proxy_async_smem();
                        __syncwarp();
                        const uint32_t first = r_tma ? taken : 0u;             // (of the round's tiles the last one was taken before)
                        int n = 0;
#pragma unroll
                        for (int c = c0; c < c0 + kSlotBuffers && c < kRuns; ++c) n += run_ok(c) ? 1 : 0;
                        if (elect_one()) {
                            for (int i = 0; i < n; ++i) {
                                const uint32_t b = r_tma ? (first - n + i) % kSlotBuffers : static_cast<uint32_t>(i);
                                tma_store_2d(&p.tmap_c, my_slots + b * kSlot, tc.n0 + run_col(c0 + i), row0);
                            }
                            tma_store_commit();
                        }
                        __syncwarp();
                    }
                }
            }
        }
        // unwinding: tiles still on their way into the slots
        for (uint32_t i = taken; r_tma && i < loads; ++i) {
            const uint64_t t0 = globaltimer_ns();
            while (!mbar_try_wait(my_bar + 8u * (i % kSlotBuffers), (i / kSlotBuffers) & 1u)) {
                if (globaltimer_ns() - t0 > budget) break;
            }
        }
        __syncwarp();
        if (!kRaw && c_tma && elect_one()) tma_store_wait<0>();
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
        tmem_dealloc<kCtas>(tmem_base, 512);
    }
    if (threadIdx.x == 0 && *abort_flag != 0) atomicOr(p.status, 1u);
}

// Adds planes of partial sums in the order of K, the bias and the residual.  Without planes every sum is 0.
constexpr int kFinishThreads = 256, kFinishCols = 4;
__global__ void __launch_bounds__(kFinishThreads)
mip_f8_finish_kernel(const F8ProductArgs a, const PartialPlanes s) {
    const long long row = static_cast<long long>(blockIdx.y) * blockDim.y + threadIdx.y;
    const long long col = (static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x) * kFinishCols;
    if (row >= a.M || col >= a.N) return;
    float v[kFinishCols] = {0.0f, 0.0f, 0.0f, 0.0f};
    const float* src = static_cast<const float*>(s.base) + row * s.pitch + col;
#pragma unroll 4
    for (int k = 0; k < s.split; ++k) {
        const float4 x = *reinterpret_cast<const float4*>(src + k * s.plane_rows * s.pitch);
        v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
    }
    const int cols = static_cast<int>(min(static_cast<long long>(kFinishCols), a.N - col));
#pragma unroll
    for (int j = 0; j < kFinishCols; ++j)
        if (j < cols) v[j] += (a.bias ? __ldg(a.bias + col + j) : 0.0f) + (a.R ? load_element(a.R, row * a.ldr + col + j, a.type) : 0.0f);
#pragma unroll
    for (int j = 0; j < kFinishCols; ++j)
        if (j < cols) store_element(a.C, row * a.ldc + col + j, a.type, v[j]);
}

// (checks the register split against what the kernel was compiled to: a warp that asks for more than the block holds waits for ever)
template <bool kPair, bool kVec, bool kWide, bool kRaw>
cudaError_t init_t() {
    const auto kernel = mip_f8_product_kernel<kPair, kVec, kWide, kRaw>;
    if (kPair) {
        cudaFuncAttributes attr;
        const cudaError_t e = cudaFuncGetAttributes(&attr, kernel);
        if (e != cudaSuccess) return e;
        if (attr.numRegs < kLaunchRegs) return cudaErrorInvalidKernelImage;
    }
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBudget);
}
template <bool kPair, bool kVec>
cudaError_t init_form() {
    for (cudaError_t e : {init_t<kPair, kVec, false, false>(), init_t<kPair, kVec, true, false>(), init_t<kPair, kVec, true, true>()})
        if (e != cudaSuccess) return e;
    return cudaSuccess;
}
template <bool kPair, bool kVec>
cudaError_t launch_form(const F8ProductParams& p, bool raw, const cudaLaunchConfig_t& cfg) {
    if (raw) return cudaLaunchKernelEx(&cfg, mip_f8_product_kernel<kPair, kVec, true, true>, p);
    return p.type == kF32 ? cudaLaunchKernelEx(&cfg, mip_f8_product_kernel<kPair, kVec, true, false>, p)
                          : cudaLaunchKernelEx(&cfg, mip_f8_product_kernel<kPair, kVec, false, false>, p);
}

size_t smem_of(int type, bool pair, bool vec, bool raw, int stages) {
    return static_cast<size_t>(stages) * 32768 + (raw ? 0 : all_slot_bytes(type == kF32)) + scale_places(pair) * scale_bytes(pair, vec) + kBiasBytes + kCtrlBytes + tile_bytes(pair) + 1024;
}

}  // namespace

int f8_product_stages(int type, bool pair, bool vec, bool raw) {
    int stages = kMaxF8Stages;
    while (smem_of(type, pair, vec, raw, stages) > kSmemBudget) --stages;
    return stages;
}

cudaError_t f8_product_init() {
    for (cudaError_t e : {init_form<false, false>(), init_form<false, true>(), init_form<true, false>(), init_form<true, true>()})
        if (e != cudaSuccess) return e;
    return cudaSuccess;
}

cudaError_t launch_f8_product(const F8ProductParams& p, bool pair, bool vec, bool raw, int grid, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(grid), 1, 1);
    cfg.blockDim = dim3(kF8Threads, 1, 1);
    cfg.dynamicSmemBytes = std::max(kSmemFloor, smem_of(p.type, pair, vec, raw, p.stages));
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
    if (pair) return vec ? launch_form<true, true>(p, raw, cfg) : launch_form<true, false>(p, raw, cfg);
    return vec ? launch_form<false, true>(p, raw, cfg) : launch_form<false, false>(p, raw, cfg);
}

cudaError_t launch_f8_finish(const F8ProductArgs& a, const PartialPlanes& s, cudaStream_t stream, int* launches) {
    int tx = 8;
    while (tx < kFinishThreads && tx * kFinishCols < a.N) tx *= 2;
    const int ty = kFinishThreads / tx;
    const long long step = 65535LL * ty, size = a.type == kF32 ? 4 : 2;      // (the grid's second dimension holds 65535 blocks)
    for (long long row = 0; row < a.M; row += step) {
        F8ProductArgs part = a;
        PartialPlanes planes = s;
        part.M = a.M - row < step ? a.M - row : step;
        part.C = static_cast<char*>(a.C) + row * a.ldc * size;
        if (a.R) part.R = static_cast<const char*>(a.R) + row * a.ldr * size;
        if (s.base) planes.base = static_cast<const char*>(s.base) + row * s.pitch * 4;
        const dim3 grid(static_cast<unsigned>((a.N + tx * kFinishCols - 1) / (tx * kFinishCols)), static_cast<unsigned>((part.M + ty - 1) / ty));
        mip_f8_finish_kernel<<<grid, dim3(tx, ty), 0, stream>>>(part, planes);
        ++*launches;
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace mip
