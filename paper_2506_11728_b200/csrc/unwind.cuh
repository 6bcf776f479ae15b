// What a kernel that gives up a bounded wait does about the copies still on their way into its shared memory: all of them
// have to land before the memory is given back, also those that only one of several producers has asked for.
//
// Producers walk the same stages, each at its own pace, and stop wherever they notice the abort word; up to `stages` uses
// of the stage buffers may then have been asked for by some of them only, and the "full" barrier of such a use would
// never complete.  The leader CTA, whose barriers count the bytes of both CTAs of a pair, supplies what is missing once
// every producer has stopped -- the arrivals that were never made, without bytes, and the bytes it expects of copies
// that were never asked for -- and then waits for the barriers, which complete when the copies in flight have landed.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define MIP_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define MIP_HOST_DEVICE inline
#endif

namespace mip {

// What is missing on the barrier of one use, for one operand: an arrival (with the bytes it expects), or bytes that an
// arrival made earlier expects of a copy that was never asked for.
struct MissingCopy {
    bool arrive;
    uint32_t expect, complete;
};
// leader, peer: uses that the operand's producer has asked for, in the leader CTA (which arrives, expecting both CTAs'
// bytes) and in its peer; without a peer both are the same.  bytes: of the operand, per CTA.
MIP_HOST_DEVICE MissingCopy missing_copy(uint32_t use, uint32_t leader, uint32_t peer, uint32_t bytes) {
    MissingCopy m = {false, 0u, 0u};
    if (leader > use) {
        if (peer <= use) m.complete = bytes;
    } else {
        m.arrive = true;
        if (peer > use) m.expect = bytes;
    }
    return m;
}
// The uses that may still be on their way: [first, last).  Older ones have been read by the MMAs of a later use.
MIP_HOST_DEVICE uint32_t uses_last(uint32_t a, uint32_t b) { return a > b ? a : b; }
MIP_HOST_DEVICE uint32_t uses_first(uint32_t last, uint32_t stages) { return last > stages ? last - stages : 0u; }

}  // namespace mip

#ifdef __CUDACC__
#include "ptx.cuh"

namespace mip {

// Uses that a CTA's producers have asked for, by operand (0: A, 1: B), and whether it unwinds, as words in shared memory:
// [abort of the peer, its A, its B] of the pair forms, then this CTA's A and B (the product's B is its CTA's own affair).
struct UnwindWords {
    uint32_t addr;
    static constexpr uint32_t kBytes = 20;
    __device__ __forceinline__ void put(int operand, uint32_t uses) const {
        asm volatile("st.shared.b32 [%0], %1;" ::"r"(addr + 12u + 4u * operand), "r"(uses) : "memory");
    }
    __device__ __forceinline__ uint32_t get(int word) const {
        uint32_t v;
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(addr + 4u * word) : "memory");
        return v;
    }
    // One thread of a pair's CTA tells the other one; the cluster barrier after it makes it visible.
    __device__ __forceinline__ void tell(uint32_t other, uint32_t abort) const {
        const uint32_t dst = mapa_u32(addr, other);
        asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(dst), "r"(abort) : "memory");
        asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(dst + 4u), "r"(get(3)) : "memory");
        asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(dst + 8u), "r"(get(4)) : "memory");
    }
};

// Waits (bounded) until no copy into the stages is on its way; all lanes of one warp of the leader CTA, when every
// producer of the CTA and of its peer has stopped.  kOperands: that arrive on the barriers (1: A alone).
template <bool kPair, int kOperands>
__device__ __forceinline__ void drain_copies(const UnwindWords& words, uint32_t bar_full, uint32_t stages, uint32_t a_bytes, uint32_t b_bytes,
                                             int lane, uint64_t budget_ns) {
    uint32_t mine[2], peer[2], last = 0;
    for (int o = 0; o < kOperands; ++o) {
        mine[o] = words.get(3 + o);
        peer[o] = kPair ? words.get(1 + o) : mine[o];
        last = uses_last(last, uses_last(mine[o], peer[o]));
    }
    if (lane == 0) {
        for (uint32_t use = uses_first(last, stages); use < last; ++use) {
            const uint32_t bar = bar_full + 8u * (use % stages);
            for (int o = 0; o < kOperands; ++o) {
                const MissingCopy m = missing_copy(use, mine[o], peer[o], o ? b_bytes : a_bytes);
                if (m.complete) mbar_complete_tx(bar, m.complete);
                if (m.arrive) mbar_arrive_expect_tx(bar, m.expect);
            }
        }
    }
    __syncwarp();
    for (uint32_t use = uses_first(last, stages); use < last; ++use) {
        const uint64_t t0 = globaltimer_ns();
        while (!mbar_try_wait(bar_full + 8u * (use % stages), (use / stages) & 1u)) {
            if (globaltimer_ns() - t0 > budget_ns) break;
        }
    }
    __syncwarp();
}

}  // namespace mip
#endif
