// What the forward and the backward kernel of the step between two blocks share: the dropout mask and sums over a row.
#pragma once
#include <cstdint>

#include "float8_math.cuh"
#include "internal.h"

namespace mip {

// values of mipgemm_norm_t and mipgemm_codes_t (checked in api.cu)
constexpr int kNormNone = 0, kNormRms = 1, kNormLayer = 2;
constexpr int kCodesNone = 0, kCodesS8 = 1, kCodesE4M3 = 2, kCodesE5M2 = 3;

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011): four words of 32 bits
// from a counter of 128 and a key of 64.  The rounds' keys -- the key, raised by two constants from round to round -- come
// worked out, as kernel arguments: an exclusive-or takes them from there.
constexpr int kPhiloxRounds = 10;
inline void philox_keys(unsigned long long seed, uint32_t (&keys)[2 * kPhiloxRounds]) {
    for (int r = 0; r < kPhiloxRounds; ++r) {
        keys[2 * r] = static_cast<uint32_t>(seed) + static_cast<uint32_t>(r) * 0x9E3779B9u;
        keys[2 * r + 1] = static_cast<uint32_t>(seed >> 32) + static_cast<uint32_t>(r) * 0xBB67AE85u;
    }
}
__device__ __forceinline__ uint4 philox(uint4 c, const uint32_t (&keys)[2 * kPhiloxRounds]) {
#pragma unroll
    for (int r = 0; r < kPhiloxRounds; ++r) {
        // (one wide multiplication instead of two halves)
        const uint64_t p0 = static_cast<uint64_t>(0xD2511F53u) * c.x, p1 = static_cast<uint64_t>(0xCD9E8D57u) * c.z;
        c = make_uint4(static_cast<uint32_t>(p1 >> 32) ^ c.y ^ keys[2 * r], static_cast<uint32_t>(p1),
                       static_cast<uint32_t>(p0 >> 32) ^ c.w ^ keys[2 * r + 1], static_cast<uint32_t>(p0));
    }
    return c;
}

// The mask of eight neighbouring columns: one draw, 16 bits for each.  An element becomes itself times `scale` where its bits
// are the bar or more, 0 (whatever it is) where they are below.
struct Dropout {
    const StepMask& m;                   // (kernel arguments)
    uint32_t bar;                        // shifted up by 16 bits; 0: nothing is dropped
    unsigned long long step;             // the caller's counter
    unsigned long long groups;           // of eight columns in a row
    __device__ __forceinline__ Dropout(const StepMask& mask, long long N)
        : m(mask), bar(mask.bar << 16), step(mask.bar && mask.counter ? *mask.counter : 0ull), groups((static_cast<unsigned long long>(N) + 7) / 8) {}
    __device__ __forceinline__ uint4 draw(long long row, long long col) const {
        const unsigned long long g = static_cast<unsigned long long>(row) * groups + (static_cast<unsigned long long>(col) >> 3);
        return philox(make_uint4(static_cast<uint32_t>(g), static_cast<uint32_t>(g >> 32), static_cast<uint32_t>(step), static_cast<uint32_t>(step >> 32)), m.keys);
    }
    // A pair without its dropped elements.  (The high half of a word is compared with the low half still behind it: that changes
    // nothing.)
    static __device__ __forceinline__ uint64_t where(bool keep_lo, bool keep_hi, uint64_t v) {
        float lo, hi;
        unpack_f2(v, lo, hi);
        return pack_f2(keep_lo ? lo : 0.0f, keep_hi ? hi : 0.0f);
    }
    __device__ __forceinline__ uint64_t kept(uint32_t word, uint64_t v) const { return where(word << 16 >= bar, word >= bar, v); }
    __device__ __forceinline__ uint64_t scaled(uint64_t v) const { return mul_f2(v, pack_f2(m.scale, m.scale)); }
    __device__ __forceinline__ void apply(const uint4& bits, uint64_t (&v)[4]) const {
        const uint32_t w[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = kept(w[j], scaled(v[j]));
    }
};
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}

__device__ __forceinline__ float sum_pair(uint64_t v) {
    float a, b;
    unpack_f2(v, a, b);
    return a + b;
}
// Eight float32 of a vector that every row reads, as pairs.
__device__ __forceinline__ void load_vector_pairs(const float* p, long long at, int count, bool wide, float fill, uint64_t (&v)[4]) {
    float x[8];
    load_vector8(p, at, count, wide, fill, x);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = pack_f2(x[2 * j], x[2 * j + 1]);
}
// Elements that do not exist become 0.
__device__ __forceinline__ void clear_behind(uint64_t (&v)[4], int count) {
    if (count >= 8) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float a, b;
        unpack_f2(v[j], a, b);
        v[j] = pack_f2(2 * j < count ? a : 0.0f, 2 * j + 1 < count ? b : 0.0f);
    }
}

// A run of eight columns of a thread whose own address is `at`; `limit` of its warp's 256 columns exist.  All lanes together, and
// `buf` is the warp's own; run_pairs brings what load_run took into order.
template <bool kWide, int kType>
__device__ __forceinline__ void load_run(Eight<kType>& e, const void* at, int count, int limit) {
    if constexpr (kWide) e.load(at, 0, count);
    else e.load_spread(static_cast<const char*>(at) - (threadIdx.x & 31) * (kType == kF32 ? 32 : 16), limit);
}
template <bool kWide, int kType>
__device__ __forceinline__ void run_pairs(Eight<kType> e, uint32_t* buf, uint64_t (&v)[4]) {
    if constexpr (!kWide) e.gather(buf);
    e.pairs(v);
}
template <bool kWide, int kType>
__device__ __forceinline__ void store_run(const uint64_t (&v)[4], void* at, int count, int limit, uint32_t* buf) {
    Eight<kType> e;
    e.set_pairs(v);
    if constexpr (kWide) {
        e.store(at, 0, count, true);
    } else {
        e.scatter(buf);
        e.store_spread(static_cast<char*>(at) - (threadIdx.x & 31) * (kType == kF32 ? 32 : 16), limit);
    }
}

// A multiple of 32 threads a row, up to 1024; blockDim.y rows side by side go through the same calls.
constexpr int kMaxRowWarps = 32;
constexpr int kMaxBlockRows = 8;         // rows side by side in a block

}  // namespace mip
