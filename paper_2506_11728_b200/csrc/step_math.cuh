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
// from a counter of 128 and a key of 64.
__device__ __forceinline__ uint4 philox10(uint4 c, uint2 k) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint32_t h0 = __umulhi(0xD2511F53u, c.x), l0 = 0xD2511F53u * c.x;
        const uint32_t h1 = __umulhi(0xCD9E8D57u, c.z), l1 = 0xCD9E8D57u * c.z;
        c = make_uint4(h1 ^ c.y ^ k.x, l1, h0 ^ c.w ^ k.y, l0);
        k.x += 0x9E3779B9u;
        k.y += 0xBB67AE85u;
    }
    return c;
}

// The mask of eight neighbouring columns: one draw, 16 bits for each.  v[j] becomes v[j] * scale where the bits are `bar`
// or more, 0 (whatever v[j] is) where they are below.
struct Dropout {
    uint32_t bar;                        // 0: nothing is dropped
    float scale;                         // 65536 / (65536 - bar)
    uint2 key;
    unsigned long long step;             // the caller's counter
    unsigned long long groups;           // of eight columns in a row
    __device__ __forceinline__ uint4 draw(long long row, long long col) const {
        const unsigned long long g = static_cast<unsigned long long>(row) * groups + (static_cast<unsigned long long>(col) >> 3);
        return philox10(make_uint4(static_cast<uint32_t>(g), static_cast<uint32_t>(g >> 32), static_cast<uint32_t>(step), static_cast<uint32_t>(step >> 32)), key);
    }
    __device__ __forceinline__ void apply(const uint4& bits, float (&v)[8]) const {
        const uint32_t w[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t r = j & 1 ? w[j / 2] >> 16 : w[j / 2] & 0xFFFFu;
            v[j] = r >= bar ? v[j] * scale : 0.0f;
        }
    }
};
__device__ __forceinline__ Dropout dropout_of(uint32_t bar, float scale, unsigned long long seed, const unsigned long long* counter, long long N) {
    return Dropout{bar, scale, make_uint2(static_cast<uint32_t>(seed), static_cast<uint32_t>(seed >> 32)), bar && counter ? *counter : 0ull,
                   (static_cast<unsigned long long>(N) + 7) / 8};
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}

// A multiple of 32 threads a row, up to 1024; blockDim.y rows side by side go through the same calls.
constexpr int kMaxRowWarps = 32;
constexpr int kMaxBlockRows = 4;         // rows per block where a row takes fewer than 128 threads

}  // namespace mip
