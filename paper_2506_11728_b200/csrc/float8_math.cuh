// What the kernels of the 8-bit floating-point operators share: conversions, the rule for a block's scale, and accesses
// to runs of elements.
#pragma once
#include <cstdint>

#include "layer_math.cuh"

namespace mip {

// values of mipgemm_f8_format_t, mipgemm_f8_blocks_t (checked in api.cu)
constexpr int kE4M3 = 0, kE5M2 = 1;
constexpr int kBlocksRows = 0, kBlocksColumns = 1, kBlocksSquares = 2;
constexpr int kF8Block = 128;        // elements along a block's side

// Two values to codes in the low and the high byte, rounded to nearest even; codes back to float16 pairs, exact.
template <int kFormat>
__device__ __forceinline__ uint32_t f8_pair(float lo, float hi) {
    uint16_t r;
    if (kFormat == kE4M3) asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
template <int kFormat>
__device__ __forceinline__ float2 f8_values(uint32_t pair) {
    uint32_t h;
    const uint16_t p = static_cast<uint16_t>(pair);
    if (kFormat == kE4M3) asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(p));
    else asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(h) : "h"(p));
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// A block's scale and multiplier from its largest magnitude: scale = top / L, codes = rne(x * (L / top)), L the format's
// largest value.  Below 2^-119 (e4m3) or 2^-112 (e5m2), where L / top would leave the binary32 range: scale 0, codes 0.
// An infinity or a NaN in the block: scale NaN, codes 0.  (A multiplier of 0 stands for "codes 0".)
struct F8Scale {
    float scale, mult;
};
template <int kFormat>
__device__ __forceinline__ F8Scale f8_scale(float top) {
    constexpr float kLargest = kFormat == kE4M3 ? 448.0f : 57344.0f, kLeast = kFormat == kE4M3 ? 0x1p-119f : 0x1p-112f;
    F8Scale s{0.0f, 0.0f};
    if (!(top <= 3.402823466e38f)) s.scale = __int_as_float(0x7FFFFFFF);
    else if (top >= kLeast) s = F8Scale{__fdiv_rn(top, kLargest), __fdiv_rn(kLargest, top)};
    return s;
}
// Four codes in a word (0 where the multiplier is: an infinity times 0 would be NaN).
template <int kFormat>
__device__ __forceinline__ uint32_t f8_codes4(float a, float b, float c, float d, float mult) {
    const uint32_t q = f8_pair<kFormat>(__fmul_rn(a, mult), __fmul_rn(b, mult)) | (f8_pair<kFormat>(__fmul_rn(c, mult), __fmul_rn(d, mult)) << 16);
    return mult == 0.0f ? 0u : q;
}

// The bits of |x|: they order like the magnitudes, with infinities and NaNs on top.
__device__ __forceinline__ uint32_t magnitude_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// The larger magnitude; a NaN stays one.
__device__ __forceinline__ float max_magnitude(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)));
    return r;
}

// ---- elements as they lie, in words: 2 of 16 bits or 1 of 32 per word
template <int kType>
__device__ __forceinline__ float2 unpack_pair(uint32_t w) {          // 16-bit types
    if (kType == kF16) return __half22float2(*reinterpret_cast<const __half2*>(&w));
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <int kType>
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {
    if (kType == kF16) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <int kType>
__device__ __forceinline__ float load_one(const void* p, long long i) { return load_element(p, i, kType); }
template <int kType>
__device__ __forceinline__ void store_one(void* p, long long i, float v) { store_element(p, i, kType, v); }

// Reads that pass the first-level cache by; not through the read-only path, as the output may be the input.
__device__ __forceinline__ uint4 ld_once_v4(const void* p) {
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}

// Eight consecutive elements.  load, and store where `wide`: 16-byte accesses, all eight exist or none; store else: element by
// element, `count` of them exist.  Where rows lie on no 16-byte boundary a warp takes its 256 by turns, lane by lane, and brings
// them into order, or out of it, through 256 elements of shared memory (load_spread and gather, scatter and store_spread: all
// lanes together).
template <int kType>
struct Eight {
    uint32_t w[kType == kF32 ? 8 : 4];
    __device__ __forceinline__ void load(const void* base, long long at, int count) {
        if (count > 0) {
            const char* p = static_cast<const char*>(base) + at * (kType == kF32 ? 4 : 2);
#pragma unroll
            for (int i = 0; i < (kType == kF32 ? 2 : 1); ++i) put(i, ld_once_v4(p + 16 * i));
        } else {
            clear();
        }
    }
    __device__ __forceinline__ void put(int i, uint4 x) { w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w; }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < (kType == kF32 ? 8 : 4); ++i) w[i] = 0u;
    }
    // The warp's elements lane, lane + 32, ...; `limit` of its 256 exist.  (A whole run, as nearly all are, without a question for
    // each element.  16-bit elements one at a time: in words, of which every other row's are split at both ends, it took longer.)
    template <bool kWhole>
    __device__ __forceinline__ void load_spread_as(const void* base, int limit) {
        const int lane = threadIdx.x & 31;
        const auto get = [&](int i) -> uint32_t {
            if (!kWhole && lane + 32 * i >= limit) return 0u;
            if constexpr (kType == kF32) return static_cast<const uint32_t*>(base)[lane + 32 * i];
            else return static_cast<const uint16_t*>(base)[lane + 32 * i];
        };
        if constexpr (kType == kF32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = get(i);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = get(2 * i) | (get(2 * i + 1) << 16);
        }
    }
    __device__ __forceinline__ void load_spread(const void* base, int limit) {
        if (limit == 256) load_spread_as<true>(base, limit);
        else load_spread_as<false>(base, limit);
    }
    template <bool kWhole>
    __device__ __forceinline__ void store_spread_as(void* base, int limit) const {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (!kWhole && lane + 32 * i >= limit) continue;
            if constexpr (kType == kF32) static_cast<uint32_t*>(base)[lane + 32 * i] = w[i];
            else static_cast<uint16_t*>(base)[lane + 32 * i] = static_cast<uint16_t>(w[i / 2] >> (16 * (i & 1)));
        }
    }
    __device__ __forceinline__ void store_spread(void* base, int limit) const {
        if (limit == 256) store_spread_as<true>(base, limit);
        else store_spread_as<false>(base, limit);
    }
    // by turns -> in order, and back; buf: the warp's 256 elements of shared memory
    __device__ __forceinline__ void gather(uint32_t* buf) {
        const int lane = threadIdx.x & 31;
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (kType == kF32) buf[lane + 32 * i] = w[i];
            else reinterpret_cast<uint16_t*>(buf)[lane + 32 * i] = static_cast<uint16_t>(w[i / 2] >> (16 * (i & 1)));
        }
        __syncwarp();
        const uint4* const q = reinterpret_cast<const uint4*>(buf) + lane * (kType == kF32 ? 2 : 1);
#pragma unroll
        for (int i = 0; i < (kType == kF32 ? 2 : 1); ++i) put(i, q[i]);
    }
    __device__ __forceinline__ void scatter(uint32_t* buf) {
        const int lane = threadIdx.x & 31;
        __syncwarp();
        uint4* const q = reinterpret_cast<uint4*>(buf) + lane * (kType == kF32 ? 2 : 1);
#pragma unroll
        for (int i = 0; i < (kType == kF32 ? 2 : 1); ++i) q[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        __syncwarp();
        if constexpr (kType == kF32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = buf[lane + 32 * i];
        } else {
            const uint16_t* const b = reinterpret_cast<const uint16_t*>(buf);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = b[lane + 64 * i] | (static_cast<uint32_t>(b[lane + 64 * i + 32]) << 16);
        }
    }
    __device__ __forceinline__ void values(float (&v)[8]) const {
        if constexpr (kType == kF32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 t = unpack_pair<kType>(w[i]);
                v[2 * i] = t.x;
                v[2 * i + 1] = t.y;
            }
        }
    }
    // Two neighbours in a register pair, for the packed instructions.
    __device__ __forceinline__ void pairs(uint64_t (&v)[4]) const {
        if constexpr (kType == kF32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = pack_f2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 t = unpack_pair<kType>(w[i]);
                v[i] = pack_f2(t.x, t.y);
            }
        }
    }
    __device__ __forceinline__ void set_pairs(const uint64_t (&v)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float lo, hi;
            unpack_f2(v[i], lo, hi);
            if constexpr (kType == kF32) {
                w[2 * i] = __float_as_uint(lo);
                w[2 * i + 1] = __float_as_uint(hi);
            } else {
                w[i] = pack_pair<kType>(lo, hi);
            }
        }
    }
    __device__ __forceinline__ void set(const float (&v)[8]) {
        if constexpr (kType == kF32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = pack_pair<kType>(v[2 * i], v[2 * i + 1]);
        }
    }
    __device__ __forceinline__ void store(void* base, long long at, int count, bool wide) const {
        if (wide) {
            char* p = static_cast<char*>(base) + at * (kType == kF32 ? 4 : 2);
            if (count > 0) {
                *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(w);
                if constexpr (kType == kF32) *reinterpret_cast<uint4*>(p + 16) = *reinterpret_cast<const uint4*>(w + 4);
            }
        } else if constexpr (kType == kF32) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) static_cast<uint32_t*>(base)[at + i] = w[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) static_cast<uint16_t*>(base)[at + i] = static_cast<uint16_t>(w[i / 2] >> (16 * (i & 1)));
        }
    }
};

// Eight float32 of a vector that every row reads (cached), `fill` where it is absent.  `wide`: it lies on 16 bytes.
__device__ __forceinline__ void load_vector8(const float* p, long long at, int count, bool wide, float fill, float (&v)[8]) {
    if (!p) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fill;
    } else if (wide && (count == 0 || count == 8)) {
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
        if (count > 0) {
            a = __ldg(reinterpret_cast<const float4*>(p + at));
            b = __ldg(reinterpret_cast<const float4*>(p + at) + 1);
        }
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < count ? __ldg(p + at + i) : 0.0f;
    }
}

}  // namespace mip
