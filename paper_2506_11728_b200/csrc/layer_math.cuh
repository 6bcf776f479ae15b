// Arithmetic shared by the kernels of the 8-bit transformer layer: element types, activations and
// their derivatives, and the transforms from exact integer sums to outputs.  Everything behind the
// integer sum is binary32; a value is rounded once, when it is stored in its type.
#pragma once
#include <cstdint>
#include <type_traits>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace mip {

// values of mipgemm_type_t and mipgemm_activation_t (checked in api.cu)
constexpr int kF32 = 0, kF16 = 1, kBF16 = 2;
constexpr int kActNone = 0, kActRelu = 1, kActGelu = 2, kActGeluTanh = 3, kActSilu = 4;

// The hardware's 2^x and 1/x without the steps that keep subnormal numbers: one instruction each, 2 units in the last
// place and 1.  (The library forms of the exponential and the quotient are four to six: half of an epilogue's time.)
__device__ __forceinline__ float fast_exp2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float fast_rcp(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
constexpr float kLog2E = 1.4426950408889634f;

// 1 / (1 + e^-x): the rounded product x log2(e) puts 0.7 |x| units in the last place into the exponential, at most
// 1e-5 relative where the result is above 1e-35; e^-x = infinity gives the limit 0.
__device__ __forceinline__ float sigmoid(float x) { return fast_rcp(1.0f + fast_exp2(-kLog2E * x)); }

// 2 sqrt(2/pi) (x + 0.044715 x^3): tanh(y/2) = 2 sigmoid(y) - 1 turns the tanh form of the Gaussian
// error unit, x (1 + tanh(sqrt(2/pi) (x + 0.044715 x^3))) / 2, into x sigmoid(gelu_inner(x)).
constexpr float kGeluC = 1.5957691216057308f, kGeluC3 = 0.044715f;
__device__ __forceinline__ float gelu_inner(float x) { return kGeluC * x * (1.0f + kGeluC3 * x * x); }
// x^2 as the factor in its slope takes it: for |x| > 20 what it is multiplied with, x sigmoid (1 - sigmoid), is 0, and has to
// stay 0 where the square leaves the range of binary32.
__device__ __forceinline__ float gelu_square(float xx) { return fminf(xx, 1e4f); }

// The normal distribution's integral Phi(x) = (1 + erf(x / sqrt 2)) / 2 and e^(-x^2 / 2), which its density shares.
// Phi(-|x|) = t P(t) e^(-x^2 / 2), t = 1 / (1 + c |x|): the form of Abramowitz and Stegun 7.1.26, with P and c fitted for the
// least RELATIVE error over |x| <= 13.3, so that small values of the Gaussian error unit and of its slope keep their relative
// size.  Degree 7: 8e-8, and 8e-7 with the rounding of t and of the evaluation; the exponential adds 1.25 x^2 2^-24 and 2
// units.  Degree 5, for results of 16 bits in the dense kernel, whose pace the epilogue's arithmetic can set: 4e-6, 1/60 of a
// float16's half unit.  Measured, linear 16384 x 4096 x 1024 gelu bf16: 80.0 us with the published fit of degree 4 (whose tail is
// off by 1.6e-3 of itself at x = -5), 1.6 % more with degree 5, 3.5 % with degree 7; with a float32 result 95.0 / degree 7 95.8.
// Below x = -13.2 the exponential is 0.  No branch, one exponential and one reciprocal (erff: two polynomials by case and its
// own exponential, twice the time of a whole epilogue).
template <bool kFine>
struct CdfFit {
    static constexpr int kDegree = kFine ? 7 : 5;
    static constexpr float kC = kFine ? 0.23334524f : 0.30759144f;
    __host__ __device__ static constexpr float p(int i) {
        constexpr float kP7[8] = {0.093180843f, 0.091449231f, 0.10078691f, 0.023042437f, 0.20531413f, -0.17672996f, 0.23079321f, -0.067836836f};
        constexpr float kP5[6] = {0.12297821f, 0.11849553f, 0.13743502f, 0.0050410316f, 0.19192345f, -0.075875066f};
        return kFine ? kP7[i] : kP5[i < 6 ? i : 5];
    }
};
__device__ __forceinline__ float normal_cdf(float x, float& gauss) {
    gauss = fast_exp2((-0.5f * kLog2E) * (x * x));
    using Fit = CdfFit<true>;
    const float t = fast_rcp(1.0f + Fit::kC * fabsf(x));
    float q = Fit::p(Fit::kDegree);
#pragma unroll
    for (int i = Fit::kDegree - 1; i >= 0; --i) q = q * t + Fit::p(i);
    const float tail = q * t * gauss;
    return x < 0.0f ? tail : 1.0f - tail;
}

template <int kAct>
__device__ __forceinline__ float activation(float x) {
    if (kAct == kActRelu) return x < 0.0f ? 0.0f : x;           // (NaN stays NaN)
    if (kAct == kActGelu) {
        float gauss;
        return x * normal_cdf(x, gauss);
    }
    if (kAct == kActGeluTanh) return x * sigmoid(gelu_inner(x));
    if (kAct == kActSilu) return x * sigmoid(x);
    return x;
}

// The activation and its derivative, which share the exponential.
template <int kAct>
__device__ __forceinline__ void activation_slope(float x, float& value, float& slope) {
    if (kAct == kActRelu) {
        value = x < 0.0f ? 0.0f : x;
        slope = x > 0.0f ? 1.0f : value;                        // (0 at 0; NaN stays NaN)
    } else if (kAct == kActGelu) {
        float gauss;
        const float cdf = normal_cdf(x, gauss);
        value = x * cdf;
        slope = cdf + x * 0.3989422804014327f * gauss;
    } else if (kAct == kActGeluTanh) {
        const float e = sigmoid(gelu_inner(x));
        value = x * e;
        slope = e + value * (1.0f - e) * kGeluC * (1.0f + 3.0f * kGeluC3 * gelu_square(x * x));
    } else if (kAct == kActSilu) {
        const float e = sigmoid(x);
        value = x * e;
        slope = e * (1.0f + x * (1.0f - e));
    } else {
        value = x;
        slope = 1.0f;
    }
}

// Two binary32 values in a register pair, for the packed instructions: half the issue slots.
__device__ __forceinline__ uint64_t pack_f2(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack_f2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t mul_f2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t add_f2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma_f2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t both(float a) { return pack_f2(a, a); }
template <typename F>
__device__ __forceinline__ uint64_t each(uint64_t v, F&& f) {
    float a, b;
    unpack_f2(v, a, b);
    return pack_f2(f(a), f(b));
}
// 1 / (1 + 2^x)
__device__ __forceinline__ uint64_t sigmoid_exp2_f2(uint64_t x) {
    return each(add_f2(each(x, fast_exp2), both(1.0f)), fast_rcp);
}

template <bool kFine>
__device__ __forceinline__ uint64_t normal_cdf_f2(uint64_t x, uint64_t& gauss) {
    using Fit = CdfFit<kFine>;
    gauss = each(mul_f2(mul_f2(x, x), both(-0.5f * kLog2E)), fast_exp2);
    // (scalar: the magnitude costs no instruction there)
    const uint64_t t = each(x, [](float v) { return fast_rcp(__fmaf_rn(Fit::kC, fabsf(v), 1.0f)); });
    uint64_t q = both(Fit::p(Fit::kDegree));
#pragma unroll
    for (int i = Fit::kDegree - 1; i >= 0; --i) q = fma_f2(q, t, both(Fit::p(i)));
    const uint64_t tail = mul_f2(mul_f2(q, t), gauss);
    const uint64_t rest = fma_f2(tail, both(-1.0f), both(1.0f));
    float x0, x1, t0, t1, r0, r1;
    unpack_f2(x, x0, x1);
    unpack_f2(tail, t0, t1);
    unpack_f2(rest, r0, r1);
    return pack_f2(x0 < 0.0f ? t0 : r0, x1 < 0.0f ? t1 : r1);
}

// The same formulas as activation() and activation_slope(), two values at a time.  kFine: for results of 32 bits.
template <int kAct, bool kFine>
__device__ __forceinline__ uint64_t activation_f2(uint64_t x) {
    if constexpr (kAct == kActSilu) return mul_f2(x, sigmoid_exp2_f2(mul_f2(x, both(-kLog2E))));
    else if constexpr (kAct == kActGeluTanh)
        return mul_f2(x, sigmoid_exp2_f2(mul_f2(x, fma_f2(mul_f2(x, x), both(-kLog2E * kGeluC * kGeluC3), both(-kLog2E * kGeluC)))));
    else if constexpr (kAct == kActGelu) {
        uint64_t gauss;
        return mul_f2(x, normal_cdf_f2<kFine>(x, gauss));
    } else if constexpr (kAct == kActRelu) return each(x, [](float v) { return v < 0.0f ? 0.0f : v; });
    else return x;
}
template <int kAct, bool kFine>
__device__ __forceinline__ void activation_slope_f2(uint64_t x, uint64_t& value, uint64_t& slope) {
    if constexpr (kAct == kActSilu) {
        const uint64_t e = sigmoid_exp2_f2(mul_f2(x, both(-kLog2E)));
        value = mul_f2(x, e);
        slope = fma_f2(value, fma_f2(e, both(-1.0f), both(1.0f)), e);
    } else if constexpr (kAct == kActGeluTanh) {
        const uint64_t xx = mul_f2(x, x);
        const uint64_t e = sigmoid_exp2_f2(mul_f2(x, fma_f2(xx, both(-kLog2E * kGeluC * kGeluC3), both(-kLog2E * kGeluC))));
        value = mul_f2(x, e);
        slope = fma_f2(mul_f2(value, fma_f2(e, both(-1.0f), both(1.0f))),
                       fma_f2(each(xx, gelu_square), both(3.0f * kGeluC * kGeluC3), both(kGeluC)), e);
    } else if constexpr (kAct == kActGelu) {
        uint64_t gauss;
        const uint64_t cdf = normal_cdf_f2<kFine>(x, gauss);
        value = mul_f2(x, cdf);
        slope = fma_f2(mul_f2(x, gauss), both(0.3989422804014327f), cdf);
    } else if constexpr (kAct == kActRelu) {
        value = each(x, [](float v) { return v < 0.0f ? 0.0f : v; });
        float x0, x1, v0, v1;
        unpack_f2(x, x0, x1);
        unpack_f2(value, v0, v1);
        slope = pack_f2(x0 > 0.0f ? 1.0f : v0, x1 > 0.0f ? 1.0f : v1);
    } else {
        value = x;
        slope = both(1.0f);
    }
}

__device__ __forceinline__ float load_element(const void* base, long long i, int type) {
    if (type == kF32) return static_cast<const float*>(base)[i];
    if (type == kF16) return __half2float(static_cast<const __half*>(base)[i]);
    return __bfloat162float(static_cast<const __nv_bfloat16*>(base)[i]);
}
__device__ __forceinline__ void store_element(void* base, long long i, int type, float v) {
    if (type == kF32) static_cast<float*>(base)[i] = v;
    else if (type == kF16) static_cast<__half*>(base)[i] = __float2half_rn(v);
    else static_cast<__nv_bfloat16*>(base)[i] = __float2bfloat16_rn(v);
}

__device__ __forceinline__ float scale_at(const float* s, long long i) { return s ? __ldg(s + i) : 1.0f; }

// Runs `body` with the activation as a compile-time constant.
template <typename F>
__device__ __forceinline__ void with_activation(int act, F&& body) {
    switch (act) {
        case kActRelu: body(std::integral_constant<int, kActRelu>{}); break;
        case kActGelu: body(std::integral_constant<int, kActGelu>{}); break;
        case kActGeluTanh: body(std::integral_constant<int, kActGeluTanh>{}); break;
        case kActSilu: body(std::integral_constant<int, kActSilu>{}); break;
        default: body(std::integral_constant<int, kActNone>{}); break;
    }
}

}  // namespace mip
