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

// 1 / (1 + e^-x).  The fast exponential is off by 2 + |1.16 x| units in the last place, at most 1e-5
// relative where the result is above 1e-35; e^-x = infinity gives the limit 0.
__device__ __forceinline__ float sigmoid(float x) { return __fdividef(1.0f, 1.0f + __expf(-x)); }

// 2 sqrt(2/pi) (x + 0.044715 x^3): tanh(y/2) = 2 sigmoid(y) - 1 turns the tanh form of the Gaussian
// error unit, x (1 + tanh(sqrt(2/pi) (x + 0.044715 x^3))) / 2, into x sigmoid(gelu_inner(x)).
constexpr float kGeluC = 1.5957691216057308f, kGeluC3 = 0.044715f;
__device__ __forceinline__ float gelu_inner(float x) { return kGeluC * x * (1.0f + kGeluC3 * x * x); }

template <int kAct>
__device__ __forceinline__ float activation(float x) {
    if (kAct == kActRelu) return x < 0.0f ? 0.0f : x;           // (NaN stays NaN)
    if (kAct == kActGelu) return 0.5f * x * (1.0f + erff(x * 0.70710678118654752f));
    if (kAct == kActGeluTanh) return x * sigmoid(gelu_inner(x));
    if (kAct == kActSilu) return x * sigmoid(x);
    return x;
}

// The activation and its derivative, which share the exponential.
template <int kAct>
__device__ __forceinline__ void activation_slope(float x, float& value, float& slope) {
    if (kAct == kActRelu) {
        value = x < 0.0f ? 0.0f : x;
        slope = x > 0.0f ? 1.0f : 0.0f;                         // (0 at 0)
    } else if (kAct == kActGelu) {
        const float cdf = 0.5f * (1.0f + erff(x * 0.70710678118654752f));
        value = x * cdf;
        slope = cdf + x * 0.3989422804014327f * __expf(-0.5f * x * x);
    } else if (kAct == kActGeluTanh) {
        const float e = sigmoid(gelu_inner(x));
        value = x * e;
        slope = e + value * (1.0f - e) * kGeluC * (1.0f + 3.0f * kGeluC3 * x * x);
    } else if (kAct == kActSilu) {
        const float e = sigmoid(x);
        value = x * e;
        slope = e * (1.0f + x * (1.0f - e));
    } else {
        value = x;
        slope = 1.0f;
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
